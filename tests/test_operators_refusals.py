"""What the language model operators refuse, without a GPU: the C calls answer with status codes before anything is enqueued, the binding raises."""
import ctypes

import pytest
import torch

from paper_1805_10032_b200 import build as zbuild
from paper_1805_10032_b200 import zeno

INVALID, UNSUPPORTED = zeno.ERR_INVALID_ARG, zeno.ERR_UNSUPPORTED
P = 0x1000           # an address that is checked and never read


@pytest.fixture(scope="module")
def lib():
    zbuild.build()
    return zeno.load_library()


def rows(row=64, group=640, data=P):
    return zeno.RowsDesc(data, row, group)


def norm(lib, **k):
    a = dict(device=0, type=0, ptype=1, x=rows(), m=2, n=10, cols=64, w=P, b=P, ldw=0, eps=1e-5, y=rows(), mean=P, rstd=P)
    a.update(k)
    return lib.zeno_layer_norm(*a.values(), None)


def norm_gradient(lib, **k):
    a = dict(device=0, type=0, ptype=1, dy=rows(), x=rows(), codes=None, scales=None, m=2, n=10, cols=64, w=P, ldw=0, mean=P, rstd=P, dx=rows(), dw=P,
             db=P, ldg=64, ws=P, bytes=1 << 40)
    a.update(k)
    return lib.zeno_layer_norm_gradient(*a.values(), None)


def pack(lib, **k):
    a = dict(device=0, type=0, x=rows(), m=2, n=10, cols=64, codes=rows(), scales=rows(1, 10))
    a.update(k)
    return lib.zeno_pack_activations(*a.values(), None)


def dense(lib, **k):
    a = dict(device=0, type=0, ptype=1, dy=rows(), codes=rows(), scales=rows(1, 10), m=2, n=10, inputs=64, outputs=64, dw=P, ldw=4096, db=P, ldb=64, ws=P,
             bytes=1 << 40)
    a.update(k)
    return lib.zeno_dense_gradient(*a.values(), None)


def logprobs(lib, **k):
    a = dict(device=0, type=0, z=rows(), m=2, n=10, vocab=64, t=P, top=2, lp=P, entropy=P, lse=P, idx=P, top_lp=P)
    a.update(k)
    return lib.zeno_token_logprobs(*a.values(), None)


def gradient(lib, **k):
    a = dict(device=0, type=0, z=rows(), m=2, n=10, vocab=64, t=P, lse=P, entropy=P, g=P, gh=P, out=rows())
    a.update(k)
    return lib.zeno_token_gradient(*a.values(), None)


CALLS = {f.__name__: f for f in (norm, norm_gradient, pack, dense, logprobs, gradient)}
SIZE = {"norm": "cols", "norm_grad": "cols", "norm_gradient": "cols", "pack": "cols", "dense": "inputs", "logprobs": "vocab", "gradient": "vocab"}
ROWS = {"norm": ("x", "y"), "norm_gradient": ("dy", "x", "dx"), "pack": ("x", "codes", "scales"), "dense": ("dy", "codes", "scales"),
        "logprobs": ("z",), "gradient": ("z", "out")}
OUT = {"norm": "y", "norm_gradient": "dx", "pack": "codes", "gradient": "out"}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_sizes_types_and_rows(lib, name):
    call = CALLS[name]
    if not torch.cuda.is_available():                      # accepted: what is missing is the device
        assert call(lib) == zeno.ERR_CUDA
    assert call(lib, type=2) == INVALID and call(lib, type=-1) == INVALID
    assert call(lib, m=-1) == INVALID and call(lib, n=-1) == INVALID and call(lib, **{SIZE[name]: 0}) == INVALID
    assert call(lib, m=65536) == UNSUPPORTED and call(lib, n=1 << 31) == UNSUPPORTED and call(lib, m=2, n=1 << 30) == UNSUPPORTED
    assert call(lib, **{SIZE[name]: (1 << 30) + 1}) == UNSUPPORTED
    for arg in ROWS[name]:
        if arg == "dx":
            continue
        assert call(lib, **{arg: None}) == INVALID or arg == "x" and name == "norm_gradient"
    for arg in ROWS[name]:
        width = 1 if arg == "scales" else 64
        assert call(lib, **{arg: rows(width, 10 * width, None)}) == INVALID, arg
        assert call(lib, **{arg: rows(width - 1, 10 * width)}) == INVALID, arg
        assert call(lib, **{arg: rows(-64, 640)}) == INVALID, arg
        assert call(lib, **{arg: rows(width, 10 * width - 1)}) == INVALID, arg
        assert call(lib, **{arg: rows(1 << 60, 1 << 62)}) == INVALID, arg
    for arg in ROWS[name]:                                 # no address of an entry
        if arg != "codes":
            assert call(lib, **{arg: rows(64, 640, P + 1)}) == INVALID, arg
    if name in OUT:                                        # an input may be shared by the groups, an output not
        assert call(lib, **{OUT[name]: rows(64, 0)}) == INVALID


@pytest.mark.parametrize("name", sorted(CALLS))
def test_nothing_to_do_is_no_error(lib, name):
    none = {k: rows(64, 640, None) for k in ROWS[name]}
    assert CALLS[name](lib, m=0, **none) == zeno.OK
    if name not in ("norm_gradient", "dense"):             # those write zeros
        assert CALLS[name](lib, n=0, **none) == zeno.OK


def test_misplaced_addresses(lib):
    for call, names in ((norm, ("w", "b", "mean", "rstd")), (norm_gradient, ("w", "mean", "rstd", "dw", "db")), (dense, ("dw", "db")),
                        (logprobs, ("t", "lp", "entropy", "lse", "idx", "top_lp")), (gradient, ("t", "lse", "entropy", "g", "gh"))):
        for name in names:
            assert call(lib, **{name: P + 1}) == INVALID, (call.__name__, name)


def test_widths_of_weight_gradients(lib):
    wide = (1 << 20) + 8
    r = rows(wide, 10 * wide)
    assert norm_gradient(lib, cols=wide, dy=r, x=r, dx=r, ldg=wide) == UNSUPPORTED
    assert dense(lib, inputs=wide, codes=r) == UNSUPPORTED and dense(lib, outputs=wide, dy=r) == UNSUPPORTED
    assert lib.zeno_layer_norm_gradient_workspace(1, 1000, wide) == 0


def test_norm_refusals(lib):
    assert norm(lib, ptype=2) == INVALID and norm(lib, w=None) == INVALID and norm(lib, ldw=63) == INVALID
    for eps in (-1e-5, float("nan"), float("inf")):
        assert norm(lib, eps=eps) == INVALID


def test_norm_gradient_refusals(lib):
    f = norm_gradient
    assert f(lib, ptype=9) == INVALID and f(lib, w=None) == INVALID and f(lib, ldw=5) == INVALID
    assert f(lib, mean=None) == INVALID and f(lib, rstd=None) == INVALID and f(lib, ldg=63) == INVALID
    assert f(lib, x=None) == INVALID and f(lib, x=None, codes=rows()) == INVALID
    assert f(lib, x=None, codes=rows(), scales=rows(0, 10)) == INVALID
    need = lib.zeno_layer_norm_gradient_workspace(2, 1000, 4096)
    assert need >= 0
    if need:
        big = dict(n=1000, cols=4096, dy=rows(4096, 4096000), x=rows(4096, 4096000), dx=rows(4096, 4096000), ldg=4096)
        assert f(lib, **big, ws=None) == INVALID and f(lib, **big, bytes=need - 1) == INVALID and f(lib, **big, ws=P + 4) == INVALID
    assert lib.zeno_layer_norm_gradient_workspace(-1, 4, 4) == 0


def test_dense_refusals(lib):
    assert dense(lib, ptype=5) == INVALID and dense(lib, dw=None) == INVALID and dense(lib, ldw=4095) == INVALID and dense(lib, ldb=63) == INVALID
    assert dense(lib, outputs=0) == INVALID and dense(lib, outputs=65) == INVALID and dense(lib, inputs=65) == INVALID
    need = lib.zeno_dense_gradient_workspace(0, rows(), rows(), 2, 10, 64, 64)
    if need:
        assert dense(lib, ws=None) == INVALID and dense(lib, bytes=need - 1) == INVALID and dense(lib, ws=P + 8) == INVALID
    big = rows(4096, 4096 * 1000)
    assert lib.zeno_dense_gradient_workspace(0, big, big, 2, 1000, 4096, 4096) >= 6 * 2 * 1000 * 4096       # three terms of dy
    assert lib.zeno_dense_gradient_workspace(1, big, big, 2, 1000, 4096, 4096) == 0
    assert lib.zeno_dense_gradient_workspace(7, big, big, 2, 1000, 4096, 4096) == 0
    assert lib.zeno_dense_gradient_workspace(1, None, big, 2, 1000, 4096, 4096) == 0


def test_token_refusals(lib):
    assert logprobs(lib, top=-1) == INVALID and logprobs(lib, top=65) == INVALID and logprobs(lib, top=33) == UNSUPPORTED
    assert logprobs(lib, t=None) == INVALID
    for arg in ("t", "lse", "g", "entropy"):
        assert gradient(lib, **{arg: None}) == INVALID


def test_binding_refuses_what_does_not_fit(lib):
    x = torch.zeros(2, 3, 8)
    w = torch.zeros(8)
    t = torch.zeros(2, 3, dtype=torch.int32)
    for call in (lambda: zeno.layer_norm(x, w), lambda: zeno.pack_activations(x), lambda: zeno.token_logprobs(x, t),
                 lambda: zeno.token_gradient(x, t, x[..., 0], x[..., 0]), lambda: zeno.layer_norm_gradient(x, x, w, x[..., 0], x[..., 0]),
                 lambda: zeno.dense_gradient(x, zeno.Saved(x, x), x)):
        with pytest.raises(ValueError, match="CUDA"):
            call()


def test_binding_checks_shapes_types_and_layouts(lib, monkeypatch):
    """With the check of the device out of the way: nothing here reaches the library."""
    monkeypatch.setattr(zeno, "_device", lambda *a: 0)
    monkeypatch.setattr(zeno, "load_library", lambda: ctypes.CDLL(None))
    x = torch.zeros(2, 3, 8)
    w, s, t = torch.zeros(8), torch.zeros(2, 3), torch.zeros(2, 3, dtype=torch.int32)
    codes, scales = torch.zeros(2, 3, 8, dtype=torch.uint8), torch.zeros(2, 3, 1)
    bad = [
        lambda: zeno.layer_norm(x, w[:7]), lambda: zeno.layer_norm(x, torch.zeros(3, 8)), lambda: zeno.layer_norm(x, w, w.bfloat16()),
        lambda: zeno.layer_norm(x, torch.zeros(2, 8), torch.zeros(2, 9)[:, :8]), lambda: zeno.layer_norm(x, w, out=x[:, :2]),
        lambda: zeno.layer_norm(x, w, out=x.bfloat16()), lambda: zeno.layer_norm(x, torch.zeros(8, 2).T[:, ::1]),
        lambda: zeno.layer_norm_gradient(x, x.bfloat16(), w, s, s), lambda: zeno.layer_norm_gradient(x, x[:, :2], w, s, s),
        lambda: zeno.layer_norm_gradient(x, (codes, scales.double()), w, s, s), lambda: zeno.layer_norm_gradient(x, (codes[..., :7], scales), w, s, s),
        lambda: zeno.layer_norm_gradient(x, (x, scales), w, s, s), lambda: zeno.layer_norm_gradient(x, x, w, s[:1], s),
        lambda: zeno.layer_norm_gradient(x, x, w, s.T.contiguous().T, s), lambda: zeno.layer_norm_gradient(x, x, w, s, s.double()),
        lambda: zeno.layer_norm_gradient(x, x, w, s, s, w), lambda: zeno.layer_norm_gradient(x, x, w, s, s, torch.zeros(2, 8, dtype=torch.bfloat16)),
        lambda: zeno.layer_norm_gradient(x, x, w, s, s, torch.zeros(2, 8), torch.zeros(2, 9)[:, :8]),
        lambda: zeno.layer_norm_gradient(x, x, w, s, s, dx=x[:, :, :4]),
        lambda: zeno.dense_gradient(x, (codes, scales), torch.zeros(2, 8, 7)), lambda: zeno.dense_gradient(x, (codes, scales), torch.zeros(2, 8, 16)[..., :8]),
        lambda: zeno.dense_gradient(x, (codes, scales), torch.zeros(2, 8, 8), torch.zeros(8)),
        lambda: zeno.dense_gradient(x[:, :2], (codes, scales), torch.zeros(2, 8, 8)),
        lambda: zeno.token_logprobs(x, t.long()), lambda: zeno.token_logprobs(x, t[:, :2]),
        lambda: zeno.token_gradient(x, t, s, s, g_entropy=s), lambda: zeno.token_gradient(x, t, s[:1], s), lambda: zeno.token_gradient(x, t, s, s, out=x[:1]),
    ]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(f"call {k} was accepted")


def test_operators_say_what_type_or_layout_they_need(monkeypatch, lib):
    monkeypatch.setattr(zeno, "_device", lambda *a: 0)
    with pytest.raises(ValueError, match="bfloat16"):
        zeno._type(torch.zeros(2, dtype=torch.float16), "x")
    for t in (torch.zeros(4), torch.zeros(2, 2, 2, 2), torch.zeros(2, 3, 8)[..., ::2], torch.zeros(8, 3).T):
        with pytest.raises(ValueError):
            zeno._rows(t, "x")
