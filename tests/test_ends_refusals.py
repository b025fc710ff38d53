"""What the operators at a language model's two ends accept and refuse, without a GPU and on one: the calls name a device that no machine has, so that one whose
arguments are fine ends with an error of the device, and nothing is ever enqueued."""
import pytest
import torch

from paper_1805_10032_b200 import build as zbuild
from paper_1805_10032_b200 import zeno

INVALID, UNSUPPORTED, ACCEPTED = zeno.ERR_INVALID_ARG, zeno.ERR_UNSUPPORTED, zeno.ERR_CUDA
NOWHERE = 4095
P = 0x1000           # an address that is checked and never read
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    zbuild.build()
    return zeno.load_library()


def rows(row=64, group=640, data=P):
    return zeno.RowsDesc(data, row, group)


def embed(lib, **k):
    a = dict(device=NOWHERE, type=0, ptype=1, tokens=P, m=2, n=10, vocab=100, cols=64, table=P, ldt=6400, scale=1.0, y=rows())
    a.update(k)
    return lib.zeno_embed(*a.values(), None)


def embed_gradient(lib, **k):
    a = dict(device=NOWHERE, type=0, ptype=1, tokens=P, dy=rows(), m=2, n=10, vocab=100, cols=64, scale=1.0, add=0, table=P, ldt=6400, ws=P, bytes=1 << 50)
    a.update(k)
    return lib.zeno_embed_gradient(*a.values(), None)


def logprobs(lib, **k):
    a = dict(device=NOWHERE, type=0, ptype=1, x=rows(), m=2, n=10, cols=64, vocab=100, w=P, ldw=0, targets=P, scale=1.0, lp=P, lse=P, ws=P, bytes=1 << 50)
    a.update(k)
    return lib.zeno_linear_logprobs(*a.values(), None)


def gradient(lib, **k):
    a = dict(device=NOWHERE, type=0, ptype=1, x=rows(), m=2, n=10, cols=64, vocab=100, w=P, ldw=0, targets=P, scale=1.0, lse=P, g=P, dx=rows(), dw=P, lddw=6400,
             ws=P, bytes=1 << 50)
    a.update(k)
    return lib.zeno_linear_logprobs_gradient(*a.values(), None)


CALLS = {f.__name__: f for f in (embed, embed_gradient, logprobs, gradient)}
ROWS = {"embed": ("y",), "embed_gradient": ("dy",), "logprobs": ("x",), "gradient": ("x", "dx")}
OUTS = {"embed": ("y",), "gradient": ("dx",)}
NEEDED = {"embed": ("tokens", "table", "y"), "embed_gradient": ("tokens", "dy", "table", "ws"), "logprobs": ("x", "w", "targets", "ws"),
          "gradient": ("x", "w", "targets", "lse", "g", "ws")}
MAY_MISS = {"logprobs": ("lp", "lse"), "gradient": ("dx", "dw")}
MATRIX = {"embed": ("table", "ldt", True), "embed_gradient": ("table", "ldt", False), "logprobs": ("w", "ldw", True), "gradient": ("w", "ldw", True)}


@pytest.mark.parametrize("name", sorted(CALLS))
def test_sizes_types_and_scalars(lib, name):
    call = CALLS[name]
    assert call(lib) == ACCEPTED
    for t in (-1, 2):
        assert call(lib, type=t) == INVALID and call(lib, ptype=t) == INVALID
    assert call(lib, m=-1) == INVALID and call(lib, n=-1) == INVALID and call(lib, vocab=0) == INVALID and call(lib, cols=0) == INVALID
    assert call(lib, m=65536) == UNSUPPORTED and call(lib, n=1 << 31) == UNSUPPORTED and call(lib, n=1 << 30) == UNSUPPORTED
    assert call(lib, vocab=(1 << 24) + 1) == UNSUPPORTED and call(lib, cols=(1 << 20) + 1) == UNSUPPORTED
    for s in (NAN, INF, -INF):
        assert call(lib, scale=s) == INVALID
    assert call(lib, scale=-2.0) == ACCEPTED and call(lib, scale=0.0) == ACCEPTED


@pytest.mark.parametrize("name", sorted(CALLS))
def test_rows_and_matrices(lib, name):
    call = CALLS[name]
    for arg in ROWS[name]:
        assert call(lib, **{arg: rows(63, 640)}) == INVALID and call(lib, **{arg: rows(64, 639)}) == INVALID       # rows, and groups, over one another
        assert call(lib, **{arg: rows(data=P + 2)}) == INVALID                                                     # no multiple of an entry's size
        assert call(lib, **{arg: rows(128, 64)}) == ACCEPTED                                                       # groups side by side
        assert call(lib, **{arg: rows((1 << 44) + 1)}) == INVALID
        assert call(lib, **{arg: rows(64, 0)}) == (INVALID if arg in OUTS.get(name, ()) else ACCEPTED)             # one group for all
    at, ld, shared = MATRIX[name]
    assert call(lib, **{ld: 6399}) == INVALID and call(lib, **{ld: 6401}) == ACCEPTED and call(lib, **{ld: 0}) == (ACCEPTED if shared else INVALID)
    assert call(lib, **{at: P + 1}) == INVALID and call(lib, **{at: P + 2}) == ACCEPTED
    assert call(lib, **{ld: 3, "m": 1}) == ACCEPTED                                                                # of a single group
    if name == "gradient":
        assert call(lib, lddw=6399) == INVALID and call(lib, lddw=0) == INVALID and call(lib, dw=P + 1) == INVALID
        assert call(lib, lddw=0, dw=None) == ACCEPTED


@pytest.mark.parametrize("name", sorted(CALLS))
def test_pointers(lib, name):
    call = CALLS[name]
    for arg in NEEDED[name]:
        assert call(lib, **{arg: None}) == INVALID, arg
    for arg in MAY_MISS.get(name, ()):
        assert call(lib, **{arg: None}) == ACCEPTED, arg
    for arg in ("tokens", "targets", "lp", "lse", "g"):
        if arg in NEEDED[name] + MAY_MISS.get(name, ()):
            assert call(lib, **{arg: P + 2}) == INVALID, arg
    if name == "gradient":
        assert call(lib, dx=None, dw=None) == zeno.OK                          # nothing is wanted
    # no groups, or no tokens: nothing to do, but weight gradients become zero
    assert call(lib, m=0) == zeno.OK
    none = dict(n=0, **{a: None for a in NEEDED[name] if a in ("tokens", "targets", "lse", "g")})
    assert call(lib, **none) == (zeno.OK if name in ("embed", "logprobs") else ACCEPTED)


@pytest.mark.parametrize("n", [1, 7, 300])
def test_workspaces(lib, n):
    r = rows(64, 64 * n)
    need = lib.zeno_embed_gradient_workspace(2, n, 100, 64)
    assert need > 0
    assert embed_gradient(lib, n=n, dy=r, bytes=need) == ACCEPTED and embed_gradient(lib, n=n, dy=r, bytes=need - 1) == INVALID
    assert embed_gradient(lib, n=n, dy=r, ws=P + 8) == INVALID
    for type in (0, 1):
        for ptype in (0, 1):
            for w, ldw in ((P, 0), (P, 6400), (P + 4, 6400)):
                need = lib.zeno_linear_logprobs_workspace(type, ptype, 2, n, 64, 100, w, ldw)
                a = dict(type=type, ptype=ptype, n=n, x=r, w=w, ldw=ldw)
                assert need > 0
                assert logprobs(lib, **a, bytes=need) == ACCEPTED and logprobs(lib, **a, bytes=need - 1) == INVALID and logprobs(lib, **a, ws=P + 8) == INVALID
                for dx in (None, r):
                    need = lib.zeno_linear_logprobs_gradient_workspace(type, ptype, 2, n, 64, 100, w, ldw, dx is not None)
                    assert need > 0
                    assert gradient(lib, **a, dx=dx, bytes=need) == ACCEPTED and gradient(lib, **a, dx=dx, bytes=need - 1) == INVALID
                    assert gradient(lib, **a, dx=dx, ws=P + 8) == INVALID
    # what cannot be asked for takes no workspace
    assert lib.zeno_embed_gradient_workspace(2, -1, 100, 64) == 0 and lib.zeno_embed_gradient_workspace(0, 3, 100, 64) == 0
    assert lib.zeno_linear_logprobs_workspace(0, 0, 2, n, 64, 100, None, 0) == 0 and lib.zeno_linear_logprobs_workspace(3, 0, 2, n, 64, 100, P, 0) == 0
    assert lib.zeno_linear_logprobs_gradient_workspace(0, 0, 2, n, 64, 0, P, 0, 1) == 0


def test_the_binding_refuses_what_does_not_fit():
    """Shapes, types and devices are looked at before the library is asked."""
    t, x, w = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3, 8), torch.zeros(5, 8)
    for call in (lambda: zeno.embed(t, w), lambda: zeno.embed_gradient(t, x, torch.zeros(2, 5, 8)), lambda: zeno.linear_logprobs(x, w, t),
                 lambda: zeno.linear_logprobs_gradient(x, w, t, torch.zeros(2, 3), torch.zeros(2, 3)), lambda: zeno.embed(t.view(1, 1, 6), w)):
        with pytest.raises(ValueError):
            call()
