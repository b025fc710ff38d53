"""A language model's two ends on the GPU against their definitions in 64 bits: sizes from one token to many, odd and unaligned ones, strides, tokens that
carry nothing, values that are not finite, other streams, captured graphs, and a whole step of tied weights."""
import pytest
import torch

from paper_1805_10032_b200 import zeno

import ends_ref as E
import operators_ref as R

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
INF, NAN = float("inf"), float("nan")
TYPES = [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)]


@pytest.fixture(scope="module", autouse=True)
def _library():
    from paper_1805_10032_b200 import build as zbuild
    zbuild.build()
    assert torch.cuda.is_available(), "these tests need a CUDA device"
    zeno.load_library()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _tokens(g, m, n, vocab, masked=0.2):
    t = torch.randint(0, vocab, (m, n), generator=g, device="cuda")
    t[torch.rand(m, n, generator=g, device="cuda") < 0.2] = vocab // 3                     # one that is frequent
    t = torch.where(torch.rand(m, n, generator=g, device="cuda") < masked, -1, t)
    if masked and n > 3:
        t[:, 1], t[:, 2] = vocab, -(2 ** 31)                                              # neither is in the vocabulary
    return t.int()


def _slice(m, width, dtype, pad=0, fill=NAN):
    """A slice of the rows of V, and V: what lies around it is NaN."""
    V = torch.full((m, 32 + pad + width + 40), fill, device="cuda", dtype=dtype)
    return V[:, 32 + pad: 32 + pad + width], V


def _around_is_nan(V, width, pad=0):
    assert torch.isnan(V[:, : 32 + pad]).all() and torch.isnan(V[:, 32 + pad + width:]).all()


def _rows(v, layout):
    m, n, cols = v.shape
    if layout == "dense":
        return v.contiguous()
    if layout == "padded":
        t = torch.full((m, n, cols + 3), NAN, device="cuda", dtype=v.dtype)
        t[..., 1:1 + cols] = v
        return t[..., 1:1 + cols]
    if layout == "interleaved":
        t = torch.full((n, m, cols), NAN, device="cuda", dtype=v.dtype).transpose(0, 1)
        t.copy_(v)
        return t
    return v[:1].expand(m, n, cols)


EMBED = [(1, 1, 1, 1), (1, 1, 32000, 4096), (2, 3, 5, 7), (3, 70, 50, 33), (2, 9, 1000, 264), (4, 33, 777, 1025), (21, 2, 100, 64), (1, 300, 4099, 520), (2, 5, 17, 16384)]


@pytest.mark.parametrize("m,n,vocab,cols", EMBED)
@pytest.mark.parametrize("act,par", TYPES)
def test_embed(m, n, vocab, cols, act, par):
    g = _gen(vocab + cols)
    tokens = _tokens(g, m, n, vocab)
    for pad in (0, 1):
        tables, P = _slice(m, vocab * cols, par, pad)
        tables.copy_(torch.randn(m, vocab * cols, generator=g, device="cuda"))
        tables = tables.unflatten(1, (vocab, cols))
        for table in (tables, tables[0]):
            R.assert_near(zeno.embed(tokens, table, scale=2.5, dtype=act), *E.embed(tokens, table, 2.5), "new")
            out = torch.full((m, n + 1, cols + 8 + pad), NAN, device="cuda", dtype=act)
            zeno.embed(tokens, table, scale=-0.3, out=out[:, :n, pad:pad + cols])
            want, off = E.embed(tokens, table, -0.30000001192092896)
            R.assert_near(out[:, :n, pad:pad + cols], want, off, "into")
            assert torch.isnan(out[:, n:]).all() and torch.isnan(out[..., pad + cols:]).all() and torch.isnan(out[..., :pad]).all()
    flat = zeno.embed(tokens[0], tables[0], dtype=act)
    assert flat.shape == (n, cols) and torch.equal(flat, zeno.embed(tokens, tables, dtype=act)[0])


GRADIENT = [(1, 1, 1, 1), (1, 1, 3000, 512), (2, 3, 5, 7), (3, 70, 50, 33), (2, 900, 11, 264), (4, 333, 777, 1025), (21, 40, 100, 64), (1, 5000, 4099, 520),
            (2, 129, 17, 4096), (1, 20000, 40, 24), (3, 1, 2, 3), (2, 0, 70, 40)]


@pytest.mark.parametrize("m,n,vocab,cols", GRADIENT)
@pytest.mark.parametrize("act,par", TYPES)
def test_embed_gradient(m, n, vocab, cols, act, par):
    g = _gen(vocab + cols)
    tokens = _tokens(g, m, n, vocab)
    dy = torch.randn(m, n, cols, generator=g, device="cuda").to(act)
    for pad, layout in ((0, "dense"), (1, "padded"), (0, "interleaved"), (3, "shared")):
        d = _rows(dy, layout)
        into, V = _slice(m, vocab * cols, par, pad)
        into = into.unflatten(1, (vocab, cols))
        assert zeno.embed_gradient(tokens, d, into, scale=1.5) is into
        R.assert_near(into, *E.embed_gradient(tokens, d, vocab, 1.5), layout)
        _around_is_nan(V, vocab * cols, pad)
        first = into.clone()
        zeno.embed_gradient(tokens, d, into, scale=1.5)
        assert torch.equal(first, into)                        # the same bits
        before = torch.randn(m, vocab, cols, generator=g, device="cuda").to(par)
        into.copy_(before)
        zeno.embed_gradient(tokens, d, into, scale=1.5, add=True)
        R.assert_near(into, *E.embed_gradient(tokens, d, vocab, 1.5, before), "added")
        _around_is_nan(V, vocab * cols, pad)


def test_embed_gradient_of_one_row_and_of_none():
    """Every token the same; no token in the vocabulary, whose dy is not read; all of a tokens' sum in few bits off."""
    n, cols = 30000, 520
    for dtype in (F32, BF16):
        dy = torch.full((1, n, cols), 0.1, device="cuda").to(dtype)
        into = torch.full((1, 7, cols), NAN, device="cuda")
        zeno.embed_gradient(torch.full((1, n), 3, device="cuda", dtype=torch.int32), dy, into)
        want = n * dy[0, 0].double()
        assert ((into[0, 3].double() - want).abs() <= 90 * R.U * want).all()
        assert (into[0, [0, 1, 2, 4, 5, 6]] == 0).all()
        into.fill_(NAN)
        zeno.embed_gradient(torch.full((1, n), 7, device="cuda", dtype=torch.int32), torch.full_like(dy, NAN), into)
        assert (into == 0).all()


def _head(g, m, n, cols, vocab, act, par, models=False, scale=1.0):
    w = torch.randn(*((m,) if models else ()), vocab, cols, generator=g, device="cuda") * (2.0 / scale / cols ** 0.5)
    return torch.randn(m, n, cols, generator=g, device="cuda").to(act), w.to(par)


HEAD = [(1, 1, 1, 1), (1, 1, 4096, 1000), (2, 3, 7, 5), (3, 70, 33, 300), (2, 9, 264, 1000), (1, 130, 1025, 257), (5, 65, 64, 128), (2, 300, 520, 777), (1, 1000, 96, 5000),
        (17, 2, 40, 513), (1, 257, 2048, 2049), (2, 64, 136, 64), (1, 2, 8192, 70)]


@pytest.mark.parametrize("m,n,cols,vocab", HEAD)
@pytest.mark.parametrize("act,par", TYPES)
def test_linear_logprobs(m, n, cols, vocab, act, par):
    g = _gen(vocab + cols)
    targets = _tokens(g, m, n, vocab)
    for models, layout, scale in ((False, "dense", 1.0), (True, "padded", 0.25), (True, "interleaved", -1.5)):
        x, w = _head(g, m, n, cols, vocab, act, par, models, scale)
        if models and layout == "padded":                      # slices of parameter vectors, wherever they begin
            held, _ = _slice(m, vocab * cols, par, 1)
            held.copy_(w.flatten(1))
            w = held.unflatten(1, (vocab, cols))
        x[targets < 0] = NAN                                   # hidden states of padding are not read
        x[targets >= vocab] = INF
        clean = torch.where(((targets >= 0) & (targets < vocab)).unsqueeze(-1), x, 0.0)
        got = zeno.linear_logprobs(_rows(x, layout), w, targets, scale=scale)
        want = E.logprobs(clean, w, targets, scale)
        R.assert_near(got.logprobs, want[0], want[2], layout)
        R.assert_near(got.lse, want[1], want[3], layout)
        again = zeno.linear_logprobs(_rows(x, layout), w, targets, scale=scale)
        assert torch.equal(got.logprobs, again.logprobs) and torch.equal(got.lse, again.lse)
    zeno.check_operator_status()


@pytest.mark.parametrize("m,n,cols,vocab", HEAD)
@pytest.mark.parametrize("act,par", TYPES)
def test_linear_logprobs_gradient(m, n, cols, vocab, act, par):
    g = _gen(vocab + cols + 1)
    targets = _tokens(g, m, n, vocab)
    wider = F32 if F32 in (act, par) else BF16
    given = (targets >= 0) & (targets < vocab)
    for models, layout, pad, scale in ((False, "dense", 0, 1.0), (True, "padded", 1, 0.25)):
        x, w = _head(g, m, n, cols, vocab, act, par, models, scale)
        x[~given] = NAN
        clean = torch.where(given.unsqueeze(-1), x, 0.0)
        lse = torch.where(given, E.logprobs(clean, w, targets, scale)[1], NAN).float()
        gl = torch.where(given, torch.randn(m, n, generator=g, device="cuda"), NAN)
        into, V = _slice(m, vocab * cols, par, pad)
        into = into.unflatten(1, (vocab, cols))
        dx = zeno.linear_logprobs_gradient(_rows(x, layout), w, targets, lse, gl, dweight=into, scale=scale)
        want = E.logprobs_gradient(clean, w, targets, lse, gl, scale, wider)
        R.assert_near(dx, want[0], want[2], "dx " + layout)
        R.assert_near(into, want[1], want[3], "dw " + layout)
        _around_is_nan(V, vocab * cols, pad)
        first = into.clone()
        again = zeno.linear_logprobs_gradient(_rows(x, layout), w, targets, lse, gl, dweight=into, scale=scale)
        assert torch.equal(again, dx) and torch.equal(first, into)
        out = torch.full((m, n, cols + 5), NAN, device="cuda", dtype=act)
        zeno.linear_logprobs_gradient(_rows(x, layout), w, targets, lse, gl, dx=out[..., 2:2 + cols], scale=scale)
        assert torch.equal(out[..., 2:2 + cols], dx) and torch.isnan(out[..., :2]).all() and torch.isnan(out[..., 2 + cols:]).all()
        into.fill_(NAN)
        assert zeno.linear_logprobs_gradient(_rows(x, layout), w, targets, lse, gl, dweight=into, want_dx=False, scale=scale) is None
        assert torch.equal(first, into)
    zeno.check_operator_status()


@pytest.mark.parametrize("act,par", [(F32, F32), (BF16, BF16)])
def test_waits_that_run_out_are_reported(act, par):
    """With no polls allowed every wait on the tensor cores' path that is not satisfied at once gives up; the next call is sound."""
    g = _gen(5)
    m, n, cols, vocab = 2, 150, 264, 700
    targets = _tokens(g, m, n, vocab, 0.0)
    x, w = _head(g, m, n, cols, vocab, act, par)
    want = zeno.linear_logprobs(x, w, targets)
    gl = torch.ones(m, n, device="cuda")
    dw = torch.empty(m, vocab, cols, device="cuda", dtype=par)
    dx = zeno.linear_logprobs_gradient(x, w, targets, want.lse, gl, dweight=dw)
    kept = dw.clone()
    zeno.check_operator_status()
    zeno.debug_set_operator_wait_limit(0)
    try:
        zeno.linear_logprobs(x, w, targets)
        with pytest.raises(zeno.ZenoError) as e:
            zeno.check_operator_status()
        assert e.value.status == zeno.ERR_TIMEOUT
        zeno.linear_logprobs_gradient(x, w, targets, want.lse, gl, dweight=dw)
        with pytest.raises(zeno.ZenoError):
            zeno.check_operator_status()
    finally:
        zeno.debug_set_operator_wait_limit(1 << 22)
    again = zeno.linear_logprobs(x, w, targets)
    assert torch.equal(again.logprobs, want.logprobs) and torch.equal(again.lse, want.lse)
    assert torch.equal(zeno.linear_logprobs_gradient(x, w, targets, want.lse, gl, dweight=dw), dx) and torch.equal(dw, kept)
    zeno.check_operator_status()
