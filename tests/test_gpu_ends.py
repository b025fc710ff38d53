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
            (2, 129, 17, 4096), (1, 20000, 40, 24), (2, 40000, 9, 100), (3, 1, 2, 3), (2, 0, 70, 40)]


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


@pytest.mark.parametrize("m,n,cols,vocab", [(2, 150, 264, 700), (1, 60, 264, 3000), (1, 60, 4096, 300), (1, 300, 4096, 300)])
@pytest.mark.parametrize("act,par", [(F32, F32), (BF16, BF16)])
def test_waits_that_run_out_are_reported(m, n, cols, vocab, act, par):
    """With no polls allowed every wait on the tensor cores' path that is not satisfied at once gives up, of pairs of blocks and single ones, of whole logits and
    those in parts; the next call is sound."""
    g = _gen(5)
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


def test_the_binding_refuses_what_does_not_fit():
    m, n, cols, vocab = 2, 3, 8, 5
    t = torch.zeros(m, n, device="cuda", dtype=torch.int32)
    x, w = torch.zeros(m, n, cols, device="cuda"), torch.zeros(vocab, cols, device="cuda")
    p = torch.zeros(m, n, device="cuda")
    dw = torch.zeros(m, vocab, cols, device="cuda")
    good = zeno.linear_logprobs(x, w, t)
    assert torch.allclose(good.lse, torch.full_like(p, 5.0).log())
    bad = [lambda: zeno.embed(t.long(), w), lambda: zeno.embed(t, w.half()), lambda: zeno.embed(t, w[:, ::2]), lambda: zeno.embed(t, w.expand(3, vocab, cols)),
           lambda: zeno.embed(t.t(), w), lambda: zeno.embed(t, w, out=x[:, :2]), lambda: zeno.embed(t, w, dtype=BF16, out=x),
           lambda: zeno.embed_gradient(t, x, w), lambda: zeno.embed_gradient(t, x[..., :7], dw), lambda: zeno.embed_gradient(t[:, :2], x, dw),
           lambda: zeno.embed_gradient(t, x, dw.expand(m, vocab, cols)[:1]), lambda: zeno.linear_logprobs(x, w[:, :7], t), lambda: zeno.linear_logprobs(x, w, t.float()),
           lambda: zeno.linear_logprobs(x, w.t().contiguous().t(), t), lambda: zeno.linear_logprobs(x, w, t.cpu()),
           lambda: zeno.linear_logprobs_gradient(x, w, t, p.double(), p), lambda: zeno.linear_logprobs_gradient(x, w, t, p, p[:, :2]),
           lambda: zeno.linear_logprobs_gradient(x, w, t, p, p, dweight=dw.to(BF16)), lambda: zeno.linear_logprobs_gradient(x, w, t, p, p, dweight=dw[0]),
           lambda: zeno.linear_logprobs_gradient(x, w, t, p, p, dx=x[:, :2])]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            raise AssertionError(k)
    # a gradient that all groups would write to the same place is the library's to refuse
    with pytest.raises(zeno.ZenoError):
        zeno.embed_gradient(t, x, dw[:1].expand(m, vocab, cols))


def test_no_tokens_and_no_groups():
    for act, par in TYPES:
        V = torch.full((3, 70), NAN, device="cuda", dtype=par)
        dw = V[:, 5:65].unflatten(1, (6, 10))
        x, t = torch.zeros(3, 0, 10, device="cuda", dtype=act), torch.zeros(3, 0, device="cuda", dtype=torch.int32)
        w = torch.ones(6, 10, device="cuda", dtype=par)
        p = torch.zeros(3, 0, device="cuda")
        assert zeno.embed(t, w).shape == (3, 0, 10) and zeno.linear_logprobs(x, w, t).lse.shape == (3, 0)
        for write in (lambda: zeno.embed_gradient(t, x, dw), lambda: zeno.linear_logprobs_gradient(x, w, t, p, p, dweight=dw)):
            V.fill_(NAN)
            write()
            assert (dw == 0).all() and torch.isnan(V[:, :5]).all() and torch.isnan(V[:, 65:]).all()
        V.fill_(1.0)
        zeno.embed_gradient(t, x, dw, add=True)
        assert (V == 1).all()
        empty = torch.zeros(0, 4, 10, device="cuda", dtype=act), torch.zeros(0, 4, device="cuda", dtype=torch.int32)
        assert zeno.embed(empty[1], w).shape == (0, 4, 10) and zeno.linear_logprobs(empty[0], w, empty[1]).lse.shape == (0, 4)
        # tokens, none of which carries anything: gradients are zero, nothing is read
        x, t = torch.full((3, 70, 10), NAN, device="cuda", dtype=act), torch.full((3, 70), -1, device="cuda", dtype=torch.int32)
        p = torch.full((3, 70), NAN, device="cuda")
        s = zeno.linear_logprobs(x, w, t)
        assert (s.lse == 0).all() and (s.logprobs == 0).all()
        V.fill_(NAN)
        assert (zeno.linear_logprobs_gradient(x, w, t, p, p, dweight=dw) == 0).all() and (dw == 0).all()


@pytest.mark.parametrize("n", [2, 40])
@pytest.mark.parametrize("act", [F32, BF16])
def test_values_that_are_not_finite(act, n):
    """One row's infinity or NaN is that row's; a word whose logits are minus infinity has probability zero."""
    g = _gen(n)
    cols, vocab = 64, 300
    x, w = _head(g, 1, n, cols, vocab, act, act)
    t = torch.randint(1, vocab, (1, n), generator=g, device="cuda").int()
    clean = zeno.linear_logprobs(x, w, t)
    for value in (NAN, INF):
        y = x.clone()
        y[0, 1, 7] = value
        got = zeno.linear_logprobs(y, w, t)
        assert torch.isnan(got.lse[0, 1]) and torch.isnan(got.logprobs[0, 1])
        assert torch.equal(got.lse[0, :1], clean.lse[0, :1]) and torch.equal(got.lse[0, 2:], clean.lse[0, 2:])
        dx = zeno.linear_logprobs_gradient(y, w, t, got.lse, torch.ones(1, n, device="cuda"))
        assert torch.isnan(dx[0, 1]).all() and torch.isfinite(dx[0, 0]).all() and torch.isfinite(dx[0, 2:]).all()
    # hidden states with a positive first entry, and a word that only has minus a lot there
    x = x.abs()
    w = w.clone()
    w[0] = 0.0
    w[0, 0] = -3e38
    x[..., 0] = 1.0
    got = zeno.linear_logprobs(x, w, t)
    want = E.logprobs(x, w[1:], t - 1, 1.0)                     # without that word
    R.assert_near(got.logprobs, want[0], want[2], "logprobs")
    R.assert_near(got.lse, want[1], want[3], "lse")
    # and as the target
    t[0, 0] = 0
    got = zeno.linear_logprobs(x, w, t)
    assert got.logprobs[0, 0] < -2.9e38 and torch.isfinite(got.lse).all()


BIG = [(60, 5, 40, 300, True, F32, F32), (60, 70, 72, 200, True, BF16, BF16), (1, 5000, 72, 600, False, BF16, BF16), (2, 3000, 64, 9000, False, F32, F32),
       (1, 2600, 2100, 3000, False, BF16, BF16), (1, 14, 8192, 12000, False, F32, F32), (3, 900, 100, 40000, False, BF16, F32),
       (3, 70, 6000, 300, True, BF16, BF16), (2, 200, 5000, 513, True, F32, BF16), (1, 600, 7001, 255, False, BF16, F32), (9, 1, 4096, 90, False, BF16, BF16),
       (1, 4100, 64, 70000, False, BF16, BF16)]


@pytest.mark.parametrize("m,n,cols,vocab,models,act,par", BIG)
def test_many_groups_tiles_and_pieces(m, n, cols, vocab, models, act, par):
    """More groups than shared memory has room for, more rows than a band, a vocabulary of several pieces, tiles that are cut, logits in parts."""
    g = _gen(m + n)
    targets = _tokens(g, m, n, vocab)
    x, w = _head(g, m, n, cols, vocab, act, par, models)
    given = (targets >= 0) & (targets < vocab)
    clean = torch.where(given.unsqueeze(-1), x, 0.0)
    want = E.logprobs(clean, w, targets, 1.0)
    got = zeno.linear_logprobs(x, w, targets)
    R.assert_near(got.logprobs, want[0], want[2], "logprobs")
    R.assert_near(got.lse, want[1], want[3], "lse")
    gl = torch.randn(m, n, generator=g, device="cuda")
    into, V = _slice(m, vocab * cols, par)
    into = into.unflatten(1, (vocab, cols))
    dx = zeno.linear_logprobs_gradient(x, w, targets, got.lse, gl, dweight=into)
    for i in range(0, m, 1 if m < 5 else 13):
        wi = w[i:i + 1] if models else w
        ref = E.logprobs_gradient(clean[i:i + 1], wi, targets[i:i + 1], got.lse[i:i + 1], gl[i:i + 1], 1.0, F32 if F32 in (act, par) else BF16)
        R.assert_near(dx[i:i + 1], ref[0], ref[2], "dx")
        R.assert_near(into[i:i + 1], ref[1], ref[3], "dw")
    _around_is_nan(V, vocab * cols)
    zeno.check_operator_status()


def test_gradients_against_differences():
    """In binary32, the loss's slope along a direction against both gradients."""
    g = _gen(9)
    m, n, cols, vocab, scale = 1, 20, 48, 90, 0.7
    x, w = _head(g, m, n, cols, vocab, F32, F32, scale=scale)
    t = torch.randint(0, vocab, (m, n), generator=g, device="cuda").int()
    gl = torch.randn(m, n, generator=g, device="cuda")
    s = zeno.linear_logprobs(x, w, t, scale=scale)
    dw = torch.empty(m, vocab, cols, device="cuda")
    dx = zeno.linear_logprobs_gradient(x, w, t, s.lse, gl, dweight=dw, scale=scale)
    ux, uw = torch.randn_like(x), torch.randn_like(w) * 0.1

    def loss(h):
        z = scale * ((x + h * ux).double() @ (w + h * uw).double().T)
        return (torch.log_softmax(z, -1).gather(-1, t.long().unsqueeze(-1)).squeeze(-1) * gl).sum()

    h = 2.0 ** -10
    slope = (loss(h) - loss(-h)) / (2 * h)
    along = (dx.double() * ux).sum() + (dw[0].double() * uw).sum()
    # the third derivative's share is h^2/6 of a few units, x + h u rounds to 2^-24 of itself
    assert abs(float(slope - along)) <= 2e-4 * float((dx * ux).abs().sum() + (dw[0] * uw).abs().sum())
    # the embedding: linear, so that a difference is exact but for rounding
    table, dy = torch.randn(vocab, cols, generator=g, device="cuda"), torch.randn(m, n, cols, generator=g, device="cuda")
    de = zeno.embed_gradient(t, dy, torch.empty(1, vocab, cols, device="cuda"), scale=scale)
    u = torch.randn_like(table)
    change = ((zeno.embed(t, table + u, scale=scale).double() - zeno.embed(t, table - u, scale=scale).double()) / 2 * dy.double()).sum()
    assert abs(float(change - (de[0].double() * u).sum())) <= 1e-5 * float((de[0] * u).abs().sum())


def test_offsets_beyond_32_bits():
    """Tables, gradients and rows of more than 2^31 entries."""
    g = _gen(3)
    cols, vocab = 4096, (1 << 19) + 77
    table = torch.zeros(vocab, cols, device="cuda", dtype=BF16)
    at = torch.tensor([[0, vocab - 1, 300000, vocab - 1, -1, (1 << 19) + 3]], device="cuda", dtype=torch.int32)
    rows = at[0, [0, 1, 2, 5]].long()
    table[rows] = torch.randn(4, cols, generator=g, device="cuda").to(BF16)
    y = zeno.embed(at, table, scale=2.0)
    R.assert_near(y, *E.embed(at, table, 2.0))
    far = torch.empty((1 << 31) + 8 + 6 * cols, device="cuda", dtype=BF16).as_strided((2, 3, cols), ((1 << 31) + 8, cols, 1))
    far.copy_(y.view(2, 3, cols))
    two = torch.full((2 * vocab * cols + 8,), NAN, device="cuda", dtype=BF16)
    dtable = two[8:].view(2, vocab, cols)
    zeno.embed_gradient(at.view(2, 3), far, dtable)
    for i in range(2):
        ids = at.view(2, 3)[i]
        want = torch.zeros(4, cols, device="cuda", dtype=torch.float64)
        for k in range(3):
            want += torch.where((rows == ids[k]).unsqueeze(1), far[i, k].double(), 0.0)
        R.assert_near(dtable[i, rows], want, 4 * R.U * want.abs(), "row sums")
        dtable[i, rows] = 0
        assert not dtable[i].any()
    # the same table as output weights: nearly all logits are zero
    x = torch.randn(1, 2, cols, generator=g, device="cuda").to(BF16) / 64
    t = torch.tensor([[vocab - 1, 5]], device="cuda", dtype=torch.int32)
    for n in (2, 6):
        xs, ts = x.repeat(1, n // 2, 1), t.repeat(1, n // 2)
        got = zeno.linear_logprobs(xs, table, ts)
        z = xs[0].double() @ table[rows].double().T
        lse = torch.log((vocab - 4) + z.exp().sum(-1))
        off = 200 * R.U * (1 + (xs[0].double().abs() @ table[rows].double().abs().T).amax(-1))
        R.assert_near(got.lse[0], lse, off, "lse")
        zt = torch.where(ts[0] == vocab - 1, z[:, 1], 0.0)
        R.assert_near(got.logprobs[0], zt - lse, 2 * off, "logprobs")
    gl = torch.ones(1, 2, device="cuda")
    s = zeno.linear_logprobs(x, table, t)
    two.fill_(NAN)
    dx = zeno.linear_logprobs_gradient(x, table, t, s.lse, gl, dweight=dtable[:1])
    p = torch.exp(-s.lse[0].double())
    for word in (5, 12345, vocab - 2):
        want = (((t[0] == word).double() - p).unsqueeze(1) * x[0].double()).sum(0)
        R.assert_near(dtable[0, word], want, (2.0 ** -15 + 1e-5) * ((((t[0] == word).double() + p).unsqueeze(1)) * x[0].double().abs()).sum(0), "dw")
    assert torch.isfinite(dtable[0]).all() and torch.isnan(two[:8]).all() and torch.isfinite(dx).all()


def _every_call(seed, stream=None, act=BF16, m=3, n=65, cols=136, vocab=1000):
    """Both ends once; returns their outputs, and the inputs that a later pass may change."""
    g = _gen(seed)
    t = _tokens(g, m, n, vocab)
    x, w = _head(g, m, n, cols, vocab, act, act)
    gl = torch.randn(m, n, generator=g, device="cuda")
    V = torch.zeros(m, vocab * cols, device="cuda", dtype=act)
    dw = V.unflatten(1, (vocab, cols))
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())

    def run():
        y = zeno.embed(t, w, scale=3.0, stream=stream)
        s = zeno.linear_logprobs(x, w, t, stream=stream)
        one = zeno.linear_logprobs(x[:, :1].contiguous() if stream is None else x, w, t[:, :1].contiguous() if stream is None else t, stream=stream)
        dx = zeno.linear_logprobs_gradient(x, w, t, s.lse, gl, dweight=dw, stream=stream)
        zeno.embed_gradient(t, dx, dw, scale=3.0, add=True, stream=stream)
        return [y, *s, one.lse[:, :1], dx, V]
    return run, (x, t, gl)


@pytest.mark.parametrize("act", [F32, BF16])
def test_the_same_bits_again_and_on_another_stream(act):
    run, _ = _every_call(1, act=act)
    first = [v.clone() for v in run()]
    assert all(torch.equal(p, q) for p, q in zip(first, run()))
    side = torch.cuda.Stream()
    torch.cuda._sleep(20_000_000)                               # the default stream is busy: nothing may be waited for there
    run, _ = _every_call(1, stream=side, act=act)
    got = run()
    side.synchronize()
    for k, (p, q) in enumerate(zip(first, got)):
        if k != 3:                                              # there all of the tokens, here one of each group
            assert torch.equal(p, q), k


@pytest.mark.parametrize("act", [F32, BF16])
def test_captured_and_replayed_on_other_values(act):
    run, inputs = _every_call(4, act=act)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = run()
    fresh, other = _every_call(5, act=act)
    for p, q in zip(inputs, other):                             # other tokens, and other ones of them that carry nothing
        p.copy_(q)
    want = [v.clone() for v in run()]
    for v in outs:
        v.zero_()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(outs, want))
    del fresh


def test_two_graphs_replayed_side_by_side():
    made = []
    for seed in (6, 7):
        run, _ = _every_call(seed)
        want = [v.clone() for v in run()]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = run()
        made.append((graph, outs, want, run))                   # run holds the inputs that the graph reads
    streams = [torch.cuda.Stream() for _ in made]
    torch.cuda.synchronize()
    for _ in range(5):
        for (graph, *_), s in zip(made, streams):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for _, outs, want, _ in made:
        assert all(torch.equal(p, q) for p, q in zip(outs, want))


@pytest.mark.parametrize("act", [F32, BF16])
def test_calls_that_follow_one_another(act):
    """Calls of other sizes right behind each other, their workspaces in the same memory, on two streams at once."""
    sizes = [(1, 1, 64, 500), (2, 300, 64, 500), (1, 40, 1031, 70), (3, 9, 264, 2000)]
    made = []
    for k, (m, n, cols, vocab) in enumerate(sizes):
        g = _gen(k)
        t = _tokens(g, m, n, vocab, 0.0)
        x, w = _head(g, m, n, cols, vocab, act, act)
        gl = torch.randn(m, n, generator=g, device="cuda")
        s = zeno.linear_logprobs(x, w, t)
        torch.cuda.synchronize()
        dw = torch.empty(m, vocab, cols, device="cuda", dtype=act)
        dx = zeno.linear_logprobs_gradient(x, w, t, s.lse, gl, dweight=dw)
        torch.cuda.synchronize()
        de = zeno.embed_gradient(t, x, torch.empty_like(dw))
        torch.cuda.synchronize()
        made.append((x, w, t, gl, s, dx, dw, de))
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for turn in range(6):
        for k, (x, w, t, gl, s, dx, dw, de) in enumerate(made):
            with torch.cuda.stream(streams[(turn + k) % 2]):
                a, b, c = zeno.linear_logprobs(x, w, t), torch.empty_like(dw), torch.empty_like(dw)
                d = zeno.linear_logprobs_gradient(x, w, t, s.lse, gl, dweight=b)
                zeno.embed_gradient(t, x, c)
                got.append((k, a, d, b, c))
    torch.cuda.synchronize()
    for k, a, d, b, c in got:
        _, _, _, _, s, dx, dw, de = made[k]
        assert torch.equal(a.lse, s.lse) and torch.equal(a.logprobs, s.logprobs) and torch.equal(d, dx) and torch.equal(b, dw) and torch.equal(c, de), k


def test_workers_gradients_of_a_tied_language_model_and_the_step_on_them():
    """Workers' gradients of a small model whose embedding is its output layer (embedding, norm layer, token loss) through the operators into the rows of V,
    against the derivatives in 64 bits; then a failure, the candidates' losses on the server's tokens, and the average of the best."""
    m, n, cols, vocab, scale = 6, 33, 96, 250, 4.0
    g = _gen(11)
    d = vocab * cols + 2 * cols
    params = torch.cat([0.3 * torch.randn(vocab * cols, generator=g, device="cuda"), torch.ones(cols, device="cuda"), torch.zeros(cols, device="cuda")])
    text = torch.randint(0, vocab, (m, n + 1), generator=g, device="cuda").int()
    t, nxt = text[:, :-1].contiguous(), text[:, 1:].contiguous()
    t[:, -4:], nxt[:, -5:] = -1, -1                             # padding, and the last token has no next one

    def split(v):
        return v[..., :vocab * cols].unflatten(-1, (vocab, cols)), v[..., vocab * cols:vocab * cols + cols], v[..., vocab * cols + cols:d]

    W, w, b = split(params)
    V = torch.full((m, d + 32), NAN, device="cuda")
    dW, dw, db = split(V[:, :d])
    h = zeno.embed(t, W, scale=scale)
    y, mean, rstd = zeno.layer_norm(h, w, b)
    s = zeno.linear_logprobs(y, W, nxt, scale=0.2)
    count = int((nxt[0] >= 0).sum())
    dy = zeno.linear_logprobs_gradient(y, W, nxt, s.lse, torch.full((m, n), -1.0 / count, device="cuda"), dweight=dW, scale=0.2)
    dh = zeno.layer_norm_gradient(dy, h, w, mean, rstd, dw, db)
    zeno.embed_gradient(t, dh, dW, scale=scale, add=True)
    leaves = [p.double().repeat(m, *([1] * p.dim())).requires_grad_(True) for p in (W, w, b)]
    losses = []
    for i in range(m):
        hi = torch.where((t[i] >= 0).unsqueeze(-1), scale * leaves[0][i][t[i].clamp(min=0).long()], 0.0)
        yi = torch.nn.functional.layer_norm(hi, (cols,), leaves[1][i], leaves[2][i], eps=1e-5)
        lp = torch.log_softmax(0.2 * yi @ leaves[0][i].T, -1)
        losses.append(-(lp.gather(-1, nxt[i].clamp(min=0).long().unsqueeze(-1)).squeeze(-1) * (nxt[i] >= 0)).sum() / count)
    grads = torch.autograd.grad(sum(losses), leaves)
    for i in range(m):
        assert abs(float(-s.logprobs[i].sum() / count - losses[i].detach())) <= 1e-5
    for got, want in zip((dW, dw, db), grads):
        assert float((got.double() - want).norm() / want.norm()) <= 1e-5
    assert torch.isnan(V[:, d:]).all()
    with zeno.Zeno(zeno.LOSS_LEAST_SQUARES, zeno.F32, (d, 1), False, m_max=m, n_r_max=4) as z:
        z.inject_faults(V, torch.tensor([2], device="cuda", dtype=torch.int32), zeno.FAULT_SCALE, -20.0)
        models = torch.cat([params.unsqueeze(0), params - 0.5 * V[:, :d]])
        mW, mw, mb = split(models)
        batch = torch.randint(0, vocab, (1, 41), generator=g, device="cuda").int()
        ids, following = batch[:, :-1].repeat(m + 1, 1), batch[:, 1:].repeat(m + 1, 1)
        hidden, _, _ = zeno.layer_norm(zeno.embed(ids, mW, scale=scale), mw, mb)
        loss = -zeno.linear_logprobs(hidden, mW, following, scale=0.2).logprobs.double().mean(-1)
        scores = (loss[0] - loss[1:] - 1e-4 * (V[:, :d].double() ** 2).sum(-1)).float()
        assert int(scores.argmin()) == 2                        # the failure
        kept = z.select(scores, 2)
        assert 2 not in kept.tolist()
        average = z.aggregate(V, kept)
        want = V[kept.long(), :d].double().mean(0)
        assert float((average.double() - want).norm() / want.norm()) <= 1e-6
    zeno.check_operator_status()


@pytest.mark.parametrize("m,n,cols,vocab,act,par", [(33, 5, 96, 700, F32, BF16), (17, 21, 200, 300, BF16, BF16), (50, 1, 264, 513, BF16, F32), (9, 33, 1100, 257, F32, F32),
                                                    (5, 17, 4096, 300, BF16, BF16), (20, 130, 72, 90, BF16, BF16)])
def test_workers_of_few_tokens_keep_to_themselves(m, n, cols, vocab, act, par):
    """Workers that share weights and whose tokens lie next to one another: one worker's NaN reaches no other's gradient, nor does what memory held before."""
    g = _gen(m * n)
    targets = _tokens(g, m, n, vocab)
    targets[1] = -1
    targets[2, -1] = vocab - 1
    x, w = _head(g, m, n, cols, vocab, act, par, False)
    given = (targets >= 0) & (targets < vocab)
    x = torch.where(given.unsqueeze(-1), x, NAN)
    clean = torch.where(given.unsqueeze(-1), x, 0.0)
    gl = torch.where(given, torch.randn(m, n, generator=g, device="cuda"), NAN)
    for bad in (False, True):
        if bad:
            x[2, -1, cols // 2] = NAN
        stale = torch.full((64 << 20,), NAN, device="cuda")
        del stale
        got = zeno.linear_logprobs(x, w, targets)
        rest = [i for i in range(m) if i != 2 or not bad]
        want = E.logprobs(clean, w, targets, 1.0)
        R.assert_near(got.logprobs[rest], want[0][rest], want[2][rest], "logprobs")
        R.assert_near(got.lse[rest], want[1][rest], want[3][rest], "lse")
        stale = torch.full((64 << 20,), NAN, device="cuda")
        del stale
        dw = torch.full((m, vocab, cols), NAN, device="cuda", dtype=par)
        dx = zeno.linear_logprobs_gradient(x, w, targets, torch.where(given, got.lse, NAN), gl, dweight=dw)
        for i in rest[:: 1 if m < 10 else 5] + [1]:
            ref = E.logprobs_gradient(clean[i:i + 1], w, targets[i:i + 1], got.lse[i:i + 1], torch.where(given, gl, 0.0)[i:i + 1], 1.0, F32 if F32 in (act, par) else BF16)
            R.assert_near(dx[i:i + 1], ref[0], ref[2], "dx")
            R.assert_near(dw[i:i + 1], ref[1], ref[3], "dw")
        assert torch.isfinite(dw[rest]).all() and torch.isfinite(dx[rest]).all()
        if bad:
            assert torch.isnan(got.lse[2, -1]) and torch.isnan(dx[2, -1]).all() and torch.isnan(dw[2]).all()
    zeno.check_operator_status()
