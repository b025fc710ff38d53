"""How near the gradients of the log probabilities from hidden states come to their definitions in 64 bits: bounds that leave no room for more than the kernels'
own roundings."""
import pytest
import torch

from paper_1805_10032_b200 import zeno

import ends_ref as E
import operators_ref as R

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _library():
    from paper_1805_10032_b200 import build as zbuild
    zbuild.build()
    assert torch.cuda.is_available(), "these tests need a CUDA device"
    zeno.load_library()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _head(g, m, n, cols, vocab, act, par, models):
    w = torch.randn(*((m,) if models else ()), vocab, cols, generator=g, device="cuda") * (2.0 / cols ** 0.5)
    return torch.randn(m, n, cols, generator=g, device="cuda").to(act), w.to(par)


def _two_terms(x, w, t, lse, gl):
    """One group's (dx, dw, their slacks) where D is held as two bfloat16 terms: the first is off by 2^-8 of D, the second by 2^-8 of that.  D's logits are summed
    as lse's are (ends_ref); its products with w and x in stretches of at most 1,024 indices, 64 truncating steps of 2 U each (those of the second term, 2^-8 of
    the sums, are 0.5 U together), stretches, tiles that are cut (80 parts at most) and pieces added to nearest."""
    x, w = x.double(), w.double()
    z, off = E.logits(x, w, 1.0)
    L, gs = lse.double().unsqueeze(-1), gl.double().unsqueeze(-1)
    hot = torch.zeros_like(z).scatter_(-1, t.long().unsqueeze(-1), 1.0)
    p = torch.exp(z - L)
    d = gs * (hot - p)
    # the logits', the argument's roundings, the exponential's own error
    p_off = p * (torch.expm1(off + R.U * L.abs() + 4 * R.U * (z - L).abs()) + 8 * R.U)
    d_off = gs.abs() * p_off
    d_off = d_off + (2.0 ** -16 + 2 * R.U) * (d.abs() + d_off)
    size = d.abs() + d_off
    products = lambda terms: (2 * 64 + 1 + terms / 1024 + 24 + 80) * R.U  # noqa: E731
    return d @ w, d.T @ x, d_off @ w.abs() + products(len(w)) * (size @ w.abs()), d_off.T @ x.abs() + products(len(x)) * (size.T @ x.abs())


# a token or a few of each worker, where a result hangs on one entry of D; workers with weights of their own; more tokens; long contractions of few tiles
@pytest.mark.parametrize("m,n,cols,vocab,models", [(1, 1, 264, 700, False), (17, 1, 264, 700, False), (2, 1, 520, 300, True), (21, 5, 96, 513, True), (1, 300, 1032, 2000, False),
                                                   (3, 333, 77, 1000, False), (16, 61, 136, 3003, False), (2, 40, 4096, 300, True), (1, 700, 4096, 130, False), (1, 2600, 64, 30000, False)])
def test_bfloat16_operands_gradients_are_off_by_their_own_rounding(m, n, cols, vocab, models):
    g = _gen(cols + vocab)
    x, w = _head(g, m, n, cols, vocab, BF16, BF16, models)
    t = torch.randint(0, vocab, (m, n), generator=g, device="cuda").int()
    gl = torch.randn(m, n, generator=g, device="cuda")
    lse = zeno.linear_logprobs(x, w, t).lse
    dw = torch.empty(m, vocab, cols, device="cuda", dtype=BF16)
    dx = zeno.linear_logprobs_gradient(x, w, t, lse, gl, dweight=dw)
    for i in range(m):
        want = _two_terms(x[i], w[i] if models else w, t[i], lse[i], gl[i])
        R.assert_near(dx[i], want[0], want[2], "dx")
        R.assert_near(dw[i], want[1], want[3], "dw")
    zeno.check_operator_status()


# whole logits, of few and many tokens, a narrow and a wide layer, and (of 4096 columns) logits in parts of the contraction
@pytest.mark.parametrize("n,cols", [(2, 64), (40, 64), (300, 1200), (2, 4096), (40, 4096)])
@pytest.mark.parametrize("first", [1.0, 7.3])
@pytest.mark.parametrize("act,par", [(F32, F32), (BF16, F32), (F32, BF16), (BF16, BF16)])
def test_gradients_of_a_word_whose_logits_are_minus_a_lot(n, cols, first, act, par):
    """A word whose weights are finite and whose logits are -3e38, or beyond binary32 and so minus infinity, has probability zero: its gradient is zero, and dx is
    what it is without that word."""
    g = _gen(n + cols)
    vocab, m = 300, 1
    x, w = _head(g, m, n, cols, vocab, act, par, False)
    x[..., 0] = first
    w[0] = 0.0
    w[0, 0] = -3e38
    t = torch.randint(1, vocab, (m, n), generator=g, device="cuda").int()
    gl = torch.randn(m, n, generator=g, device="cuda")
    got = zeno.linear_logprobs(x, w, t)
    want = E.logprobs(x, w[1:], t - 1, 1.0)
    R.assert_near(got.logprobs, want[0], want[2], "logprobs")
    R.assert_near(got.lse, want[1], want[3], "lse")
    dw = torch.full((m, vocab, cols), float("nan"), device="cuda", dtype=par)
    dx = zeno.linear_logprobs_gradient(x, w, t, got.lse, gl, dweight=dw)
    ref = E.logprobs_gradient(x, w[1:], t - 1, got.lse, gl, 1.0, BF16 if act == par == BF16 else F32)
    R.assert_near(dx, ref[0], ref[2], "dx")
    R.assert_near(dw[:, 1:], ref[1], ref[3], "dw")
    assert (dw[:, 0] == 0).all()
    # as the target of the first token: D of it is g, and that word's gradient g times the hidden states
    t[0, 0] = 0
    gl[0, 0] = 0.25
    got = zeno.linear_logprobs(x, w, t)
    assert torch.isfinite(got.lse).all() and (got.logprobs[0, 0] < -2.9e38)
    dx = zeno.linear_logprobs_gradient(x, w, t, got.lse, gl, dweight=dw)
    # g times the word's entry: the largest product of terms, each of three bfloat16 terms' products off by 4 U of the sum of their magnitudes
    R.assert_near(dx[0, 0, 0], 0.25 * w[0, 0].double().cpu(), 100 * R.U * 0.25 * 3e38, "dx")
    R.assert_near(dx[0, 1:], ref[0][0, 1:], ref[2][0, 1:], "dx of the others")
    own = 0.25 * x[0, 0].double()
    R.assert_near(dw[0, 0], own, 100 * R.U * own.abs(), "dw")
    assert torch.isfinite(dw).all() and torch.isfinite(dx).all()


@pytest.mark.parametrize("m,n,cols,vocab", [(2, 332, 667, 93), (3, 57, 777, 5001), (16, 61, 1024, 3203)])
@pytest.mark.parametrize("act,par", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)])
def test_gradients_are_as_near_to_64_bits_as_plain_products_in_binary32(m, n, cols, vocab, act, par):
    """Of confident tokens (whose D is a small difference of a probability from one): the norm of what dx and dweight are off by is no larger than that of products
    in binary32 whose results are rounded once; in bfloat16, where both are that rounding, by no more than a hundredth."""
    g = _gen(cols)
    w = (torch.randn(vocab, cols, generator=g, device="cuda") * (2.5 / cols ** 0.5)).to(par)
    t = torch.randint(0, vocab, (m, n), generator=g, device="cuda").int()
    x = (torch.randn(m, n, cols, generator=g, device="cuda") + w.float()[t.long()] * 0.96).to(act)
    gl = torch.randn(m, n, generator=g, device="cuda") / n
    hot = torch.nn.functional.one_hot(t.long(), vocab)

    def gradients(kind):
        xs, ws = x.to(kind), w.to(kind)
        lse = torch.logsumexp(xs.double() @ ws.double().transpose(-1, -2), -1).float()        # the same for all
        d = (hot - torch.exp(xs @ ws.T - lse.to(kind).unsqueeze(-1))) * gl.to(kind).unsqueeze(-1)
        return lse, d @ ws, d.transpose(-1, -2) @ xs

    allowed = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    try:
        lse, *want = gradients(torch.float64)
        _, dx, dw = gradients(F32)
    finally:
        torch.backends.cuda.matmul.allow_tf32 = allowed
    own_dw = torch.empty(m, vocab, cols, device="cuda", dtype=par)
    own_dx = zeno.linear_logprobs_gradient(x, w, t, lse, gl, dweight=own_dw)
    for got, plain, exact in ((own_dx, dx.to(act), want[0]), (own_dw, dw.to(par), want[1])):
        off, plain_off = ((v.double() - exact).norm() for v in (got, plain))
        assert off <= (1.01 if got.dtype == BF16 else 1.0) * plain_off, (float(off / plain_off))
    zeno.check_operator_status()


@pytest.mark.parametrize("m,n", [(32, 64), (33, 2), (500, 3), (4000, 1), (9, 250)])
@pytest.mark.parametrize("act", [F32, BF16])
def test_many_workers_of_few_tokens(m, n, act):
    """Workers that share weights, few tokens each, some without a target: every one's log probabilities, lse and gradient."""
    g = _gen(m)
    cols, vocab = 40, 70
    x, w = _head(g, m, n, cols, vocab, act, act, False)
    t = torch.randint(-20, vocab, (m, n), generator=g, device="cuda").int()
    gl = torch.randn(m, n, generator=g, device="cuda")
    got = zeno.linear_logprobs(x, w, t)
    flat = lambda v: v.reshape(1, m * n, *v.shape[2:])  # noqa: E731
    want = E.logprobs(flat(x), w, flat(t), 1.0)
    R.assert_near(flat(got.logprobs), want[0], want[2], "logprobs")
    R.assert_near(flat(got.lse), want[1], want[3], "lse")
    dw = torch.full((m, vocab, cols), float("nan"), device="cuda", dtype=act)
    dx = zeno.linear_logprobs_gradient(x, w, t, got.lse, gl, dweight=dw)
    for i in range(0, m, max(1, m // 40)):
        ref = E.logprobs_gradient(x[i:i + 1], w, t[i:i + 1], got.lse[i:i + 1], gl[i:i + 1], 1.0, act)
        R.assert_near(dx[i:i + 1], ref[0], ref[2], "dx")
        R.assert_near(dw[i:i + 1], ref[1], ref[3], "dw")
    assert torch.isfinite(dw).all()
    zeno.check_operator_status()
