"""Calls of the language model operators at the ends of their ranges: magnitudes next to binary32's, sums of many terms, logits far from zero,
layouts that only the C ABI makes, reports of waits that ran out."""
import numpy as np
import pytest
import torch

from paper_1805_10032_b200 import zeno

import operators_ref as R

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module", autouse=True)
def _library():
    from paper_1805_10032_b200 import build as zbuild
    zbuild.build()
    assert torch.cuda.is_available(), "these tests need a CUDA device"
    zeno.load_library()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _rows(g, m, n, cols, dtype, scale=1.0):
    return (torch.randn(m, n, cols, generator=g, device="cuda") * scale).to(dtype)


@pytest.mark.parametrize("cols", [8, 132, 136, 520, 1032, 2056, 4104, 5000])
@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("saved", [False, True])
def test_layer_norm_gradient_of_large_constant_rows(cols, act, saved):
    """Finite statistics whose product is beyond binary32 (a constant row of 2^112: mean rstd is 2^120 and more; eps 2^-16 to 2^-96): columns that no
    entry of the row has must not reach its averages.  h is zero in such a row, so dx = rstd (g - avg(g)) and dweight is zero."""
    g = _gen(cols)
    m, n = 2, 19
    x = torch.full((m, n, cols), 2.0 ** 112, device="cuda").to(act)
    mean = torch.full((m, n), 2.0 ** 112, device="cuda")
    rstd = (2.0 ** torch.linspace(8, 48, n, device="cuda").round()).expand(m, n).contiguous()
    dy = torch.randn(m, n, cols, generator=g, device="cuda").to(act)
    w = 1 + 0.2 * torch.randn(cols, generator=g, device="cuda")
    source = zeno.pack_activations(x) if saved else x
    dw, db = torch.full((m, cols), NAN, device="cuda"), torch.full((m, cols), NAN, device="cuda")
    dx = zeno.layer_norm_gradient(dy, source, w, mean, rstd, dw, db)
    want = R.norm_gradient(dy, x, w, mean, rstd)
    # the slacks without what stands for the rounding of x - mean, which is exact here
    g64 = dy.double() * w.double()
    size = rstd.double().unsqueeze(-1) * (g64.abs() + g64.abs().mean(-1, keepdim=True))
    R.assert_near(dx, want[0], (cols / 32 + 40) * R.U * size, "dx")
    assert torch.equal(dw, torch.zeros_like(dw))
    R.assert_near(db, want[2], want[5], "db")


# 40 tiles and more, so that a tile's sum over the tokens is not cut into parts; binary32 dy in three terms, up to where the small ones fill stretches
@pytest.mark.parametrize("n,act,par", [(2048, F32, F32), (8192, BF16, F32), (8192, F32, F32), (32768, BF16, F32), (70000, F32, F32), (8200, BF16, BF16),
                                       (140000, F32, BF16)])
def test_dense_gradient_of_many_tokens_is_summed_in_binary32(n, act, par):
    """All products positive.  The tensor core adds 16 tokens at a time and truncates: off by less than a step of binary32, 2^-23 of the sum.  Its
    sums go on after at most 1,024 tokens (64 additions; 4,096 and 256 into bfloat16, with up to 65,536 and 262,144 of the two small terms before, 2^-8
    of the sum together: 2 * 16,384 * 2^-23 * 2^-8 at most), in n / 1,024 additions to nearest, of half a step each."""
    g = _gen(n)
    inputs, outputs = 2560, 1024
    saved = zeno.pack_activations(torch.rand(1, n, inputs, generator=g, device="cuda").to(BF16))
    dy = torch.rand(1, n, outputs, generator=g, device="cuda").to(act)
    dw, db = torch.full((1, outputs, inputs), NAN, device="cuda", dtype=par), torch.full((1, outputs), NAN, device="cuda", dtype=par)
    zeno.dense_gradient(dy, saved, dw, db)
    zeno.check_operator_status()
    want = torch.zeros(outputs, inputs, device="cuda", dtype=torch.float64)
    for at in range(0, n, 8192):
        want += dy[0, at:at + 8192].double().T @ R.unpack(saved.codes[0, at:at + 8192], saved.scales[0, at:at + 8192])
    additions = 64 if par == F32 else 256
    small = 0 if act == BF16 else min(2 * n / 16, 64 * additions) * 2.0 ** -31
    R.assert_near(dw[0], want, want * (additions * 2.0 ** -23 + small + (n / 1024 + 1) * R.U), "dw")
    R.assert_near(db, dy.double().sum(1), (n + 32) * R.U * dy.double().sum(1), "db")


def test_dense_gradient_keeps_the_small_terms_of_few_tokens():
    """Three terms of 160 tokens in one stretch: 10 truncating additions of the largest term, 2^-23 each, on what the small ones left (2^-8, and 20 more of
    those), and the half step that the result is rounded by."""
    g = _gen(4)
    saved = zeno.pack_activations(torch.rand(8, 160, 512, generator=g, device="cuda").to(BF16))
    dy = 1 + torch.rand(8, 160, 512, generator=g, device="cuda")
    dw = torch.full((8, 512, 512), NAN, device="cuda")
    zeno.dense_gradient(dy, saved, dw)
    zeno.check_operator_status()
    want = dy.double().transpose(1, 2) @ R.unpack(saved.codes, saved.scales)
    R.assert_near(dw, want, want * (10 + 30 / 256) * 2.0 ** -23, "dw")


@pytest.mark.parametrize("vocab,rows", [(64, 3000), (3001, 500), (40000, 600), (140000, 20)])
@pytest.mark.parametrize("act", [F32, BF16])
def test_lse_is_rounded_once_at_its_own_size(vocab, rows, act):
    """Rows of 1, 2 or 4 equal entries and nothing else: lse = v + log k.  Besides the half step of lse there is only what is rounded at the size of log2 S and
    of the remainder (a step of v at most): an exponential and a logarithm, 2^-22 each, and four roundings of at most 3."""
    g = _gen(vocab)
    v = ((torch.rand(rows, generator=g, device="cuda") * 230 + 20) * torch.where(torch.rand(rows, generator=g, device="cuda") < 0.5, -1.0, 1.0)).to(act)
    z = torch.full((rows, vocab), -INF, device="cuda", dtype=act)
    k = 2 ** (torch.arange(rows, device="cuda") % 3)
    for r in range(rows):
        z[r, torch.randperm(vocab, generator=g, device="cuda")[: int(k[r])]] = v[r]
    got = zeno.token_logprobs(z, torch.zeros(rows, device="cuda", dtype=torch.int32), top=1)
    want = v.double() + torch.log(k.double())
    R.assert_near(got.lse, want, 2.0 ** -21 + 12 * R.U, "lse")
    R.assert_near(got.top_logprobs[:, 0], -torch.log(k.double()), 2.0 ** -21 + 12 * R.U, "log probability")


def _gradient_from_logits(z, t, g, gh):
    """The gradient by its definition, in 64 bits, from the logits alone; p and what multiplies it."""
    z = z.double()
    p = torch.softmax(z, -1)
    logp = torch.log_softmax(z, -1)
    h = -torch.where(p > 0, p * logp, 0.0).sum(-1, keepdim=True)
    given = (t >= 0).unsqueeze(-1)
    hot = torch.zeros_like(z).scatter_(-1, t.long().clamp(min=0).unsqueeze(-1), 1.0) * given
    g = g.double().unsqueeze(-1) * given
    factor = g if gh is None else g + gh.double().unsqueeze(-1) * torch.where(p > 0, logp + h, 0.0)
    return g * hot - p * factor, p, factor


@pytest.mark.parametrize("vocab", [1, 9, 1000, 20011, 140001])
@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("with_entropy", [False, True])
def test_token_gradient_of_logits_far_from_zero(vocab, act, with_entropy):
    """Whatever the size of the logits, p is off by 2^-16 of itself at most in binary32: half a step of an lse under 2^8 (2^-17) and an eighth of that each for the
    errors of lse, of the exponential and of a row's sum.  In bfloat16 half a step of an lse under 2^12 (2^-13), 2^-12 in all, beside the result's own.  With the entropy
    log p + H is off by as much, absolutely, and H by 2^-16 of 1 + H.  The rows' gradients of the log probability sum to zero."""
    g = _gen(vocab)
    far = [0.0, 100.0, -250.0, 300.0, 1e3, 5e3, -1e4, 65504.0, 3e5, -5e5, 1e6, 5e6, -3e8]
    n = len(far) + 3
    z = torch.randn(n, vocab, generator=g, device="cuda") * 2
    for r, off in enumerate(far):
        z[r] += off
    z[-3] = -3e38                                                 # masked throughout by the type's lowest, or nearly
    z[-2] -= 1e4
    z[-2, vocab // 2:] = -INF
    z[-1] += 4e4
    z[-1, 1::2] = -3e38
    z = z.to(act)
    t = torch.randint(0, (vocab + 1) // 2, (n,), generator=g, device="cuda", dtype=torch.int32)
    if vocab == 1:
        z[-2] = -1e4
    t[5] = -1
    gl = torch.randn(n, generator=g, device="cuda")
    gh = torch.randn(n, generator=g, device="cuda") if with_entropy else None
    s = zeno.token_logprobs(z, t)
    want, p, factor = _gradient_from_logits(z, t, gl, gh)
    off = 2.0 ** -16 if act == F32 else 2.0 ** -12
    h = gh.double().abs().unsqueeze(-1) if with_entropy else 0.0
    slack = p * off * (factor.abs() + h * (2 + s.entropy.double().unsqueeze(-1))) + 4 * R.U * (p * factor).abs() + 2.0 ** -120
    base = torch.full((n, vocab + 3), NAN, device="cuda", dtype=act)
    for out in (None, base[:, 3:], z):                            # lying otherwise, too; last over the logits
        got = zeno.token_gradient(z, t, s.lse, gl, s.entropy, gh, out=out)
        R.assert_near(got, want, slack, "gradient")
        if act == F32 and not with_entropy:
            total = got.double().sum(-1).abs()
            assert (total <= gl.double().abs() * (off + 2 * R.U) + vocab * 2.0 ** -120).all(), total
    assert torch.isnan(base[:, :3]).all()


# Long sums.  Chains of additions have at most 64 terms along a row (then sums of sums lose next to nothing), and 18 additions join a block's: k = 96.
# A single chain over such a row adds equal terms with the same rounding each time.
@pytest.mark.parametrize("cols", [(1 << 20) - 3, 1 << 20, (1 << 26) + 1])
@pytest.mark.parametrize("act", [F32, BF16])
def test_layer_norm_of_very_long_rows(cols, act):
    g = _gen(cols)
    x = torch.rand(2, cols, generator=g, device="cuda").to(act)
    x[0] = 0.1
    w, b = torch.full((cols,), 1.25, device="cuda"), torch.full((cols,), 0.5, device="cuda")
    y, mean, rstd = zeno.layer_norm(x, w, b, eps=1e-5)
    k, eps = 96 * R.U, float(np.float32(1e-5))
    for r in range(2):
        v = x[r].double()
        m = v.mean()
        want = ((v - m).square().mean() + eps) ** -0.5
        mean_off = k * v.abs().mean()
        rstd_off = want * (k + (mean_off * want) ** 2 + 4 * R.U)
        R.assert_near(mean[r], m, mean_off, "mean")
        R.assert_near(rstd[r], want, rstd_off, "rstd")
        y_off = 1.25 * ((mean_off + 2 * R.U) * want + 4 * (rstd_off + 4 * R.U * want)) + 4 * R.U * 4
        R.assert_near(y[r], 1.25 * (v - m) * want + 0.5, y_off, "y")


@pytest.mark.parametrize("act", [F32, BF16])
def test_layer_norm_gradient_of_very_long_rows(act):
    """Constant rows have h = 0: dx = rstd (g - avg(g)), zero where dy is constant too."""
    cols = (1 << 20) - 1
    x = torch.full((2, cols), 0.25, device="cuda", dtype=act)
    dy = torch.full((2, cols), 0.1, device="cuda", dtype=act)
    dy[1] = torch.rand(cols, generator=_gen(1), device="cuda").to(act)
    w = torch.ones(cols, device="cuda")
    mean, rstd = torch.full((2,), 0.25, device="cuda"), torch.full((2,), 300.0, device="cuda")
    dx = zeno.layer_norm_gradient(dy, x, w, mean, rstd)
    d = dy.double()
    R.assert_near(dx, 300 * (d - d.mean(-1, keepdim=True)), 300 * (96 + 8) * R.U * (d.abs() + d.mean(-1, keepdim=True)), "dx")


@pytest.mark.parametrize("cols,rows_side_by_side", [(5, 1), (8, 8)])
def test_layer_norm_weight_gradients_over_many_rows(cols, rows_side_by_side):
    """600 groups leave a block to each; 4,096 rows at most make a chain."""
    m, n = 600, 131072
    x = torch.full((1, n, cols), 0.3, device="cuda").expand(m, n, cols)
    dy = torch.full((1, n, cols), 0.1, device="cuda").expand(m, n, cols)
    mean, rstd = torch.zeros(m, n, device="cuda"), torch.ones(m, n, device="cuda")
    dw, db = torch.full((m, cols), NAN, device="cuda"), torch.full((m, cols), NAN, device="cuda")
    zeno.layer_norm_gradient(dy, x, torch.ones(cols, device="cuda"), mean, rstd, dw, db, want_dx=False)
    a, b = float(np.float32(0.1)), float(np.float32(0.3))
    k = (4096 / rows_side_by_side + 64) * R.U
    R.assert_near(dw, torch.full((m, cols), n * a * b), n * a * b * (k + 3 * R.U), "dw")
    R.assert_near(db, torch.full((m, cols), n * a), n * a * k, "db")


def test_token_logprobs_and_gradient_of_very_long_rows():
    """One largest entry and 2^26 equal ones: S = 1 + (vocab - 1) e^-0.35.  Besides the sums an exponential, 2^-21, and the logarithm."""
    vocab = (1 << 26) + 3
    d = float(np.float32(-0.3125))
    for off in (0.0, 1024.0):
        z = torch.full((1, vocab), off + d, device="cuda")
        z[0, 7] = off
        t = torch.full((1,), 7, device="cuda", dtype=torch.int32)
        s = zeno.token_logprobs(z, t, top=2)
        S = 1 + (vocab - 1) * np.exp(d)
        lse = off + np.log(S)
        S_off = 96 * R.U + 2.0 ** -20
        R.assert_near(s.lse, torch.tensor([lse]), S_off + 20 * R.U, "lse")
        R.assert_near(s.logprobs, torch.tensor([-np.log(S)]), S_off + 40 * R.U, "log probability")
        H = np.log(S) - (vocab - 1) * np.exp(d) * d / S
        R.assert_near(s.entropy, torch.tensor([H]), 4 * S_off + 60 * R.U, "entropy")
        assert s.top_idx.tolist() == [[7, 0]]
        grad = zeno.token_gradient(z, t, s.lse, torch.ones(1, device="cuda"))
        p = torch.full((1, vocab), np.exp(d) / S, device="cuda", dtype=torch.float64)
        want = -p
        want[0, 7] = 1 - 1 / S
        R.assert_near(grad, want, p * 2.0 ** -16 + 4 * R.U * (want == want[0, 7]), "gradient")


def test_dense_gradient_over_very_many_rows():
    """One tile of 2^24 rows: on the tensor cores in 74 parts of 222 stretches (64 truncating additions), and the sums of dY in chains of 1,024."""
    n, inputs, outputs = (1 << 24) + 5, 16, 8
    saved = zeno.Saved(torch.full((n, inputs), 0x38, device="cuda", dtype=torch.uint8), torch.ones(n, 1, device="cuda"))     # ones
    dy = torch.full((n, outputs), 0.1, device="cuda", dtype=BF16)
    dw, db = torch.full((outputs, inputs), NAN, device="cuda"), torch.full((outputs,), NAN, device="cuda")
    zeno.dense_gradient(dy, saved, dw, db)
    zeno.check_operator_status()
    want = n * float(dy[0, 0])
    R.assert_near(dw, torch.full((outputs, inputs), want), want * (64 * 2.0 ** -23 + 320 * R.U), "dw")
    R.assert_near(db, torch.full((outputs,), want), want * (1024 + 64) * R.U, "db")


@pytest.mark.parametrize("act", [F32, BF16])
def test_dense_gradient_over_many_rows_of_codes_that_start_anywhere(act):
    """On the CUDA cores: chains of 1,024 rows."""
    n, inputs, outputs = (1 << 20) + 7, 19, 8
    codes = torch.full((n, inputs + 2), 0x7f, device="cuda", dtype=torch.uint8)[:, 1:-1]
    codes.fill_(0x38)
    dy = torch.full((n, outputs), 0.1, device="cuda", dtype=act)
    dw, db = torch.full((outputs, inputs), NAN, device="cuda"), torch.full((outputs,), NAN, device="cuda")
    zeno.dense_gradient(dy, zeno.Saved(codes, torch.ones(n, 1, device="cuda")), dw, db)
    want = n * float(dy[0, 0])
    R.assert_near(dw, torch.full((outputs, inputs), want), want * (1024 + 16) * R.U, "dw")
    R.assert_near(db, torch.full((outputs,), want), want * (1024 + 16) * R.U, "db")


@pytest.mark.parametrize("cols", [(1 << 20) + 1, (1 << 20) + 8, (1 << 25) + 3])
@pytest.mark.parametrize("act", [F32, BF16])
@pytest.mark.parametrize("saved", [False, True])
def test_layer_norm_gradient_of_rows_too_long_for_weight_gradients(cols, act, saved):
    g = _gen(cols)
    x = torch.randn(1, 2, cols, generator=g, device="cuda").to(act)
    dy = torch.randn(1, 2, cols, generator=g, device="cuda").to(act)
    w = 1 + 0.2 * torch.randn(cols, generator=g, device="cuda")
    mean, rstd = torch.full((1, 2), 0.125, device="cuda"), torch.full((1, 2), 0.75, device="cuda")
    source, value = x, x
    if saved:
        source = zeno.pack_activations(x)
        value = R.unpack(source.codes, source.scales)
    dx = zeno.layer_norm_gradient(dy, source, w, mean, rstd)
    k = 96 * R.U
    d, h = dy.double() * w.double(), (value.double() - 0.125) * 0.75
    want = 0.75 * (d - d.mean(-1, keepdim=True) - h * (d * h).mean(-1, keepdim=True))
    slack = 0.75 * ((k + 8 * R.U) * (d.abs().mean(-1, keepdim=True) + h.abs() * (d * h).abs().mean(-1, keepdim=True)) + 8 * R.U * d.abs())
    R.assert_near(dx, want, slack, "dx")
    with pytest.raises(zeno.ZenoError) as e:
        zeno.layer_norm_gradient(dy, source, w, mean, rstd, torch.empty(1, cols, device="cuda"))
    assert e.value.status == zeno.ERR_UNSUPPORTED


def test_a_call_that_gives_up_ends_soon():
    """With a limit of zero the warp that copies the scales gives up while the codes' copies are under way: before it ends, a block waits for those copies
    alone.  (A wait for an arrival that nobody makes any more would take a quarter of a second for every stage.)"""
    g = _gen(1)
    saved = zeno.pack_activations(_rows(g, 4, 1000, 512, BF16))
    dy = _rows(g, 4, 1000, 768, BF16, 0.1)
    dw, want = torch.empty(4, 768, 512, device="cuda"), torch.empty(4, 768, 512, device="cuda")
    zeno.dense_gradient(dy, saved, want)
    zeno.check_operator_status()
    zeno.debug_set_operator_wait_limit(0)
    try:
        for _ in range(3):
            begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            begin.record()
            zeno.dense_gradient(dy, saved, dw)
            end.record()
            with pytest.raises(zeno.ZenoError) as e:
                zeno.check_operator_status()
            assert e.value.status == zeno.ERR_TIMEOUT
            assert begin.elapsed_time(end) < 100
    finally:
        zeno.debug_set_operator_wait_limit(1 << 22)
    zeno.dense_gradient(dy, saved, dw)
    zeno.check_operator_status()
    assert torch.equal(dw, want)


def test_every_stream_is_told_of_a_wait_that_ran_out():
    g = _gen(1)
    saved = zeno.pack_activations(_rows(g, 2, 200, 512, BF16))
    dy = _rows(g, 2, 200, 768, BF16, 0.1)
    dw = torch.empty(2, 768, 512, device="cuda")
    a, b = torch.cuda.Stream(), torch.cuda.Stream()

    def told(stream):
        try:
            zeno.check_operator_status(stream=stream)
        except zeno.ZenoError as e:
            assert e.status == zeno.ERR_TIMEOUT
            return True
        return False

    for s in (a, b, None):                                       # whatever earlier calls left
        told(s)
    torch.cuda.synchronize()
    zeno.debug_set_operator_wait_limit(0)
    try:
        zeno.dense_gradient(dy, saved, dw, stream=a)
    finally:
        zeno.debug_set_operator_wait_limit(1 << 22)
    a.synchronize()
    assert told(b)                                               # which must not take the report from the stream that the call ran on
    assert told(a) and told(None)
    assert not (told(a) or told(b) or told(None))
    zeno.dense_gradient(dy, saved, dw, stream=b)
    assert not (told(b) or told(a) or told(None))


@pytest.mark.parametrize("act", [F32, BF16])
def test_dense_gradient_of_the_smallest_entries(act):
    """One token of a row that is not zero, under codes of 256: no additions.  Three bfloat16 terms hold 24 bits from 2^-110 on; below, half of bfloat16's smallest step
    is missing at most."""
    m, n, cols = 16, 64, 512
    saved = zeno.pack_activations(torch.full((m, n, cols), 256.0, device="cuda", dtype=BF16))
    dw = torch.empty(m, cols, cols, device="cuda")
    e = torch.linspace(-148, -90, cols, device="cuda").round()
    for part in (2.0 ** -7, 2.0 ** -7 + 2.0 ** -15 + 2.0 ** -23, 1 - 2.0 ** -23):
        dy = torch.zeros(m, n, cols, device="cuda", dtype=act)
        dy[:, 17] = (torch.exp2(e.double()) * (1 + part)).to(act)
        zeno.dense_gradient(dy, saved, dw)
        value = dy[:, 17].double()
        off = torch.where((act == F32) & (value < 2.0 ** -110), 2.0 ** -134, 0.0)
        R.assert_near(dw, (256 * value).unsqueeze(-1).expand(m, cols, cols), 256 * off.unsqueeze(-1), "dw")


@pytest.mark.parametrize("cols", [1, 127, 129, 777, 1024])
@pytest.mark.parametrize("act", [F32, BF16])
def test_codes_in_rows_of_any_stride_through_the_c_abi(cols, act):
    """The binding makes rows of multiples of 16 bytes; the C ABI takes any, without a byte written between them."""
    g = _gen(cols)
    m, n = 3, 7
    x = _rows(g, m, n, cols, act, 30.0)
    x[0, 1, cols // 2] = NAN
    x[1, 2, cols - 1] = INF
    x[2, 3] = 0.0
    x[2, 4] *= 2.0 ** 100
    want, want_scales = R.pack(x)
    lib = zeno.load_library()
    blocks = -(-cols // 128)
    for first, row, group in ((1, cols, n * cols), (3, cols + 2, n * (cols + 2) + 5), (0, cols + 1, n * (cols + 1))):
        codes = torch.full((first + m * group + 16,), 0xa5, device="cuda", dtype=torch.uint8)
        scales = torch.full((m * n * (blocks + 1),), -1.0, device="cuda")
        st = lib.zeno_pack_activations(0, zeno.F32 if act == F32 else zeno.BF16, zeno.RowsDesc(x.data_ptr(), cols, n * cols), m, n, cols,
                                       zeno.RowsDesc(codes.data_ptr() + first, row, group), zeno.RowsDesc(scales.data_ptr(), blocks + 1, n * (blocks + 1)),
                                       torch.cuda.current_stream().cuda_stream)
        assert st == zeno.OK
        got = codes[first:].as_strided((m, n, cols), (group, row, 1))
        got_scales = scales.as_strided((m, n, blocks), (n * (blocks + 1), blocks + 1, 1))
        assert torch.equal(got_scales.double().cpu(), want_scales)
        value = got.clone().view(torch.float8_e4m3fn).double() * got_scales.double().repeat_interleave(128, -1)[..., :cols]
        want_value = want * want_scales.repeat_interleave(128, -1)[..., :cols]
        assert torch.equal(value.cpu().nan_to_num(nan=-7.0), want_value.nan_to_num(nan=-7.0))
        # the bits of the binding's codes
        packed = zeno.pack_activations(x)
        assert torch.equal(got, packed.codes.view(torch.uint8))
        got.fill_(0xa5)
        assert (codes == 0xa5).all() and (scales.as_strided((m, n), (n * (blocks + 1), blocks + 1), blocks) == -1.0).all()
