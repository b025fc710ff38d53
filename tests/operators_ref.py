"""The language model operators from their definitions, in 64 bits, and how far binary32 arithmetic may be from them.

U is half a step of binary32 relative to the value.  A sum of terms added along chains of at most L of them, whose results are
added in a tree, is off by at most (L + the tree's depth) U times the sum of the terms' magnitudes; the kernels' chains are a
row's entries divided by at least 32 lanes, or a group's rows."""
import torch

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float8_e4m3fn: 2.0 ** -4}


def assert_near(got, want, slack, what=""):
    """|got - want| <= half a step of got's type + slack, entry by entry; equal where want is not finite."""
    want = want.double().cpu()
    slack = torch.as_tensor(slack, dtype=torch.float64).cpu().expand_as(want)
    g = got.double().cpu()
    assert g.shape == want.shape, (what, g.shape, want.shape)
    odd = ~torch.isfinite(want)
    assert torch.equal(g[odd].nan_to_num(nan=12345.0), want[odd].nan_to_num(nan=12345.0)), what
    assert torch.isfinite(g[~odd]).all(), what
    # where the slack carries the value to the next power of two, its half step is the next one's
    off = (g - want).abs()[~odd] - (HALF[got.dtype] * (want.abs() + slack) + slack)[~odd]
    assert off.numel() == 0 or off.max() <= 0, (what, float(off.max()), float((g - want).abs()[~odd].max()))


def norm(x, w, b, eps):
    """x [m, n, cols]; w, b [cols] or [m, cols].  (y, mean, rstd, slacks of the three)."""
    x = x.double()
    w, b = (t.double() if t.dim() == 1 else t.double().unsqueeze(1) for t in (w, b))
    cols = x.shape[-1]
    k = (cols / 32 + 32) * U
    mean = x.sum(-1, keepdim=True) / cols
    d = x - mean
    var = (d * d).sum(-1, keepdim=True) / cols
    rstd = (var + eps) ** -0.5
    size = x.abs().mean(-1, keepdim=True)
    # the mean is off by k avg|x|, which moves every centred entry; their squares' sum adds k/2 relative to rstd, and the shift
    # of the mean adds its square only
    mean_off = k * size
    rstd_off = rstd * (k + (mean_off * rstd) ** 2)
    h = d * rstd
    y_off = ((mean_off + 2 * U * (x.abs() + mean.abs())) * rstd + h.abs() * (k + (mean_off * rstd) ** 2 + 4 * U)) * w.abs() + 4 * U * (b.abs() + (h * w).abs())
    return h * w + b, mean.squeeze(-1), rstd.squeeze(-1), y_off, mean_off.squeeze(-1), rstd_off.squeeze(-1)


def norm_gradient(dy, x, w, mean, rstd):
    """(dx, dw, db, slacks of the three) with the mean and rstd that are given."""
    dy, x, mean, rstd = dy.double(), x.double(), mean.double().unsqueeze(-1), rstd.double().unsqueeze(-1)
    w = w.double() if w.dim() == 1 else w.double().unsqueeze(1)
    n, cols = x.shape[-2:]
    k = (cols / 32 + 32) * U
    h = (x - mean) * rstd
    h_off = 2 * U * ((x.abs() + mean.abs()) * rstd + h.abs())
    g = dy * w
    c1, c2 = g.mean(-1, keepdim=True), (g * h).mean(-1, keepdim=True)
    c1_off = k * g.abs().mean(-1, keepdim=True)
    c2_off = k * (g * h).abs().mean(-1, keepdim=True) + (g.abs() * h_off).mean(-1, keepdim=True)
    dx = rstd * (g - c1 - h * c2)
    dx_off = rstd * (c1_off + h.abs() * c2_off + h_off * c2.abs() + 6 * U * (g.abs() + c1.abs() + (h * c2).abs()))
    dw, db = (dy * h).sum(-2), dy.sum(-2)
    dw_off = (n + 32) * U * (dy * h).abs().sum(-2) + (dy.abs() * h_off).sum(-2)
    return dx, dw, db, dx_off, dw_off, (n + 32) * U * dy.abs().sum(-2)


def pack(x):
    """(code values, scales): blocks of 128 columns of finite entries by their largest, non-finite ones NaN."""
    x = x.double().cpu()
    cols = x.shape[-1]
    values, scales = torch.zeros_like(x), []
    for at in range(0, cols, 128):
        v = x[..., at:at + 128]
        fine = torch.isfinite(v)
        amax = torch.where(fine, v.abs(), 0.0).amax(-1, keepdim=True)
        k = torch.full_like(amax, -117)
        for e in range(-117, 119):                     # the smallest k whose range holds the largest entry
            k = torch.where(amax > 448 * 2.0 ** e, e + 1.0, k)
        s = torch.where(amax > 0, 2.0 ** k, 1.0)
        q = torch.where(fine, v / s, 0.0).clamp(-448, 448)
        step = 2.0 ** (torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
        values[..., at:at + 128] = torch.where(fine, torch.round(q / step) * step, float("nan"))
        scales.append(s)
    return values, torch.cat(scales, -1)


def unpack(codes, scales):
    return codes.double() * scales.double().repeat_interleave(128, -1)[..., :codes.shape[-1]]


def dense_gradient(dy, x):
    """(dw, db, slacks): x in 64 bits already."""
    dy, x = dy.double(), x.double()
    n = x.shape[-2]
    dw = dy.transpose(-1, -2) @ x
    return dw, dy.sum(-2), (n + 32) * U * (dy.abs().transpose(-1, -2) @ x.abs()), (n + 32) * U * dy.abs().sum(-2)


def token_logprobs(z, targets, top):
    """(logprob, entropy, lse, top_idx, top_logprobs, slacks of logprob, entropy, lse and top_logprobs)."""
    z = z.double().cpu()
    t = targets.long().cpu()
    vocab = z.shape[-1]
    m = z.amax(-1, keepdim=True)
    m = torch.where(m == -float("inf"), 0.0, m)
    d = z - m
    e = torch.exp(d)
    s = e.sum(-1)
    empty = s == 0
    log_s = torch.log(s)
    lse = m.squeeze(-1) + log_s
    p = e / s.unsqueeze(-1)
    dd = torch.where(e > 0, d, 0.0)
    entropy = torch.where(empty, 0.0, log_s - (p * dd).sum(-1))
    given = (t >= 0) & (t < vocab)
    zt = z.gather(-1, torch.where(given, t, 0).unsqueeze(-1)).squeeze(-1)
    of = lambda v: torch.where(empty.reshape(empty.shape + (1,) * (v.dim() - empty.dim())), -float("inf"),  # noqa: E731
                               (v - m.reshape(m.shape[:-1] + (1,) * (v.dim() - empty.dim()))) - log_s.reshape(empty.shape + (1,) * (v.dim() - empty.dim())))
    lp = torch.where(given, of(zt), 0.0)
    order = torch.where(torch.isnan(z), -float("inf"), z)
    idx = torch.sort(order, dim=-1, descending=True, stable=True).indices[..., :top]
    top_lp = of(z.gather(-1, idx))
    # an exponent t = d log2 e is off by 2 U |t| + U, so exp by (3 |d| + 4) U; S by that, weighted, and the chains
    k = (vocab / 32 + 32) * U
    depth = (p * dd.abs()).sum(-1).nan_to_num(0.0)
    s_off = k + U * (8 + 4 * depth)
    lse_off = s_off + 4 * U * (m.squeeze(-1).abs() + lse.abs())
    fin = lambda v: torch.where(torch.isfinite(v), v, 0.0)  # noqa: E731
    lse_off = fin(lse_off)
    h_off = fin((s_off + k) * (17 + depth + log_s.abs()) + U * (p * 8 * dd * dd).sum(-1))
    # a log probability comes from z - m and log S, whatever the size of m; m itself may stand 8 powers of two beside the largest entry
    lp_off = fin(s_off + 4 * U * (log_s.abs() + 16))
    return (lp, entropy, lse, idx.int(), top_lp, lp_off + 8 * U * fin(lp).abs(), h_off, lse_off, lp_off.unsqueeze(-1) + 8 * U * fin(top_lp).abs())


def token_gradient(z, targets, lse, entropy, g, gh):
    """(gradient, slack) with the lse and entropy that are given; far from zero, where lse in binary32 says little, from the logits."""
    z, t, lse, g = z.double().cpu(), targets.long().cpu(), lse.double().cpu().unsqueeze(-1), g.double().cpu()
    vocab = z.shape[-1]
    far = (lse.abs() >= 2.0 ** 20) & (lse != -float("inf"))
    if far.any():
        top = torch.where(far, z.amax(-1, keepdim=True), 0.0)
        z = z - top
        lse = torch.where(far, torch.log(torch.exp(z).sum(-1, keepdim=True)), lse)
    given = (t >= 0) & (t < vocab)
    g = torch.where(given, g, 0.0).unsqueeze(-1)
    logp = z - lse
    p = torch.exp(logp)
    hot = torch.zeros_like(z).scatter_(-1, torch.where(given, t, 0).unsqueeze(-1), 1.0) * given.unsqueeze(-1)
    # where the row is summed again, p is off by its sum too, and log p by as much: chains of vocab / 32 terms, each exponential off by
    # U (3 |d| + 4), as in token_logprobs
    depth = torch.where(p > 0, p * logp, 0.0).sum(-1, keepdim=True).abs()
    s_off = far * U * (vocab / 32 + 32 + 8 + 4 * depth)
    factor, factor_off = g, 4 * U * g.abs() + torch.zeros_like(z)
    size = torch.where(torch.isfinite(z), z.abs(), 0.0) + lse.abs()
    if gh is not None:
        gh, entropy = gh.double().cpu().unsqueeze(-1), entropy.double().cpu().unsqueeze(-1)
        safe = torch.where(p > 0, logp, 0.0)
        factor = g + gh * (safe + entropy)
        factor_off = 4 * U * (g.abs() + gh.abs() * (size + entropy.abs())) + gh.abs() * s_off
    # log p is off by U (|z| + |lse|) and its exponential by that and U (2 |log p| + 4)
    rel = U * (4 + 4 * size) + s_off
    none = lse == -float("inf")
    if gh is None:
        none = none | ~given.unsqueeze(-1)
    grad = torch.where(none, 0.0, g * hot - p * factor)
    fin = lambda v: torch.where(torch.isfinite(v), v, 0.0)  # noqa: E731
    # entries under 2^-126 may be off by a subnormal step of what multiplies them
    return grad, fin(p * (factor.abs() * rel + factor_off) + 2 * U * (g.abs() * hot) + 2.0 ** -140 * (1 + factor.abs()))
