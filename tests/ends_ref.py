"""A language model's two ends from their definitions, in 64 bits, and how far binary32 arithmetic may be from them.

U is half a step of binary32 relative to the value.  The tensor cores add 16 products at a time with truncation, off by at most 2 U of the sum of magnitudes so
far; a stretch has at most 32 such steps of the leading terms (the smaller terms, 2^-8 of them, at most 512 and so 4 U more), and stretches are added to
nearest.  Products of terms that are left out of binary32 operands are 4 U at most."""
import torch

from operators_ref import HALF, U


def embed(tokens, table, scale):
    """tokens [m, n]; table [vocab, cols] or [m, vocab, cols]."""
    vocab = table.shape[-2]
    given = (tokens >= 0) & (tokens < vocab)
    at = torch.where(given, tokens, 0).long()
    rows = table.double()[at] if table.dim() == 2 else torch.stack([table[i].double()[at[i]] for i in range(len(at))])
    want = torch.where(given.unsqueeze(-1), scale * rows, 0.0)
    return want, U * want.abs()


def embed_gradient(tokens, dy, vocab, scale, before=None):
    """[m, vocab, cols] and its slack: a row's tokens in chains of at most 64, with compensation beyond."""
    m, n = tokens.shape
    total = torch.zeros(m, vocab, dy.shape[-1], dtype=torch.float64, device=dy.device)
    size, count = torch.zeros_like(total), torch.zeros(m, vocab, dtype=torch.float64, device=dy.device)
    for i in range(m):
        has = ((tokens[i] >= 0) & (tokens[i] < vocab)).nonzero().squeeze(-1)
        at, d = tokens[i, has].long(), dy[i, has].double()
        total[i].index_add_(0, at, d)
        size[i].index_add_(0, at, d.abs())
        count[i].index_add_(0, at, torch.ones_like(at, dtype=torch.float64))
    slack = abs(scale) * (count.clamp(max=64).unsqueeze(-1) + 20) * U * size
    want = scale * total + (0 if before is None else before.double())
    return want, slack + U * want.abs()


def _products(cols):
    return (2 * 34 + cols / 512 + 24) * U


def logits(x, w, scale):
    """(z, its slack) of x [n, cols] and w [vocab, cols]."""
    x, w = x.double(), w.double()
    z = scale * (x @ w.T)
    return z, _products(x.shape[-1]) * abs(scale) * (x.abs() @ w.abs().T) + 2 * U * z.abs()


def logprobs(x, w, targets, scale):
    """x [m, n, cols], w [vocab, cols] or [m, vocab, cols]: (logprob, lse, their slacks), zero without a target."""
    out = []
    for i in range(len(x)):
        wi = w[i] if w.dim() == 3 else w
        z, off = logits(x[i], wi, scale)
        t = targets[i].long()
        given = (t >= 0) & (t < wi.shape[0])
        at = torch.where(given, t, 0).unsqueeze(-1)
        lse = torch.logsumexp(z, -1)
        p = torch.exp(z - lse.unsqueeze(-1))
        # a chain of 32 exponentials, each off by its argument's rounding and its own, then trees
        lse_off = (p * off).sum(-1) * 1.01 + (32 + 16 + 8) * U + 4 * U * (p * (z - lse.unsqueeze(-1)).abs().clamp(max=1e4)).sum(-1)
        zt, zt_off = z.gather(-1, at).squeeze(-1), off.gather(-1, at).squeeze(-1)
        of = lambda v: torch.where(given, v, 0.0)  # noqa: E731
        out.append((of(zt - lse), of(lse), of(zt_off + lse_off + 2 * U * zt.abs()), of(lse_off)))
    return tuple(torch.stack(v) for v in zip(*out))


def logprobs_gradient(x, w, targets, lse, g, scale, dtype):
    """(dx [m, n, cols], dw [m, vocab, cols], their slacks) with the lse that is given; dtype is the wider of the operands' types."""
    dxs, dws, dx_offs, dw_offs = [], [], [], []
    for i in range(len(x)):
        wi = (w[i] if w.dim() == 3 else w).double()
        t = targets[i].long()
        given = (t >= 0) & (t < wi.shape[0])
        xi = torch.where(given.unsqueeze(-1), x[i].double(), 0.0)
        z, off = logits(xi, wi, scale)
        L = torch.where(given, lse[i].double(), 0.0).unsqueeze(-1)
        hot = torch.zeros_like(z).scatter_(-1, torch.where(given, t, 0).unsqueeze(-1), 1.0)
        gs = torch.where(given, g[i].double() * scale, 0.0).unsqueeze(-1)
        p = torch.where(given.unsqueeze(-1), torch.exp(z - L), 0.0)
        d = gs * (hot - p)
        p_off = p * (torch.expm1(off + U * L.abs() + 4 * U * (z - L).abs()) + 8 * U)
        d_off = gs.abs() * p_off + (HALF[torch.bfloat16] if dtype == torch.bfloat16 else 4 * U) * (d.abs() + gs.abs() * p_off) + 2 * U * d.abs()
        dxs.append(d @ wi)
        dws.append(d.T @ xi)
        size = d.abs() + d_off
        dx_offs.append(d_off @ wi.abs() + (_products(wi.shape[0]) + 80 * U) * (size @ wi.abs()))
        dw_offs.append(d_off.T @ xi.abs() + _products(len(xi)) * (size.T @ xi.abs()))
    return tuple(torch.stack(v) for v in (dxs, dws, dx_offs, dw_offs))
