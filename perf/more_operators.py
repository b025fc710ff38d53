"""Cases of the operators at a language model's two ends: the embedding with its gradient, and the log probabilities of given tokens
from the last hidden states and the output weights, without logits, with their gradient.

A batch is [m, n]: n tokens of each of m workers (or of each of the models that the server evaluates).  Weight gradients go to the
workers' own rows of the candidate matrix V, whose rows are longer than the slice written."""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def listed():
    return [
        # the next token of one model enters it: latency
        {"name": "embed.one_token", "op": "embed", "m": 1, "n": 1, "vocab": 32000, "cols": 4096, "dtype": "bf16", "params": "bf16", "models": False, "masked": 0.0, "scale": 1.0},
        # 20 workers' batches enter a wide model
        {"name": "embed.workers", "op": "embed", "m": 20, "n": 2048, "vocab": 131072, "cols": 4096, "dtype": "bf16", "params": "bf16", "models": False, "masked": 0.1, "scale": 64.0},
        # a small binary32 model of an odd width: its gradient, a slice at an odd place of V
        {"name": "embed_grad.odd", "op": "embed_grad", "m": 7, "n": 333, "vocab": 1003, "cols": 777, "dtype": "f32", "params": "f32", "pad": 1, "masked": 0.1, "scale": 1.0},
        # eight workers' long batches into a wide table
        {"name": "embed_grad.workers", "op": "embed_grad", "m": 8, "n": 4096, "vocab": 32000, "cols": 4096, "dtype": "bf16", "params": "bf16", "pad": 0, "masked": 0.1, "scale": 64.0},
        # one worker with a very long batch of a large vocabulary
        {"name": "embed_grad.long", "op": "embed_grad", "m": 1, "n": 65536, "vocab": 131072, "cols": 2048, "dtype": "bf16", "params": "f32", "pad": 0, "masked": 0.0, "scale": 1.0},
        # how likely a served model finds one given token: latency
        {"name": "logprobs.one_token", "op": "logprobs", "m": 1, "n": 1, "vocab": 32000, "cols": 4096, "dtype": "bf16", "params": "bf16", "models": False, "masked": 0.0, "scale": 1.0},
        # a small binary32 model of an odd width and vocabulary
        {"name": "logprobs.odd", "op": "logprobs", "m": 3, "n": 57, "vocab": 5001, "cols": 777, "dtype": "f32", "params": "f32", "models": False, "masked": 0.1, "scale": 0.125},
        # the server's view: the loss of 21 perturbed models, a small batch each
        {"name": "logprobs.models", "op": "logprobs", "m": 21, "n": 128, "vocab": 32000, "cols": 1024, "dtype": "bf16", "params": "bf16", "models": True, "masked": 0.0, "scale": 1.0},
        # the loss of a batch over a large vocabulary
        {"name": "logprobs.batch", "op": "logprobs", "m": 2, "n": 2048, "vocab": 131072, "cols": 4096, "dtype": "bf16", "params": "bf16", "models": False, "masked": 0.1, "scale": 1.0},
        # gradients of a small binary32 model, odd sizes
        {"name": "logprobs_grad.odd", "op": "logprobs_grad", "m": 3, "n": 57, "vocab": 5001, "cols": 777, "dtype": "f32", "params": "f32", "masked": 0.1, "scale": 0.125},
        # many workers with a few tokens each: nearly all of it is writing their weight gradients
        {"name": "logprobs_grad.workers", "op": "logprobs_grad", "m": 16, "n": 61, "vocab": 32003, "cols": 1024, "dtype": "bf16", "params": "bf16", "masked": 0.1, "scale": 1.0},
        # gradients of a batch over a large vocabulary
        {"name": "logprobs_grad.batch", "op": "logprobs_grad", "m": 2, "n": 2048, "vocab": 131072, "cols": 4096, "dtype": "bf16", "params": "bf16", "masked": 0.1, "scale": 1.0},
    ]


def _log_uniform(rng, low, high):
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high))))))


def draw(rng):
    op = rng.choice(["embed", "embed_grad", "logprobs", "logprobs", "logprobs_grad", "logprobs_grad"])
    dtype, params = rng.choice(["f32", "bf16"]), rng.choice(["f32", "bf16"])
    vocab, cols = _log_uniform(rng, 50, 150000), _log_uniform(rng, 16, 8192)
    if rng.random() < 0.6:
        vocab, cols = -(-vocab // 64) * 64, -(-cols // 64) * 64
    while vocab * cols > 270_000_000:
        vocab //= 2
    m = _log_uniform(rng, 1, max(1, min(32, 500_000_000 // (vocab * cols))))
    case = {"op": op, "vocab": vocab, "cols": cols, "m": m, "dtype": dtype, "params": params}
    if op in ("embed", "embed_grad"):
        case["n"] = _log_uniform(rng, 1, max(2, min(65536, 100_000_000 // (m * cols))))
    else:
        case["n"] = _log_uniform(rng, 1, max(2, min(8192, 400_000_000_000 // (m * vocab * cols))))
    if op == "embed_grad":
        case["pad"] = rng.choice([0, 0, 8, 1])
    if op in ("embed", "logprobs"):
        case["models"] = rng.random() < 0.4
    case["masked"] = 0.0 if case["n"] == 1 else rng.choice([0.0, 0.1, 0.5])
    case["scale"] = rng.choice([1.0, 1.0, 0.125, 2.5])
    return case


# ---- what a program has in hand

def _tokens(g, case):
    """Token numbers: a few are very frequent, most are rare; padding has none."""
    m, n, vocab = case["m"], case["n"], case["vocab"]
    u = torch.rand(m, n, generator=g, device="cuda", dtype=torch.float64)
    ids = (torch.pow(float(vocab), u) - 1.0).long().clamp(0, vocab - 1)
    ids = (ids * 7919 + 13) % vocab if vocab % 7919 else ids              # frequent ones lie anywhere in the vocabulary
    ids[torch.rand(m, n, generator=g, device="cuda") < 0.03] = min(2, vocab - 1)
    return torch.where(torch.rand(m, n, generator=g, device="cuda") < case["masked"], -1, ids).int()


def _candidates(m, width, params):
    """The candidate matrix, rows 64 elements longer than what is written."""
    return torch.zeros(m, 32 + -(-width // 8) * 8 + 32, device="cuda", dtype=TYPES[params])


def _weights(g, case, size):
    """The table or output weights, [vocab, cols], or [m, vocab, cols]: slices of the models' parameter vectors."""
    vocab, cols = case["vocab"], case["cols"]
    if not case.get("models"):
        return (size * torch.randn(vocab, cols, generator=g, device="cuda")).to(TYPES[case["params"]])
    P = _candidates(case["m"], vocab * cols, case["params"])
    w = P[:, 32: 32 + vocab * cols].unflatten(1, (vocab, cols))
    shared = torch.randn(vocab, cols, generator=g, device="cuda")
    for i in range(case["m"]):
        w[i] = size * (shared + 0.1 * torch.randn(vocab, cols, generator=g, device="cuda"))
    return w


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, state = case["op"], dict(case)
    m, n, vocab, cols = case["m"], case["n"], case["vocab"], case["cols"]
    dtype = TYPES[case["dtype"]]
    tokens = state["tokens"] = _tokens(g, case)
    if op == "embed":
        state["w"] = _weights(g, case, 0.02)
        return state
    if op == "embed_grad":
        state["dy"] = (1e-2 * torch.randn(m, n, cols + case["pad"], generator=g, device="cuda")).to(dtype)[:, :, :cols]
        state["V"] = V = _candidates(m, vocab * cols + case["pad"], case["params"])
        at = 32 + case["pad"]
        state["dw"] = V[:, at: at + vocab * cols].unflatten(1, (vocab, cols))
        return state
    # hidden states of a model that has learnt something: logits of a few units, the given token's above most others
    w = state["w"] = _weights(g, case, 2.5 / case["scale"] / math.sqrt(cols))
    x = torch.randn(m, n, cols, generator=g, device="cuda")
    at = tokens.clamp(min=0).long()
    own_rows = torch.stack([w[i][at[i]] for i in range(m)]) if case.get("models") else w[at]
    x += own_rows.float() * (case["scale"] * 6.0 / 6.25)
    state["x"] = x.to(dtype)
    # padding's hidden states mean nothing
    state["x"][tokens < 0] = 1e4
    if op == "logprobs_grad":
        state["lse"] = _logprobs(state["x"], w, tokens, case["scale"])[1]
        state["g"] = torch.randn(m, n, generator=g, device="cuda") / n
        state["V"] = V = _candidates(m, vocab * cols, case["params"])
        state["dw"] = V[:, 32: 32 + vocab * cols].unflatten(1, (vocab, cols))
    return state


# ---- the operators in plain form

def _embed(tokens, w, scale, dtype):
    at = tokens.clamp(min=0).long()
    rows = w[torch.arange(len(tokens), device=at.device).unsqueeze(1), at] if w.dim() == 3 else w[at]
    return torch.where((tokens >= 0).unsqueeze(-1), scale * rows.float(), 0.0).to(dtype)


def _embed_grad(tokens, dy, scale, dw):
    for i in range(len(tokens)):
        given = (tokens[i] >= 0).unsqueeze(-1)
        total = torch.zeros(dw.shape[1:], device=dy.device)
        total.index_add_(0, tokens[i].clamp(min=0).long(), torch.where(given, dy[i].float(), 0.0))
        dw[i] = scale * total
    return dw


def _logits(x, w, scale):
    return scale * torch.matmul(x.float(), w.float().transpose(-1, -2))


def _logprobs(x, w, tokens, scale):
    """Log probability of each given token and the log of its row's sum of exponentials, [m, n]; zero without a token."""
    given = tokens >= 0
    lps, lses = [], []
    for i in range(len(x)):
        z = _logits(x[i], w[i] if w.dim() == 3 else w, scale)
        top = z.amax(-1)
        zt = z.gather(-1, tokens[i].clamp(min=0).long().unsqueeze(-1)).squeeze(-1)
        z -= top.unsqueeze(-1)
        lse = top + torch.log(z.exp_().sum(-1))
        lps.append(torch.where(given[i], zt - lse, 0.0))
        lses.append(torch.where(given[i], lse, 0.0))
    return torch.stack(lps), torch.stack(lses)


def _logprobs_grad(x, w, tokens, lse, g, scale, dw):
    dx = torch.empty_like(x)
    wf = w.float()
    for i in range(len(x)):
        given = tokens[i] >= 0
        xi = torch.where(given.unsqueeze(-1), x[i].float(), 0.0)
        gi = torch.where(given, g[i], 0.0) * scale
        d = _logits(xi, wf, scale)
        d -= lse[i].unsqueeze(-1)
        d.exp_()
        d *= -gi.unsqueeze(-1)
        d[torch.arange(len(d), device=d.device), tokens[i].clamp(min=0).long()] += gi
        dx[i] = torch.matmul(d, wf)
        dw[i] = torch.matmul(d.T, xi)
    return dx, dw


def run(state):
    op = state["op"]
    if own:
        from paper_1805_10032_b200 import zeno

        if op == "embed":
            return zeno.embed(state["tokens"], state["w"], scale=state["scale"], dtype=TYPES[state["dtype"]])
        if op == "embed_grad":
            return zeno.embed_gradient(state["tokens"], state["dy"], state["dw"], scale=state["scale"])
        if op == "logprobs":
            return tuple(zeno.linear_logprobs(state["x"], state["w"], state["tokens"], scale=state["scale"]))
        dx = zeno.linear_logprobs_gradient(state["x"], state["w"], state["tokens"], state["lse"], state["g"], dweight=state["dw"], scale=state["scale"])
        return dx, state["dw"]
    if op == "embed":
        return _embed(state["tokens"], state["w"], state["scale"], TYPES[state["dtype"]])
    if op == "embed_grad":
        return _embed_grad(state["tokens"], state["dy"], state["scale"], state["dw"])
    if op == "logprobs":
        return _logprobs(state["x"], state["w"], state["tokens"], state["scale"])
    return _logprobs_grad(state["x"], state["w"], state["tokens"], state["lse"], state["g"], state["scale"], state["dw"])


def _distinct(vocab, tokens):
    """How many token numbers occur among so many drawn as _tokens does."""
    return sum(1.0 - math.exp(-tokens * math.log1p(1.0 / (i + 1)) / math.log(max(vocab, 2))) for i in range(vocab))


def work(case):
    op, m, vocab, cols = case["op"], case["m"], case["vocab"], case["cols"]
    s, p = SIZE[case["dtype"]], SIZE[case["params"]]
    rows = m * case["n"]
    given = rows * (1.0 - case["masked"])
    if op == "embed":
        # of the table, the rows that occur
        table = m * _distinct(vocab, given / m) if case["models"] else _distinct(vocab, given)
        return {"bytes": table * cols * p + rows * (cols * s + 4), "flops": given * cols}
    if op == "embed_grad":
        return {"bytes": given * cols * s + 4 * rows + m * vocab * cols * p, "flops": given * cols}
    weights = (m if case.get("models") else 1) * vocab * cols * p
    if op == "logprobs":
        return {"bytes": given * cols * s + weights + rows * 12, "flops": 2 * given * vocab * cols}
    return {"bytes": 2 * given * cols * s + weights + m * vocab * cols * p + rows * 12, "flops": 6 * given * vocab * cols}


# ---- the same values from the definitions, in 64 bits

def _as(t, params):
    """Large outputs of bfloat16 are compared in binary32."""
    return t.float() if params == "bf16" else t


def exact(case, seed):
    state = prepare(case, seed)
    op, tokens, scale = case["op"], state["tokens"].long(), float(case["scale"])
    m, n, vocab, cols = case["m"], case["n"], case["vocab"], case["cols"]
    if op == "embed":
        out = torch.zeros(m, n, cols, device="cuda", dtype=torch.float64)
        for i in range(m):
            table = state["w"][i] if case["models"] else state["w"]
            has = (tokens[i] >= 0).nonzero().squeeze(-1)
            out[i, has] = table.index_select(0, tokens[i, has]).double().mul(scale)
        return out
    if op == "embed_grad":
        outs = []
        for i in range(m):
            has = (tokens[i] >= 0).nonzero().squeeze(-1)
            total = torch.zeros(vocab, cols, device="cuda", dtype=torch.float64)
            total.index_add_(0, tokens[i, has], state["dy"][i, has].double())
            outs.append(_as(total.mul_(scale), case["params"]))
        return torch.stack(outs)
    lp, lse = torch.zeros(m, n, device="cuda", dtype=torch.float64), torch.zeros(m, n, device="cuda", dtype=torch.float64)
    dx, dws = torch.zeros(m, n, cols, device="cuda", dtype=torch.float64), []
    for i in range(m):
        w = (state["w"][i] if case.get("models") else state["w"]).double()
        total = torch.zeros(vocab, cols, device="cuda", dtype=torch.float64) if op == "logprobs_grad" else None
        has = (tokens[i] >= 0).nonzero().squeeze(-1)
        for part in has.split(512):
            x, t = state["x"][i, part].double(), tokens[i, part]
            z = torch.einsum("tc,vc->tv", x, w) * scale
            if op == "logprobs":
                lse[i, part] = torch.logsumexp(z, -1)
                lp[i, part] = torch.log_softmax(z, -1).gather(-1, t.unsqueeze(-1)).squeeze(-1)
                continue
            d = torch.nn.functional.one_hot(t, vocab).double() - torch.exp(z - state["lse"][i, part].double().unsqueeze(-1))
            d *= (state["g"][i, part].double() * scale).unsqueeze(-1)
            dx[i, part] = torch.einsum("tv,vc->tc", d, w)
            total.addmm_(d.T, x)
        if total is not None:
            dws.append(_as(total, case["params"]))
    return (lp, lse) if op == "logprobs" else (dx, torch.stack(dws))
