"""Cases of the operators of language models that stand beside the worker gradients: layer norm with its backward pass,
activations kept in 8 bits and what the backward pass takes from them, log probabilities of given tokens with their gradient.

A batch of activations is [m, n, columns]: n tokens of each of m workers (or of each of the models that the server evaluates).
Weight gradients go to the workers' own rows of the candidate matrix V, whose rows are longer than the slice written."""
import math

import torch

own = False

BLOCK = 128          # columns that share a scale
E4M3_MAX = 448.0
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def listed():
    return [
        # one token through a norm layer of one model: latency
        {"name": "norm.one_token", "op": "norm", "m": 1, "n": 1, "cols": 4096, "pad": 0, "dtype": "bf16", "params": "bf16", "models": False},
        # the server's view of a norm layer: 21 perturbed models with weights of their own, the same number of tokens each
        {"name": "norm.models", "op": "norm", "m": 21, "n": 2048, "cols": 4096, "pad": 0, "dtype": "bf16", "params": "bf16", "models": True},
        # 20 workers' batches of a wide model in bfloat16
        {"name": "norm_grad.workers", "op": "norm_grad", "m": 20, "n": 2048, "cols": 4096, "pad": 0, "dtype": "bf16", "params": "bf16", "saved": "x"},
        # a small model in binary32, odd sizes, unaligned rows, its input kept in 8 bits
        {"name": "norm_grad.odd_saved", "op": "norm_grad", "m": 7, "n": 333, "cols": 777, "pad": 1, "dtype": "f32", "params": "f32", "saved": "8bit"},
        # activations kept for the backward pass: a worker's few tokens of an odd width
        {"name": "pack.odd", "op": "pack", "m": 3, "n": 57, "cols": 1029, "pad": 2, "dtype": "f32"},
        # and 20 workers' activations of a wide layer
        {"name": "pack.workers", "op": "pack", "m": 20, "n": 2048, "cols": 4096, "pad": 0, "dtype": "bf16"},
        # weight gradients of a small odd layer, a few tokens a worker
        {"name": "dense_grad.odd", "op": "dense_grad", "m": 12, "n": 37, "inputs": 301, "outputs": 131, "dtype": "f32", "params": "f32"},
        # weight gradients of a wide layer, eight workers
        {"name": "dense_grad.wide", "op": "dense_grad", "m": 8, "n": 2048, "inputs": 4096, "outputs": 4096, "dtype": "bf16", "params": "bf16"},
        # one token's alternatives out of a vocabulary: latency
        {"name": "logprobs.one_row", "op": "logprobs", "rows": 1, "vocab": 32000, "pad": 0, "dtype": "f32", "top": 8},
        # the tokens of a batch, large vocabulary
        {"name": "logprobs.batch", "op": "logprobs", "rows": 4096, "vocab": 131072, "pad": 0, "dtype": "bf16", "top": 4},
        # the loss's gradient for a few rows of an odd vocabulary in binary32
        {"name": "loss_grad.odd", "op": "loss_grad", "rows": 61, "vocab": 50001, "pad": 0, "dtype": "f32", "entropy": True},
        # and for a batch in bfloat16
        {"name": "loss_grad.batch", "op": "loss_grad", "rows": 4096, "vocab": 65536, "pad": 0, "dtype": "bf16", "entropy": False},
    ]


def _log_uniform(rng, low, high):
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high))))))


def draw(rng):
    op = rng.choice(["norm", "norm_grad", "pack", "dense_grad", "logprobs", "loss_grad"])
    dtype, params = rng.choice(["f32", "bf16"]), rng.choice(["f32", "bf16"])
    case = {"op": op}
    if op in ("logprobs", "loss_grad"):
        vocab = _log_uniform(rng, 100, 200000)
        vocab = vocab if rng.random() < 0.4 else -(-vocab // 64) * 64
        case |= {"rows": _log_uniform(rng, 1, min(8192, max(2, 100_000_000 // vocab))), "vocab": vocab, "pad": rng.choice([0, 0, 8, 3]), "dtype": dtype}
        if op == "logprobs":
            case["top"] = rng.choice([0, 1, 5, 20, 32])
        else:
            case["entropy"] = rng.random() < 0.5
        return case
    if op == "dense_grad":
        m, inputs, outputs = _log_uniform(rng, 1, 32), _log_uniform(rng, 16, 4096), _log_uniform(rng, 16, 4096)
        if rng.random() < 0.6:
            inputs, outputs = -(-inputs // 16) * 16, -(-outputs // 16) * 16
        n = _log_uniform(rng, 1, min(8192, max(2, 40_000_000_000 // (m * inputs * outputs))))
        return case | {"m": m, "n": n, "inputs": inputs, "outputs": outputs, "dtype": dtype, "params": params}
    cols = _log_uniform(rng, 24, 16384)
    cols = cols if rng.random() < 0.4 else -(-cols // 64) * 64
    m = _log_uniform(rng, 1, 40)
    n = _log_uniform(rng, 1, min(4096, max(2, 40_000_000 // (m * cols))))
    case |= {"m": m, "n": n, "cols": cols, "pad": rng.choice([0, 0, 8, 1]), "dtype": dtype}
    if op == "norm":
        case |= {"params": params, "models": rng.random() < 0.5}
    if op == "norm_grad":
        case |= {"params": params, "saved": rng.choice(["x", "8bit"])}
    return case


# ---- what a program has in hand

def _activations(g, m, n, cols, pad, dtype):
    """[m, n, cols] with rows pad elements longer: a residual stream, a few of whose columns are far larger than the rest."""
    t = torch.randn(m, n, cols + pad, generator=g, device="cuda")
    t *= 0.5 + 4.0 * (torch.rand(cols + pad, generator=g, device="cuda") < 0.01)
    return (t + 0.1).to(TYPES[dtype])[:, :, :cols]


def _gradients(g, m, n, cols, pad, dtype):
    return (1e-2 * torch.randn(m, n, cols + pad, generator=g, device="cuda")).to(TYPES[dtype])[:, :, :cols]


def _candidates(m, width, params):
    """The candidate matrix, rows 64 elements longer than what is written, and where the slice begins."""
    return torch.zeros(m, 32 + -(-width // 8) * 8 + 32, device="cuda", dtype=TYPES[params])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, state = case["op"], dict(case)
    if op in ("logprobs", "loss_grad"):
        rows, vocab = case["rows"], case["vocab"]
        z = torch.randn(rows, vocab + case["pad"], generator=g, device="cuda") * 2.5
        z = z[:, :vocab]
        targets = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
        z[torch.arange(rows, device="cuda"), targets] += 6.0
        # words that this row may not take
        z[:: 3, vocab // 2: vocab // 2 + vocab // 50] = -math.inf
        # prompts and padding carry no target
        targets = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.1, -1, targets)
        state["logits"], state["targets"] = z.to(TYPES[case["dtype"]]) if case["dtype"] == "bf16" else z, targets.int()
        if case["pad"] and case["dtype"] == "bf16":
            wide = torch.empty(rows, vocab + case["pad"], device="cuda", dtype=torch.bfloat16)
            wide[:, :vocab] = state["logits"]
            state["logits"] = wide[:, :vocab]
        if op == "loss_grad":
            state["lse"], state["h"] = _lse_entropy(state["logits"])
            state["g"] = torch.randn(rows, generator=g, device="cuda") / rows
            state["gh"] = torch.randn(rows, generator=g, device="cuda") / rows if case["entropy"] else None
        return state
    m, n = case["m"], case["n"]
    if op == "dense_grad":
        state["dy"] = _gradients(g, m, n, case["outputs"], 0, case["dtype"])
        state["saved"] = _pack(_activations(g, m, n, case["inputs"], 0, case["dtype"]))
        size = case["inputs"] * case["outputs"]
        state["V"] = V = _candidates(m, size + case["outputs"], case["params"])
        state["dw"] = V[:, 32: 32 + size].unflatten(1, (case["outputs"], case["inputs"]))
        state["db"] = V[:, 32 + size: 32 + size + case["outputs"]]
        return state
    cols = case["cols"]
    x = state["x"] = _activations(g, m, n, cols, case["pad"], case["dtype"])
    if op == "pack":
        return state
    shape = (m, cols) if case.get("models") else (cols,)
    state["w"] = (1.0 + 0.1 * torch.randn(shape, generator=g, device="cuda")).to(TYPES[case["params"]])
    state["b"] = (0.1 * torch.randn(shape, generator=g, device="cuda")).to(TYPES[case["params"]])
    if op == "norm_grad":
        _, state["mean"], state["rstd"] = _norm(x, state["w"], state["b"], 1e-5)
        state["dy"] = _gradients(g, m, n, cols, case["pad"], case["dtype"])
        if case["saved"] == "8bit":
            state["x"] = _pack(x)
        state["V"] = V = _candidates(m, 2 * cols, case["params"])
        state["dw"], state["db"] = V[:, 32: 32 + cols], V[:, 32 + cols: 32 + 2 * cols]
    return state


# ---- the operators in plain form

def _per_model(w):
    return w.float().unsqueeze(1) if w.dim() == 2 else w.float()


def _norm(x, w, b, eps):
    z = x.float()
    mean = z.mean(-1, keepdim=True)
    z = z - mean
    rstd = torch.rsqrt((z * z).mean(-1, keepdim=True) + eps)
    return (z * rstd * _per_model(w) + _per_model(b)).to(x.dtype), mean.squeeze(-1), rstd.squeeze(-1)


def _blocks(t):
    """[.., cols] -> [.., blocks, BLOCK], zeros behind the last column."""
    cols = t.shape[-1]
    count = -(-cols // BLOCK)
    return torch.cat([t, t.new_zeros(*t.shape[:-1], count * BLOCK - cols)], -1).unflatten(-1, (count, BLOCK))


def _pack(x):
    """Codes (e4m3, rows of a multiple of 16 bytes) and scales (powers of two) of x."""
    cols = x.shape[-1]
    t = _blocks(x.float())
    mantissa, exponent = torch.frexp(t.abs().amax(-1))                 # amax = mantissa 2^exponent, mantissa in [1/2, 1)
    k = torch.where(mantissa > 0.875, exponent - 8, exponent - 9).clamp(-117, 119)
    scales = torch.where(mantissa > 0, torch.ldexp(torch.ones_like(mantissa), k), 1.0)
    codes = (t / scales.unsqueeze(-1)).clamp(-E4M3_MAX, E4M3_MAX).flatten(-2)
    wide = torch.zeros(*x.shape[:-1], -(-cols // 16) * 16, device=x.device, dtype=torch.float8_e4m3fn)
    wide[..., :cols] = codes[..., :cols].to(torch.float8_e4m3fn)
    return wide[..., :cols], scales


def _unpack(codes, scales, dtype=torch.float32):
    return codes.to(dtype) * scales.to(dtype).repeat_interleave(BLOCK, -1)[..., : codes.shape[-1]]


def _norm_grad(dy, x, w, mean, rstd, params):
    x = _unpack(*x) if isinstance(x, tuple) else x.float()
    xh = (x - mean.unsqueeze(-1)) * rstd.unsqueeze(-1)
    t = dy.float()
    g = t * _per_model(w)
    dx = rstd.unsqueeze(-1) * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
    return dx.to(dy.dtype), (t * xh).sum(1).to(params), t.sum(1).to(params)


def _lse_entropy(logits):
    z = logits.float()
    top = z.amax(-1, keepdim=True)
    d = z - top
    e = torch.exp(d)
    s = e.sum(-1)
    entropy = torch.log(s) - torch.where(e > 0, e * d, 0.0).sum(-1) / s
    return top.squeeze(-1) + torch.log(s), entropy


def _order_keys(logits):
    """Integers in the order "larger value first, then lower index"."""
    i = (logits.float() + 0.0).view(torch.int32).long()
    i = torch.where(i < 0, i ^ 0x7FFFFFFF, i)
    return i * 2 ** 32 + torch.arange(logits.shape[-1] - 1, -1, -1, device=logits.device)


def _logprobs(logits, targets, top):
    lse, entropy = _lse_entropy(logits)
    given = targets >= 0
    at = torch.where(given, targets, 0).long().unsqueeze(-1)
    lp = torch.where(given, logits.gather(-1, at).squeeze(-1).float() - lse, 0.0)
    if not top:
        return lp, entropy, lse, None, None
    idx = _order_keys(logits).topk(top).indices
    return lp, entropy, lse, idx.int(), logits.gather(-1, idx).float() - lse.unsqueeze(-1)


def _loss_grad(logits, targets, lse, entropy, g, gh):
    logp = logits.float() - lse.unsqueeze(-1)
    p = torch.exp(logp)
    g = torch.where(targets >= 0, g, 0.0)
    grad = -g.unsqueeze(-1) * p
    if gh is not None:
        grad -= gh.unsqueeze(-1) * torch.where(p > 0, p * (logp + entropy.unsqueeze(-1)), 0.0)
    at = torch.where(targets >= 0, targets, 0).long()
    grad[torch.arange(len(g), device=g.device), at] += g
    return grad.to(logits.dtype)


def run(state):
    op = state["op"]
    if own:
        from paper_1805_10032_b200 import zeno

        if op == "norm":
            return zeno.layer_norm(state["x"], state["w"], state["b"], eps=1e-5)
        if op == "norm_grad":
            dx = zeno.layer_norm_gradient(state["dy"], state["x"], state["w"], state["mean"], state["rstd"], state["dw"], state["db"])
            return dx, state["dw"], state["db"]
        if op == "pack":
            return tuple(zeno.pack_activations(state["x"]))
        if op == "dense_grad":
            zeno.dense_gradient(state["dy"], state["saved"], state["dw"], state["db"])
            return state["dw"], state["db"]
        if op == "logprobs":
            return tuple(zeno.token_logprobs(state["logits"], state["targets"], top=state["top"]))
        return zeno.token_gradient(state["logits"], state["targets"], state["lse"], state["g"], entropy=state["h"], g_entropy=state["gh"])
    if op == "norm":
        return _norm(state["x"], state["w"], state["b"], 1e-5)
    if op == "norm_grad":
        return _norm_grad(state["dy"], state["x"], state["w"], state["mean"], state["rstd"], state["dw"].dtype)
    if op == "pack":
        return _pack(state["x"])
    if op == "dense_grad":
        dy, x = state["dy"].float(), _unpack(*state["saved"])
        return torch.matmul(dy.transpose(1, 2), x).to(state["dw"].dtype), dy.sum(1).to(state["db"].dtype)
    if op == "logprobs":
        return _logprobs(state["logits"], state["targets"], state["top"])
    return _loss_grad(state["logits"], state["targets"], state["lse"], state["h"], state["g"], state["gh"])


def work(case):
    op = case["op"]
    s = SIZE[case["dtype"]]
    if op in ("logprobs", "loss_grad"):
        elements = case["rows"] * case["vocab"]
        if op == "logprobs":
            return {"bytes": elements * s + case["rows"] * (4 * 4 + 8 * case["top"]), "flops": 5 * elements}
        return {"bytes": 2 * elements * s + case["rows"] * 4 * (5 if case["entropy"] else 3), "flops": 5 * elements}
    rows, p = case["m"] * case["n"], SIZE[case.get("params", "f32")]
    if op == "dense_grad":
        inputs, outputs = case["inputs"], case["outputs"]
        return {"bytes": rows * (outputs * s + inputs + 4 * -(-inputs // BLOCK)) + case["m"] * (inputs + 1) * outputs * p, "flops": 2 * rows * inputs * outputs}
    cols = case["cols"]
    elements = rows * cols
    if op == "pack":
        return {"bytes": elements * (s + 1) + 4 * rows * -(-cols // BLOCK), "flops": 2 * elements}
    if op == "norm":
        return {"bytes": 2 * elements * s + 8 * rows + 2 * cols * p * (case["m"] if case["models"] else 1), "flops": 7 * elements}
    saved = elements * s if case["saved"] == "x" else elements + 4 * rows * -(-cols // BLOCK)
    return {"bytes": 2 * elements * s + saved + 8 * rows + cols * p * (1 + 2 * case["m"]), "flops": 12 * elements}


# ---- the same values from the definitions, in 64 bits

def _code_values(x):
    """The nearest value of four exponent and three mantissa bits to each entry of x (|x| <= 448), ties to an even mantissa, and the scales."""
    t = _blocks(x.double())
    amax = t.abs().amax(-1)
    k = torch.ceil(torch.log2(torch.where(amax > 0, amax, 1.0) / E4M3_MAX))
    k = torch.where(amax > E4M3_MAX * torch.exp2(k), k + 1, k)
    k = torch.where(amax <= E4M3_MAX * torch.exp2(k - 1), k - 1, k).clamp(-117, 119)
    scales = torch.where(amax > 0, torch.exp2(k), 1.0)
    v = (t / scales.unsqueeze(-1)).clamp(-E4M3_MAX, E4M3_MAX)
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(v / step) * step).flatten(-2)[..., : x.shape[-1]], scales


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op in ("logprobs", "loss_grad"):
        parts = []
        for at in range(0, case["rows"], 512):
            z, t = state["logits"][at: at + 512].double(), state["targets"][at: at + 512].long()
            logp = torch.log_softmax(z, -1)
            p = logp.exp()
            entropy = -torch.where(p > 0, p * logp, 0.0).sum(-1)
            hot = torch.zeros_like(z).scatter_(-1, t.clamp(min=0).unsqueeze(-1), 1.0) * (t >= 0).unsqueeze(-1)
            if op == "logprobs":
                got = [torch.where(hot > 0, logp, 0.0).sum(-1), entropy, torch.logsumexp(z, -1)]
                parts.append(got + ([logp.sort(-1, descending=True).values[:, : case["top"]]] if case["top"] else []))
            else:
                grad = state["g"][at: at + 512].double().unsqueeze(-1) * (hot - p * (t >= 0).unsqueeze(-1))
                if state["gh"] is not None:
                    grad -= state["gh"][at: at + 512].double().unsqueeze(-1) * torch.where(p > 0, p * (logp + entropy.unsqueeze(-1)), 0.0)
                parts.append([grad.float() if case["dtype"] == "bf16" else grad])
        got = [torch.cat(p) for p in zip(*parts)]
        return got[0] if op == "loss_grad" else tuple(got[:3]) + ((None, got[3]) if case["top"] else (None, None))
    if op == "pack":
        return _code_values(state["x"])
    if op == "dense_grad":
        dw = []
        for i in range(case["m"]):
            dy, codes, scales = state["dy"][i].double(), state["saved"][0][i], state["saved"][1][i]
            dw.append(torch.einsum("to,ti->oi", dy, _unpack(codes, scales, torch.float64)))
        return torch.stack(dw), torch.einsum("mto->mo", state["dy"].double())
    w, b = state["w"].double(), state["b"].double()
    outs = []
    for i in range(case["m"]):
        wi, bi = (w[i], b[i]) if w.dim() == 2 else (w, b)
        if op == "norm":
            x = state["x"][i].double()
            var, mean = torch.var_mean(x, -1, unbiased=False)
            rstd = (var + 1e-5) ** -0.5
            outs.append(((x - mean[:, None]) * rstd[:, None] * wi + bi, mean, rstd))
            continue
        x = _unpack(state["x"][0][i], state["x"][1][i], torch.float64) if case["saved"] == "8bit" else state["x"][i].double()
        rstd, dy = state["rstd"][i].double(), state["dy"][i].double()
        xh = (x - state["mean"][i].double()[:, None]) * rstd[:, None]
        along = torch.einsum("tc,c,tc->t", dy, wi, xh) / case["cols"]
        dx = rstd[:, None] * (dy * wi - (dy @ wi)[:, None] / case["cols"] - xh * along[:, None])
        outs.append((dx, torch.einsum("tc,tc->c", dy, xh), dy.sum(0)))
    return tuple(torch.stack(o) for o in zip(*outs))
