"""Cases that measure the 8-bit linear operators and the token log probabilities.

  product        Y = diag(x_scale) (Xc - 128) (Wc - zero)^T diag(w_scale): 8-bit token codes times 8- or 4-bit channel codes
  logprobs       log probability of each row's given token, the row's maximum, log sum and entropy, its k likeliest tokens
  logprobs_grad  the gradient of those numbers with respect to the logits
  checkpoint     activations to 8-bit codes with one power-of-two scale per 32 of a token's values, and back
  weight_grad    dW = dY^T X from the 8-bit codes of X

`run` computes each in elementary torch operations, or with `own` set by the package's entry points.
"""
import math

import torch

own = False

F32, BF16 = "f32", "bf16"
_DT = {F32: torch.float32, BF16: torch.bfloat16}
_SZ = {F32: 4, BF16: 2}
BLOCK = 32


def listed():
    return [
        # one token through a 1024-wide model's query projection: latency
        {"name": "product_token", "kind": "product", "T": 1, "n": 1024, "m": 2048, "w_bits": 8, "zeros": False, "y": BF16},
        # eight sequences decoding through an 8192 -> 28672 projection, the sweep's own 4-bit codes and zero points
        {"name": "product_decode8_w4", "kind": "product", "T": 8, "n": 8192, "m": 28672, "w_bits": 4, "zeros": True, "y": BF16},
        # a ragged batch of short prompts through a 5120 -> 25600 projection, fp32 results
        {"name": "product_batch", "kind": "product", "T": 201, "n": 5120, "m": 25600, "w_bits": 8, "zeros": False, "y": F32},
        # a prompt batch through an 8192 x 8192 projection
        {"name": "product_prompt", "kind": "product", "T": 8192, "n": 8192, "m": 8192, "w_bits": 8, "zeros": False, "y": BF16},
        # one decoded token with its 20 alternatives, some of the vocabulary masked out
        {"name": "logprobs_token", "kind": "logprobs", "T": 1, "V": 128256, "logits": BF16, "k": 20, "masked": True},
        # perplexity of a chunk of text: two sequences of 2048 tokens
        {"name": "logprobs_text", "kind": "logprobs", "T": 4096, "V": 128256, "logits": BF16, "k": 5, "masked": False},
        # a short sequence over an odd vocabulary in fp32, masked
        {"name": "logprobs_grad_odd", "kind": "logprobs_grad", "T": 333, "V": 50257, "logits": F32, "k": 4, "masked": True},
        # the loss's gradient for two sequences of 2048 tokens
        {"name": "logprobs_grad_text", "kind": "logprobs_grad", "T": 4096, "V": 128256, "logits": BF16, "k": 0, "masked": False},
        # a ragged short sequence of an odd width in fp32
        {"name": "checkpoint_short", "kind": "checkpoint", "T": 77, "n": 1111, "x": F32},
        # a layer's inputs for 16384 tokens of an 8192-wide model
        {"name": "checkpoint_layer", "kind": "checkpoint", "T": 16384, "n": 8192, "x": BF16},
        # a key projection's gradient from one ragged sequence, fp32 output gradients
        {"name": "weight_grad_kv", "kind": "weight_grad", "T": 1999, "m": 1024, "n": 4096, "dy": F32},
        # an 8192 x 8192 projection's gradient from 8192 tokens
        {"name": "weight_grad_layer", "kind": "weight_grad", "T": 8192, "m": 8192, "n": 8192, "dy": BF16},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["product", "product", "logprobs", "logprobs_grad", "checkpoint", "weight_grad"])
    if kind == "product":
        T, n, m = _spread(rng, 1, 8192), _spread(rng, 200, 28672), _spread(rng, 200, 28672)
        if rng.random() < 0.6:  # most widths of real layers are multiples of 64
            n, m = max(64, n // 64 * 64), max(64, m // 64 * 64)
        T = max(1, min(T, 8192 ** 3 // (n * m)))
        return {"kind": kind, "T": T, "n": n, "m": m, "w_bits": rng.choice([8, 8, 4]), "zeros": rng.random() < 0.5, "y": rng.choice([F32, BF16])}
    if kind in ("logprobs", "logprobs_grad"):
        T, V, dt = _spread(rng, 1, 4096), _spread(rng, 1000, 160000), rng.choice([F32, BF16])
        T = max(1, min(T, 4096 * 128256 * 2 // (V * _SZ[dt])))
        return {"kind": kind, "T": T, "V": V, "logits": dt, "k": rng.choice([0, 1, 5, 20, 32] if kind == "logprobs" else [0, 3, 8]), "masked": rng.random() < 0.5}
    if kind == "checkpoint":
        T, n, dt = _spread(rng, 1, 16384), _spread(rng, 64, 28672), rng.choice([F32, BF16])
        T = max(1, min(T, 16384 * 8192 * 2 // (n * _SZ[dt])))
        return {"kind": kind, "T": T, "n": n, "x": dt}
    T, n, m, dt = _spread(rng, 16, 16384), _spread(rng, 200, 28672), _spread(rng, 200, 28672), rng.choice([F32, BF16])
    if rng.random() < 0.6:
        n, m = max(64, n // 64 * 64), max(64, m // 64 * 64)
    T = max(16, min(T, 8192 ** 3 // (n * m) // (3 if dt == F32 else 1)))
    return {"kind": kind, "T": T, "m": m, "n": n, "dy": dt}


# ------------------------------------------------------------------ inputs ---
def _activations(g, T, n):
    """Normal values with a few channels an order of magnitude larger, as the inputs of a decoder block's projections have."""
    x = torch.randn(T, n, generator=g, device="cuda")
    big = torch.randint(0, n, (max(1, n // 256),), generator=g, device="cuda")
    x[:, big] *= 12.0
    return x


def _codes8(x):
    """Symmetric 8-bit codes of each row (zero point 128) and their scales."""
    xmax = x.abs().amax(dim=1)
    scale = 2.0 * torch.where(xmax == 0, torch.ones_like(xmax), xmax) / 255.0
    return torch.clamp(torch.round(x / scale[:, None]) + 128.0, 0, 255).to(torch.uint8), scale


def _codes4(w, zeros):
    """4-bit codes of each row, two to a byte (even column in the low nibble), their scales and zero points."""
    if zeros:
        lo, hi = w.amin(dim=1).clamp(max=0), w.amax(dim=1).clamp(min=0)
        scale = (hi - lo) / 15.0
        zero = torch.clamp(torch.round(-lo / scale), 0, 15)
    else:
        scale = 2.0 * w.abs().amax(dim=1) / 15.0
        zero = torch.full_like(scale, 8.0)
    q = torch.clamp(torch.round(w / scale[:, None]) + zero[:, None], 0, 15).to(torch.uint8)
    if q.shape[1] % 2:
        q = torch.cat([q, torch.zeros_like(q[:, :1])], dim=1)
    return (q[:, 0::2] | (q[:, 1::2] << 4)).contiguous(), scale, zero.to(torch.uint8)


def _blocks(x):
    T, n = x.shape
    nb = -(-n // BLOCK)
    return torch.nn.functional.pad(x, (0, nb * BLOCK - n)).reshape(T, nb, BLOCK)


def _pack(x):
    """Codes (T x n int8) and scale bytes (T x ceil(n / 32)): value = code 2^(byte - 133), byte = 127 + the exponent of the block's largest magnitude."""
    T, n = x.shape
    b = _blocks(x.float())
    amax = b.abs().amax(dim=2)
    byte = torch.where(amax > 0, torch.clamp(torch.frexp(amax).exponent + 126, 0, 254), torch.zeros_like(amax, dtype=torch.int32))
    up = 133 - byte  # by two factors: one alone may pass the range of fp32
    q = torch.round(b * torch.exp2((up // 2).float())[:, :, None] * torch.exp2((up - up // 2).float())[:, :, None])
    return torch.clamp(q, -127, 127).to(torch.int8).reshape(T, -1)[:, :n].contiguous(), byte.to(torch.uint8)


def _unpack(codes, byte):
    T, n = codes.shape
    down = byte.to(torch.int32) - 133
    b = _blocks(codes.float()) * torch.exp2((down // 2).float())[:, :, None] * torch.exp2((down - down // 2).float())[:, :, None]
    return b.reshape(T, -1)[:, :n]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    c, kind, T = dict(case), case["kind"], case["T"]
    s = {"case": c}
    if kind == "product":
        s["x_codes"], s["x_scale"] = _codes8(_activations(g, T, c["n"]))
        w = 0.02 * torch.randn(c["m"], c["n"], generator=g, device="cuda")
        s["w_zero"] = None
        if c["w_bits"] == 8:
            s["w_codes"], s["w_scale"] = _codes8(w)
            if c["zeros"]:
                s["w_zero"] = torch.randint(118, 139, (c["m"],), generator=g, device="cuda").to(torch.uint8)
        else:
            s["w_codes"], s["w_scale"], zero = _codes4(w, c["zeros"])
            s["w_zero"] = zero if c["zeros"] else None
    elif kind in ("logprobs", "logprobs_grad"):
        V, k = c["V"], c["k"]
        x = 2.5 * torch.randn(T, V, generator=g, device="cuda")
        y = torch.randint(0, V, (T,), generator=g, device="cuda")
        rows = torch.arange(T, device="cuda")
        x[rows, y] += 9.0  # most tokens of a text are among the likely ones
        if c["masked"]:  # a grammar's disallowed tokens, and a vocabulary padded at its end
            x[:, torch.randint(0, V, (V // 3,), generator=g, device="cuda")] = -math.inf
            x[:, V - V // 50:] = -math.inf
            x[rows, y.clamp(max=V - V // 50 - 1)] = 4.0
        s["logits"] = x.to(_DT[c["logits"]])
        s["targets"] = torch.where(rows % 16 == 15, torch.full_like(y, -100), y)  # the separators of packed sequences are not scored
        if kind == "logprobs_grad":
            v = s["logits"].float()
            top = v.amax(dim=1)  # what the forward call gave: the row's maximum and the log of its sum
            s["norm"] = torch.stack([top, torch.log(torch.exp(v - top[:, None]).sum(dim=1))], dim=1)
            lp = v - s["norm"][:, :1] - s["norm"][:, 1:]
            s["entropy"] = -torch.where(torch.isfinite(lp), lp.exp() * lp, torch.zeros_like(lp)).sum(dim=1)
            s["d_logprob"] = -torch.rand(T, generator=g, device="cuda") / T
            s["d_entropy"] = 0.01 * torch.randn(T, generator=g, device="cuda") / T
            s["top_ids"] = torch.topk(v, k, dim=1).indices if k else None
            s["d_top"] = 0.1 * torch.randn(T, k, generator=g, device="cuda") / T if k else None
    elif kind == "checkpoint":
        s["x"] = _activations(g, T, c["n"]).to(_DT[c["x"]])
    else:
        s["codes"], s["byte"] = _pack(_activations(g, T, c["n"]).to(torch.bfloat16))
        s["dy"] = (1e-3 * torch.randn(T, c["m"], generator=g, device="cuda")).to(_DT[c["dy"]])
    if own:
        _buffers(s)
    return s


def _buffers(s):
    """The outputs and the workspace, which a user's program allocates once."""
    import paper_2609_00049_gb300 as rq
    c, T = s["case"], s["case"]["T"]
    new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    if c["kind"] == "product":
        s["out"] = new(T, c["m"], dtype=_DT[c["y"]])
        s["ws"] = rq.workspace(rq.realq_int8_product_workspace_size(T, c["n"], c["m"], c["w_bits"]))
    elif c["kind"] == "logprobs":
        s["out"] = {"logprob": new(T), "norm": new(T, 2), "entropy": new(T)}
        if c["k"]:
            s["out"] |= {"top_ids": new(T, c["k"], dtype=torch.int64), "top_logprob": new(T, c["k"])}
    elif c["kind"] == "logprobs_grad":
        s["out"] = torch.empty_like(s["logits"])
    elif c["kind"] == "checkpoint":
        s["codes"], s["byte"] = new(T, c["n"], dtype=torch.int8), new(T, -(-c["n"] // BLOCK), dtype=torch.uint8)
        s["out"] = torch.empty_like(s["x"])
    else:
        s["out"] = new(c["m"], c["n"])
        s["ws"] = rq.workspace(rq.realq_checkpoint_weight_grad_workspace_size(T, c["m"], c["n"], s["dy"].dtype))


# --------------------------------------------------------------- operators ---
def run(s):
    return _own_run(s) if own else _plain_run(s)


def _own_run(s):
    import paper_2609_00049_gb300 as rq
    kind, out = s["case"]["kind"], s["out"]
    if kind == "product":
        rq.realq_int8_product(s["x_codes"], s["x_scale"], s["w_codes"], s["w_scale"], out, w_bits=s["case"]["w_bits"], w_zero=s["w_zero"], ws=s["ws"])
    elif kind == "logprobs":
        rq.realq_token_logprobs(s["logits"], s["targets"], **out)
    elif kind == "logprobs_grad":
        rq.realq_token_logprobs_grad(s["logits"], s["targets"], s["norm"], out, d_logprob=s["d_logprob"], entropy=s["entropy"], d_entropy=s["d_entropy"],
                                     top_ids=s["top_ids"], d_top=s["d_top"])
    elif kind == "checkpoint":
        rq.realq_checkpoint_pack(s["x"], s["codes"], s["byte"])
        rq.realq_checkpoint_unpack(s["codes"], s["byte"], out)
    else:
        rq.realq_checkpoint_weight_grad(s["dy"], s["codes"], s["byte"], out, ws=s["ws"])
    return out


def _weights(s):
    c, w = s["case"], s["w_codes"]
    if c["w_bits"] == 4:
        w = torch.stack([w & 15, w >> 4], dim=2).reshape(w.shape[0], -1)[:, :c["n"]]
    zero = (128 if c["w_bits"] == 8 else 8) if s["w_zero"] is None else s["w_zero"].float()[:, None]
    return w.float() - zero


def _top_keys(v):
    """Whole numbers that order a row by value, equal values by the lower index."""
    bits = (v + 0.0).view(torch.int32).to(torch.int64)
    rank = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)
    return rank * 2 ** 32 + (2 ** 32 - 1 - torch.arange(v.shape[1], device=v.device))


def _plain_run(s):
    c, kind = s["case"], s["case"]["kind"]
    if kind == "product":
        y = (s["x_codes"].float() - 128.0) @ _weights(s).T
        return (y * s["x_scale"][:, None] * s["w_scale"]).to(_DT[c["y"]])
    if kind == "checkpoint":
        return _unpack(*_pack(s["x"])).to(s["x"].dtype)
    if kind == "weight_grad":
        return s["dy"].float().T @ _unpack(s["codes"], s["byte"])
    v, y = s["logits"].float(), s["targets"]
    scored = y >= 0
    at = y.clamp(min=0)[:, None]
    if kind == "logprobs":
        top = v.amax(dim=1, keepdim=True)
        e = torch.exp(v - top)
        total = e.sum(dim=1, keepdim=True)
        log_sum = torch.log(total)
        lp = v - top - log_sum
        entropy = -torch.where(e > 0, e / total * lp, torch.zeros_like(lp)).sum(dim=1)
        out = {"logprob": torch.where(scored, lp.gather(1, at)[:, 0], torch.zeros_like(entropy)), "norm": torch.cat([top, log_sum], dim=1), "entropy": entropy}
        if c["k"]:
            ids = 2 ** 32 - 1 - torch.topk(_top_keys(v), c["k"], dim=1).values % 2 ** 32
            best = v.gather(1, ids)
            out["top_ids"] = torch.where(torch.isfinite(best), ids, torch.full_like(ids, -1))
            out["top_logprob"] = best - top - log_sum
        return out
    lp = v - s["norm"][:, :1] - s["norm"][:, 1:]
    p = torch.exp(lp)
    g = torch.where(scored, s["d_logprob"], torch.zeros_like(s["d_logprob"]))
    d = torch.where(p > 0, -p * s["d_entropy"][:, None] * (lp + s["entropy"][:, None]), torch.zeros_like(p))
    d.scatter_add_(1, at, g[:, None])
    if c["k"]:
        d.scatter_add_(1, s["top_ids"], s["d_top"])
        g = g + s["d_top"].sum(dim=1)
    return (d - p * g[:, None]).to(s["logits"].dtype)


def work(case):
    """What each operator has to read and write once, and its arithmetic (the exponentials and sums of a row counted as six operations a value)."""
    c, kind, T = case, case["kind"], case["T"]
    if kind == "product":
        n, m = c["n"], c["m"]
        w = m * n if c["w_bits"] == 8 else m * ((n + 1) // 2)
        return {"bytes": T * n + w + 4 * T + 4 * m + (m if c["zeros"] else 0) + T * m * _SZ[c["y"]], "flops": 2 * T * n * m}
    if kind == "logprobs":
        return {"bytes": T * (c["V"] * _SZ[c["logits"]] + 8 + 16 + 12 * c["k"]), "flops": 6 * T * c["V"]}
    if kind == "logprobs_grad":
        return {"bytes": T * (2 * c["V"] * _SZ[c["logits"]] + 8 + 20 + 12 * c["k"]), "flops": 6 * T * c["V"]}
    if kind == "checkpoint":  # values in, codes and scales out, and back again
        return {"bytes": 2 * T * (c["n"] * (_SZ[c["x"]] + 1) + -(-c["n"] // BLOCK)), "flops": 4 * T * c["n"]}
    n, m = c["n"], c["m"]
    return {"bytes": T * (n + -(-n // BLOCK) + m * _SZ[c["dy"]]) + 4 * m * n, "flops": 2 * T * n * m}


# ------------------------------------------------------------ in 64 bits ---
def exact(case, seed):
    c, kind, T = case, case["kind"], case["T"]
    s = prepare(case, seed)
    if kind == "product":
        x = s["x_codes"].double().sub_(128)
        w = s["w_codes"]
        if c["w_bits"] == 4:
            full = torch.empty(w.shape[0], 2 * w.shape[1], dtype=torch.float64, device="cuda")
            full[:, 0::2], full[:, 1::2] = (w % 16).double(), (w // 16).double()
            w = full[:, :c["n"]]
        else:
            w = w.double()
        w = w - (s["w_zero"].double()[:, None] if s["w_zero"] is not None else 2.0 ** (c["w_bits"] - 1))
        return torch.mm(x, w.t()) * torch.outer(s["x_scale"].double(), s["w_scale"].double())
    if kind == "checkpoint":
        # the nearest multiple of the block's step, at most 127 steps
        x = s["x"].double()
        out = torch.empty_like(x)
        for j in range(0, c["n"], BLOCK):
            b = x[:, j:j + BLOCK]
            amax = b.abs().amax(dim=1, keepdim=True)
            exponent = (amax.clamp(min=2.0 ** -126).view(torch.int64) >> 52) - 6  # biased; a power from its bits is exact, so ties stay ties
            step = (exponent << 52).view(torch.float64)
            out[:, j:j + BLOCK] = torch.minimum(torch.maximum(torch.round(b / step), b.new_tensor(-127)), b.new_tensor(127)) * step
        return out
    if kind == "weight_grad":
        step = ((s["byte"].to(torch.int64) - 133 + 1023) << 52).view(torch.float64)
        x = s["codes"].double() * step.repeat_interleave(BLOCK, dim=1)[:, :c["n"]]
        return torch.mm(s["dy"].double().t(), x)
    parts = []
    for r in range(0, T, 256):  # 256 rows at a time: a row in 64 bits is about 1 MB
        v, y = s["logits"][r:r + 256].double(), s["targets"][r:r + 256]
        logp = torch.log_softmax(v, dim=1)
        p = torch.softmax(v, dim=1)
        plogp = torch.special.xlogy(p, p)
        mine = torch.zeros_like(v)
        rows = torch.nonzero(y >= 0)[:, 0]
        if kind == "logprobs":
            one = {"logprob": torch.zeros(len(y), dtype=torch.float64, device="cuda"), "entropy": -plogp.sum(dim=1)}
            top = v.max(dim=1).values
            one["norm"] = torch.stack([top, torch.logsumexp(v, dim=1) - top], dim=1)
            one["logprob"][rows] = logp[rows, y[rows]]
            if c["k"]:
                by = torch.sort(v, dim=1, descending=True, stable=True)
                none = by.values[:, :c["k"]] == -math.inf
                one["top_ids"] = by.indices[:, :c["k"]].masked_fill(none, -1)
                one["top_logprob"] = logp.gather(1, by.indices[:, :c["k"]])
        else:
            d = {n: s[n][r:r + 256].double() for n in ("d_logprob", "d_entropy")}
            mine[rows, y[rows]] = d["d_logprob"][rows]
            if c["k"]:
                mine.scatter_add_(1, s["top_ids"][r:r + 256], s["d_top"][r:r + 256].double())
            H = -plogp.sum(dim=1, keepdim=True)
            one = mine - p * mine.sum(dim=1, keepdim=True) - d["d_entropy"][:, None] * (plogp + p * H)
            one = one.float()  # 64 bits of all rows would not fit beside the others
        parts.append(one)
    if kind == "logprobs":
        return {n: torch.cat([p[n] for p in parts]) for n in parts[0]}
    return torch.cat(parts)
