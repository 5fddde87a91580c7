"""Cases that measure the 8-bit key/value cache and what works on it.

  rotary   rotary positions of queries and keys (half or interleaved pairs, part of a head, frequencies scaled for long contexts), and the gradient
  append   new keys and values into a paged cache of 8-bit codes with a scale for each block of tokens and head, read back as values
  attend   attention of the newest tokens over that cache: single tokens, drafts, prompts
  fork     sequences that share another's pages, then make room for one token each: pages taken, shared last pages copied
  compact  the pages in use moved to the front of the pool, tables and counts following

`run` computes each in elementary torch operations, or with `own` set by the package's entry points.
"""
import math
import random

import torch

own = False

F32, BF16 = "f32", "bf16"
_DT = {F32: torch.float32, BF16: torch.bfloat16}
_SZ = {F32: 4, BF16: 2}


def listed():
    return [
        # the next token of eight sequences, half of each head rotated, frequencies scaled for a long context
        {"name": "rotary_tokens", "kind": "rotary", "T": 8, "H": 32, "kv": 8, "D": 128, "R": 64, "interleaved": False, "stretch": 8.0, "far": 100000, "grad": False, "type": BF16},
        # two sequences of a training step at a 64-head model's sizes, forward and gradient
        {"name": "rotary_train", "kind": "rotary", "T": 16384, "H": 64, "kv": 8, "D": 128, "R": 128, "interleaved": False, "stretch": 1.0, "far": 8192, "grad": True, "type": BF16},
        # 64 sequences decoding, in the middle of their blocks
        {"name": "append_tokens", "kind": "append", "S": 64, "L": 2048, "new": 1, "kv": 8, "D": 128, "page": 64, "block": 16, "type": BF16, "mix": 1},
        # ragged prompts entering the cache
        {"name": "append_prompts", "kind": "append", "S": 6, "L": 8192, "new": 8192, "kv": 8, "D": 128, "page": 64, "block": 16, "type": BF16, "mix": 2},
        # one token of one short sequence of a 16-head model: latency
        {"name": "attend_token", "kind": "attend", "S": 1, "L": 1013, "new": 1, "H": 16, "kv": 8, "D": 128, "page": 64, "block": 16, "window": 0, "type": BF16, "mix": 3},
        # a serving batch of a 64-head model, lengths ragged
        {"name": "attend_batch", "kind": "attend", "S": 64, "L": 16384, "new": 1, "H": 64, "kv": 8, "D": 128, "page": 64, "block": 16, "window": 0, "type": BF16, "mix": 4},
        # one token over a long document, a 32-head model, large blocks
        {"name": "attend_document", "kind": "attend", "S": 1, "L": 131072, "new": 1, "H": 32, "kv": 8, "D": 128, "page": 128, "block": 64, "window": 0, "type": BF16, "mix": 5},
        # drafts of up to five tokens checked in fp32, odd head groups, small pages, a sliding window
        {"name": "attend_drafts", "kind": "attend", "S": 19, "L": 5001, "new": 5, "H": 15, "kv": 3, "D": 64, "page": 16, "block": 8, "window": 1000, "type": F32, "mix": 6},
        # the rest of ragged prompts, whose beginnings are in the cache already
        {"name": "attend_chunks", "kind": "attend", "S": 5, "L": 12000, "new": 1500, "H": 32, "kv": 8, "D": 128, "page": 64, "block": 16, "window": 0, "type": BF16, "mix": 7},
        # a whole prompt of a 64-head model
        {"name": "attend_prompt", "kind": "attend", "S": 1, "L": 8192, "new": 8192, "H": 64, "kv": 8, "D": 128, "page": 64, "block": 16, "window": 0, "type": BF16, "mix": 8},
        # seven more branches of each of eight prompts, four layers
        {"name": "fork_branches", "kind": "fork", "pages": 1024, "S": 64, "from": 8, "L": 6000, "layers": 4, "kv": 8, "D": 128, "page": 64, "block": 16, "mix": 9},
        # a pool half in use after many sequences have left, eight layers
        {"name": "compact_pool", "kind": "compact", "pages": 2048, "S": 48, "L": 4096, "layers": 8, "kv": 8, "D": 128, "page": 64, "block": 16, "mix": 10},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotary", "append", "attend", "attend", "attend", "attend", "fork", "compact"])
    D = rng.choice([64, 64, 80, 96, 112, 128, 128, 128, 192, 256])
    dt = rng.choice([BF16, BF16, F32])
    page = rng.choice([16, 32, 64, 64, 128, 256])
    block = min(page, rng.choice([1, 4, 8, 16, 16, 32, 64, 128]))
    mix = rng.randrange(1 << 20)
    kv = rng.choice([1, 2, 3, 4, 8, 8, 8])
    if kind == "rotary":
        H = kv * rng.choice([1, 2, 4, 5, 7, 8])
        T = max(1, min(_spread(rng, 1, 16384), 16384 * 72 * 128 * 2 // ((H + kv) * D * _SZ[dt])))
        return {"kind": kind, "T": T, "H": H, "kv": kv, "D": D, "R": rng.choice([D, D, D // 2, D // 4 // 2 * 2]), "interleaved": rng.random() < 0.5,
                "stretch": rng.choice([1.0, 4.0, 8.0, 32.0]), "far": _spread(rng, 100, 1000000), "grad": rng.random() < 0.5, "type": dt}
    if kind == "append":
        S, L = _spread(rng, 1, 128), _spread(rng, 1, 8192)
        L = max(1, min(L, 6 * 8192 * 8 * 128 * 2 // (S * kv * D * _SZ[dt])))
        return {"kind": kind, "S": S, "L": L, "new": rng.choice([1, min(L, 7), _spread(rng, 1, L), L]), "kv": kv, "D": D, "page": page, "block": block, "type": dt, "mix": mix}
    if kind == "attend":
        G = rng.choice([1, 2, 4, 5, 7, 8, 16])
        S, L = _spread(rng, 1, 128), _spread(rng, 1, 131072)
        new = min(L, rng.choice([1, 1, 1, rng.randint(2, 9), _spread(rng, 10, 8192)]))
        budget = 8192 ** 2 * 32 * 128 // (_SZ[dt] // 2 * S * kv * G * D)  # pairs of a query and a key in each sequence
        new = min(new, max(1, math.isqrt(budget)), max(1, 2 ** 29 // (S * kv * G * D * _SZ[dt])))
        L = max(1, min(L, 500000 * 8 * 128 // (S * kv * D), budget // new))
        new = min(L, new)
        return {"kind": kind, "S": S, "L": L, "new": new, "H": kv * G, "kv": kv, "D": D, "page": page, "block": block,
                "window": rng.choice([0, 0, 0, _spread(rng, 1, 8192)]), "type": dt, "mix": mix}
    layers, page = rng.randint(1, 8), rng.choice([16, 32, 64, 64])  # the pool a few times the sequences, as a server keeps it
    block = min(block, page)
    S = _spread(rng, 2, 64)
    if kind == "fork":
        src = rng.randint(1, max(1, S // 2))
        L = _spread(rng, 1, 6000)
        pages = src * -(-L // page) + 3 * S + 64
        while layers > 1 and pages * layers * kv * page * D > 2 ** 28:
            layers -= 1
        return {"kind": kind, "pages": pages, "S": S, "from": src, "L": L, "layers": layers, "kv": kv, "D": D, "page": page, "block": block, "mix": mix}
    L = _spread(rng, 1, 4096)
    pages = 2 * S * -(-L // page) + rng.randint(0, 99)
    while layers > 1 and pages * layers * kv * page * D > 2 ** 30:
        layers -= 1
    return {"kind": kind, "pages": pages, "S": S, "L": L, "layers": layers, "kv": kv, "D": D, "page": page, "block": block, "mix": mix}


def _lengths(case):
    """Tokens of each sequence, and how many of them are new, from the case alone."""
    r = random.Random(case["mix"])
    lens = [case["L"]] + [max(1, int(case["L"] * r.uniform(0.15, 1.0))) for _ in range(case["S"] - 1)]
    most = case.get("new", 1)
    new = [min(n, most if i == 0 or most == 1 else max(1, int(most * r.uniform(0.2, 1.0)))) for i, n in enumerate(lens)]
    return lens, new


# ------------------------------------------------------------------ inputs ---
def _frequencies(R, stretch):
    """Angles per position of R / 2 pairs; stretched, the slow ones are divided by `stretch`, with a ramp between one and four turns in 8192 positions."""
    f = 500000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)
    if stretch != 1.0:
        turns = 8192 * f / (2 * math.pi)
        keep = torch.clamp((turns - 1.0) / 3.0, 0.0, 1.0)
        f = keep * f + (1.0 - keep) * f / stretch
    return f.cuda()


def _new_cache(g, layers, pages, c):
    """A cache as earlier steps left it: keys with a few large channels, values, quantized per block of tokens and head."""
    kv, D, page, nb = c["kv"], c["D"], c["page"], c["page"] // c["block"]
    shape = (layers, pages, kv, page, D)
    cache = {n: torch.empty(shape, dtype=torch.uint8, device="cuda") for n in ("k_codes", "v_codes")}
    cache |= {n: torch.empty(shape[:3] + (nb,), device="cuda") for n in ("k_scale", "v_scale")}
    step = max(1, 2 ** 26 // (kv * page * D))
    for n in ("k", "v"):
        gain = torch.ones(kv, 1, D, device="cuda")
        if n == "k":
            gain[:, :, torch.randint(0, D, (max(1, D // 32),), generator=g, device="cuda")] = 6.0
        for la in range(layers):
            for p in range(0, pages, step):
                x = (torch.randn((min(step, pages - p), kv, page, D), generator=g, device="cuda") * gain).view(-1, kv, nb, c["block"], D)
                s = x.abs().amax(dim=(3, 4)) / 127.0
                cache[n + "_scale"][la, p:p + step] = s
                cache[n + "_codes"][la, p:p + step] = (torch.round(x / s[..., None, None]) + 128.0).to(torch.uint8).view(-1, kv, page, D)
    return cache


def _place(g, lens, page, n_pages):
    """Tables of scattered pages for sequences of these lengths (-1 behind them), and how often each page is used."""
    need = [-(-n // page) for n in lens]
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    tables = torch.full((len(lens), max(need) + 2), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(need):
        tables[i, :n] = order[at:at + n]
        at += n
    used = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    used[order[:at].long()] = 1
    return tables, used


def _i32(values):
    return torch.tensor(values, dtype=torch.int32).cuda()


def _starts(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    randn = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    c, kind = dict(case), case["kind"]
    s = {"case": c}
    if kind == "rotary":
        dt, T = _DT[c["type"]], c["T"]
        s["q"], s["k"] = randn(T, c["H"], c["D"]).to(dt), randn(T, c["kv"], c["D"]).to(dt)
        if c["grad"]:
            s["dq"], s["dk"] = randn(T, c["H"], c["D"]).to(dt), randn(T, c["kv"], c["D"]).to(dt)
            s["positions"] = torch.arange(T, device="cuda") % c["far"]
        else:
            s["positions"] = torch.randint(0, c["far"], (T,), generator=g, device="cuda")
        s["inv_freq"] = _frequencies(c["R"], c["stretch"])
        s["amplitude"] = 1.0 if c["stretch"] == 1.0 else 0.1 * math.log(c["stretch"]) + 1.0  # sharper attention over the longer context
    elif kind in ("append", "attend"):
        lens, new = _lengths(c)
        s["lens"], s["new"] = lens, new
        pages = sum(-(-n // c["page"]) for n in lens)
        pages += pages // 8 + 4
        s["cache"] = _new_cache(g, 1, pages, c)
        s["tables"], _ = _place(g, lens, c["page"], pages)
        at = _starts(new)
        s["starts_host"], s["starts"], s["lengths"] = at, _i32(at), _i32(lens)
        if kind == "append":
            s["positions"] = torch.cat([torch.arange(n - m, n) for n, m in zip(lens, new)]).cuda()
            s["k"], s["v"] = (1.3 * randn(at[-1], c["kv"], c["D"])).to(_DT[c["type"]]), randn(at[-1], c["kv"], c["D"]).to(_DT[c["type"]])
            first = [(n - m) // c["block"] * c["block"] for n, m in zip(lens, new)]  # what the new tokens' blocks held before is read back too
            s["read_starts"] = _i32(_starts([n - f for n, f in zip(lens, first)]))
            s["read_positions"] = torch.cat([torch.arange(f, n) for n, f in zip(lens, first)]).cuda()
            s["read_rows"] = torch.cat([torch.full((n - f,), i) for i, (n, f) in enumerate(zip(lens, first))]).cuda()
            s["rows"] = torch.cat([torch.full((m,), i) for i, m in enumerate(new)]).cuda()
        else:
            s["q"] = randn(at[-1], c["H"], c["D"]).to(_DT[c["type"]])
    elif kind == "fork":
        lens, _ = _lengths({**c, "S": c["from"]})
        s["cache"] = _new_cache(g, c["layers"], c["pages"], c)
        tables, s["used"] = _place(g, lens, c["page"], c["pages"])
        s["tables"] = torch.full((c["S"], tables.shape[1]), -1, dtype=torch.int32, device="cuda")
        s["tables"][:c["from"]] = tables
        s["lengths"] = _i32(lens + [0] * (c["S"] - c["from"]))
        s["src"], s["dst"] = _i32([i % c["from"] for i in range(c["from"], c["S"])]), _i32(list(range(c["from"], c["S"])))
        s["starts"] = _i32(_starts([0] * c["from"] + [1] * (c["S"] - c["from"])))  # the branches go on, the prompts stay
        s["rows"] = s["dst"].long()
    else:
        lens, _ = _lengths(c)
        s["cache"] = _new_cache(g, c["layers"], c["pages"], c)
        s["tables"], s["used"] = _place(g, lens, c["page"], c["pages"])
        s["lengths"] = _i32(lens)
    if own:
        _buffers(s)
    return s


def _buffers(s):
    """The handles, outputs and workspaces, which a user's program keeps."""
    import paper_2609_00049_gb300 as rq
    c, kind = s["case"], s["case"]["kind"]
    if "cache" in s:
        s["handle"] = rq.kv_cache(**s["cache"])
    if kind == "rotary":
        s["out"] = {n: torch.empty_like(s[n]) for n in ("q", "k", "dq", "dk") if n in s}
    elif kind == "append":
        new = lambda: torch.empty((s["read_positions"].numel(), c["kv"], c["D"]), dtype=_DT[c["type"]], device="cuda")  # noqa: E731
        s["out"] = {"k": new(), "v": new()}
    elif kind == "attend":
        s["out"] = {"out": torch.empty_like(s["q"]), "lse": torch.empty(s["q"].shape[:2], device="cuda")}
        s["ws"] = rq.workspace(rq.realq_kv_attention_workspace_size(s["handle"], c["S"], s["q"].shape[0], c["H"]))
    else:
        s["ws"] = rq.workspace(rq.realq_pages_workspace_size(c["pages"], *s["tables"].shape))
        s["pages"] = rq.kv_pages(s["used"], s["tables"], s["lengths"])
        if kind == "fork":
            s["positions"] = torch.empty(s["rows"].numel(), dtype=torch.int64, device="cuda")
        else:
            s["out"] = {"used": torch.empty_like(s["used"]), "tables": torch.empty_like(s["tables"]), "moved_to": torch.empty_like(s["used"])}


# --------------------------------------------------------------- operators ---
def run(s):
    return _own_run(s) if own else _plain_run(s)


def _own_run(s):
    import paper_2609_00049_gb300 as rq
    c, kind = s["case"], s["case"]["kind"]
    if kind == "rotary":
        o, how = s["out"], {"interleaved": c["interleaved"], "amplitude": s["amplitude"]}
        rq.realq_rotary(s["q"], s["positions"], s["inv_freq"], o["q"], k=s["k"], k_out=o["k"], **how)
        if c["grad"]:
            rq.realq_rotary(s["dq"], s["positions"], s["inv_freq"], o["dq"], k=s["dk"], k_out=o["dk"], transpose=True, **how)
        return o
    if kind == "append":
        rq.realq_kv_append(s["handle"], 0, s["k"], s["v"], s["starts"], s["positions"], s["tables"])
        rq.realq_kv_read(s["handle"], 0, s["read_starts"], s["read_positions"], s["tables"], s["out"]["k"], s["out"]["v"])
        return s["out"]
    if kind == "attend":
        rq.realq_kv_attention(s["q"], s["handle"], 0, s["starts"], s["lengths"], s["tables"], s["out"]["out"], lse=s["out"]["lse"], window=c["window"],
                              max_new=c["new"], ws=s["ws"])
        return s["out"]
    if kind == "fork":
        rq.realq_pages_fork(s["pages"], s["src"], s["dst"], ws=s["ws"])
        rq.realq_pages_reserve(s["pages"], s["starts"], s["positions"], s["handle"], ws=s["ws"])
        return {"used": s["used"], "tables": s["tables"], "lengths": s["lengths"], "positions": s["positions"], **s["cache"]}
    rq.realq_pages_compact(s["pages"], s["handle"], s["out"]["used"], s["out"]["tables"], s["out"]["moved_to"], ws=s["ws"])
    return {**s["out"], **s["cache"]}


def _rotate(x, cos, sin, R, interleaved):
    x, out = x.float(), x.float().clone()
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if interleaved else (x[..., :R // 2], x[..., R // 2:R])
    u, w = a * cos - b * sin, b * cos + a * sin
    if interleaved:
        out[..., 0:R:2], out[..., 1:R:2] = u, w
    else:
        out[..., :R // 2], out[..., R // 2:R] = u, w
    return out


def _append(codes, scale, x, rows, positions, tables, page, block):
    """Codes and scales of one layer after the tokens x (T x kv x D) have been put at their places."""
    nb, x = page // block, x.float()
    pg, slot = tables[rows, positions // page].long(), positions % page
    at = (pg * nb + slot // block)[:, None].expand(-1, x.shape[1])
    by_block = lambda t: t.transpose(1, 2).reshape(-1, x.shape[1])  # noqa: E731
    back = lambda t: t.view(-1, nb, x.shape[1]).transpose(1, 2)     # noqa: E731
    old = by_block(scale)
    fresh = torch.zeros_like(old).scatter_reduce_(0, at, (slot % block == 0).float()[:, None].expand_as(at).contiguous(), "amax")
    have = torch.where(fresh > 0, torch.zeros_like(old), old)
    top = (torch.zeros_like(old).scatter_reduce_(0, at, x.abs().amax(dim=2), "amax").double() / 127.0).float()  # (in 32 bits torch multiplies by 1 / 127)
    touched = torch.zeros_like(old).scatter_(0, at, 1.0) > 0
    now = torch.where(touched, torch.maximum(have, top), old)
    ratio = torch.where(touched & (now > have) & (have > 0), have / now, torch.ones_like(old))
    r = back(ratio).repeat_interleave(block, dim=2)[..., None]
    codes.copy_((torch.round((codes.float() - 128.0) * r) + 128.0).to(torch.uint8))
    scale.copy_(back(now))
    mine = now.gather(0, at)
    q = torch.where(mine[..., None] > 0, torch.round(x / mine[..., None]), torch.zeros_like(x))
    codes[pg, :, slot] = (torch.clamp(q, -127, 127) + 128.0).to(torch.uint8)


def _read(codes, scale, rows, positions, tables, page, block):
    pg, slot = tables[rows, positions // page].long(), positions % page
    return (codes[pg, :, slot].float() - 128.0) * scale[pg, :, slot // block][..., None]


def _values(codes, scale, pages, n, block):
    """The first n tokens on these pages: kv x n x D."""
    x = (codes[pages].float() - 128.0) * scale[pages].repeat_interleave(block, dim=2)[..., None]
    return x.transpose(0, 1).reshape(codes.shape[1], -1, codes.shape[3])[:, :n]


def _attend(s):
    c, q = s["case"], s["q"].float()
    G, at = c["H"] // c["kv"], s["starts_host"]
    cache = {n: t[0] for n, t in s["cache"].items()}
    out = torch.empty_like(s["q"])
    lse = torch.empty(q.shape[:2], device="cuda")
    for i, (L, m) in enumerate(zip(s["lens"], s["new"])):
        pages = s["tables"][i, :-(-L // c["page"])].long()
        K, V = _values(cache["k_codes"], cache["k_scale"], pages, L, c["block"]), _values(cache["v_codes"], cache["v_scale"], pages, L, c["block"])
        key = torch.arange(L, device="cuda")
        step = max(1, 2 ** 28 // (L * c["H"]))
        for a in range(0, m, step):
            b = min(m, a + step)
            place = torch.arange(L - m + a, L - m + b, device="cuda")[:, None]
            seen = key <= place
            if c["window"]:
                seen = seen & (key > place - c["window"])
            x = q[at[i] + a:at[i] + b].view(b - a, c["kv"], G, c["D"]).permute(1, 2, 0, 3).reshape(c["kv"], -1, c["D"])
            score = (x @ K.transpose(1, 2)) * (1.0 / math.sqrt(c["D"]))
            score = score.view(c["kv"], G, b - a, L).masked_fill(~seen, -math.inf)
            top = score.amax(dim=3, keepdim=True)
            e = torch.exp(score - top)
            total = e.sum(dim=3, keepdim=True)
            y = (e.view(c["kv"], -1, L) @ V).view(c["kv"], G, b - a, c["D"]) / total
            out[at[i] + a:at[i] + b] = y.permute(2, 0, 1, 3).reshape(b - a, c["H"], c["D"]).to(out.dtype)
            lse[at[i] + a:at[i] + b] = (top + torch.log(total))[..., 0].permute(2, 0, 1).reshape(b - a, c["H"])
    return {"out": out, "lse": lse}


def _count(used, tables, by):
    used += torch.zeros(used.numel() + 1, dtype=torch.int32, device="cuda").scatter_add_(
        0, torch.where(tables >= 0, tables, torch.full_like(tables, used.numel())).reshape(-1).long(), torch.full((tables.numel(),), by, dtype=torch.int32, device="cuda"))[:-1]


def _fork(s):
    c, used, tables, lengths, page = s["case"], s["used"], s["tables"], s["lengths"], s["case"]["page"]
    src, dst = s["src"].long(), s["dst"].long()
    mine, their_len = tables[src], lengths[src]
    _count(used, tables[dst], -1)
    _count(used, mine, 1)
    tables[dst], lengths[dst] = mine, their_len
    # room for one more token in each branch: a new page where the last one is full, a copy where it is shared
    n, rows = used.numel(), s["rows"]
    L = lengths[rows].long()
    last = tables[rows, (L // page).clamp(max=tables.shape[1] - 1)].long()
    at = torch.where(last >= 0, last, torch.full_like(last, n))
    full = L % page == 0
    partial = ~full & (last >= 0)
    writers = torch.zeros(n + 1, dtype=torch.int32, device="cuda").scatter_add_(0, at, partial.int())
    order = torch.arange(rows.numel(), dtype=torch.int32, device="cuda")
    latest = torch.full((n + 1,), -1, dtype=torch.int32, device="cuda").scatter_reduce_(0, at, torch.where(partial, order, torch.full_like(order, -1)), "amax")
    holders = torch.cat([used, used.new_zeros(1)])
    keeps = partial & (latest[at] == order) & (writers[at] == holders[at])
    copies = partial & ~keeps
    takes = full | copies
    free = torch.argsort((used > 0).to(torch.int8), stable=True)
    got = free[(torch.cumsum(takes.int(), 0) - 1).clamp(min=0)]
    dump = torch.full_like(got, n)
    comes_from = torch.arange(n + 1, device="cuda")
    comes_from[torch.where(copies, got, dump)] = torch.where(copies, last, dump)
    counts = torch.cat([used, used.new_zeros(1)])
    counts.scatter_add_(0, torch.where(copies, at, dump), torch.full_like(order, -1))
    counts.scatter_add_(0, torch.where(takes, got, dump), torch.ones_like(order))
    used.copy_(counts[:-1])
    tables[rows, L // page] = torch.where(takes, got, last).int()
    lengths[rows] += 1
    for t in s["cache"].values():
        t.copy_(t[:, comes_from[:-1]])
    return {"used": used, "tables": tables, "lengths": lengths, "positions": L, **s["cache"]}


def _compact(s):
    used, n = s["used"], s["used"].numel()
    live = used > 0
    count = live.sum()
    page = torch.arange(n, device="cuda")
    moves, hole = live & (page >= count), ~live & (page < count)
    holes = torch.argsort((~hole).to(torch.int8), stable=True)  # the holes first, in order
    to = torch.where(moves, holes[(torch.cumsum(moves.int(), 0) - 1).clamp(min=0)], page)
    moved_to = torch.where(live, to, torch.full_like(to, -1)).int()
    comes_from = torch.arange(n + 1, device="cuda")
    comes_from[torch.where(moves, to, torch.full_like(to, n))] = torch.where(moves, page, torch.full_like(to, n))
    used_out = torch.zeros(n + 1, dtype=torch.int32, device="cuda").scatter_(0, torch.where(live, to, torch.full_like(to, n)), torch.where(live, used, torch.zeros_like(used)))[:-1]
    tables = torch.where(s["tables"] >= 0, moved_to[s["tables"].clamp(min=0).long()], s["tables"])
    for t in s["cache"].values():
        t.copy_(t[:, comes_from[:-1]])
    return {"used": used_out, "tables": tables, "moved_to": moved_to, **s["cache"]}


def _plain_run(s):
    c, kind = s["case"], s["case"]["kind"]
    if kind == "rotary":
        turn = s["positions"].double()[:, None] * s["inv_freq"]  # in 64 bits: far positions turn many times
        cos, sin = [(s["amplitude"] * f(turn)).float()[:, None] for f in (torch.cos, torch.sin)]
        out = {n: _rotate(s[n], cos, sin, c["R"], c["interleaved"]).to(s[n].dtype) for n in ("q", "k")}
        if c["grad"]:
            out |= {n: _rotate(s[n], cos, -sin, c["R"], c["interleaved"]).to(s[n].dtype) for n in ("dq", "dk")}
        return out
    if kind == "append":
        out = {}
        for n in ("k", "v"):
            codes, scale = s["cache"][n + "_codes"][0], s["cache"][n + "_scale"][0]
            _append(codes, scale, s[n], s["rows"], s["positions"], s["tables"], c["page"], c["block"])
            out[n] = _read(codes, scale, s["read_rows"], s["read_positions"], s["tables"], c["page"], c["block"]).to(s[n].dtype)
        return out
    return {"attend": _attend, "fork": _fork, "compact": _compact}[kind](s)


def _visible(L, m, window):
    """How many keys the m newest of L tokens see in all, and how many keys any of them sees."""
    first = L - m
    if not window:
        return m * first + m * (m + 1) // 2, L
    pairs = sum(min(p + 1, window) for p in (first, L - 1)) * m // 2 if m * window > 2 ** 24 else sum(min(p + 1, window) for p in range(first, L))
    return pairs, L - max(0, first - window + 1)


def work(case):
    """What each operator has to read and write once, and its arithmetic."""
    c, kind = case, case["kind"]
    if kind == "rotary":
        passes, values = 2 if c["grad"] else 1, c["T"] * (c["H"] + c["kv"])
        return {"bytes": passes * (2 * values * c["D"] * _SZ[c["type"]] + 8 * c["T"] + 4 * c["R"]), "flops": passes * 3 * values * c["R"]}
    token = c["kv"] * 2 * (c["D"] + 4.0 / c["block"])  # a cached token's codes and its share of the scales
    if kind in ("append", "attend"):
        lens, new = _lengths(c)
    if kind == "append":
        held = sum((n - m) % c["block"] for n, m in zip(lens, new))
        T = sum(new)
        return {"bytes": int(T * c["kv"] * 2 * c["D"] * _SZ[c["type"]] + (2 * T + 3 * held) * token + (T + held) * c["kv"] * 2 * c["D"] * _SZ[c["type"]] + 16 * T),
                "flops": 8 * T * c["kv"] * c["D"]}
    if kind == "attend":
        seen = [_visible(n, m, c["window"]) for n, m in zip(lens, new)]
        io = sum(new) * c["H"] * (2 * c["D"] * _SZ[c["type"]] + 4)
        return {"bytes": int(sum(k for _, k in seen) * (token + 4.0 / c["page"]) + io), "flops": 4 * c["D"] * c["H"] * sum(p for p, _ in seen)}
    if kind == "fork":
        lens, _ = _lengths({**c, "S": c["from"]})
        copied = sum(1 for i in range(c["from"], c["S"]) if lens[i % c["from"]] % c["page"])
        entries = sum(-(-lens[i % c["from"]] // c["page"]) for i in range(c["from"], c["S"]))
        return {"bytes": int(2 * copied * c["page"] * token * c["layers"] + 12 * entries + 8 * c["pages"]), "flops": 2 * entries}
    lens, _ = _lengths(c)
    live = sum(-(-n // c["page"]) for n in lens)
    moved = live * (c["pages"] - live) // c["pages"]  # as many of them as lie behind, on average
    return {"bytes": int(2 * moved * c["page"] * token * c["layers"] + 8 * live + 12 * c["pages"]), "flops": c["pages"]}


# ------------------------------------------------------------ in 64 bits ---
def exact(case, seed):
    c, kind = case, case["kind"]
    if kind in ("fork", "compact"):
        return None  # whole numbers and copies
    if kind == "attend" and c["D"] * c["H"] * sum(n * m for n, m in zip(*_lengths(c))) > 2e12:
        return None
    s = prepare(case, seed)
    if kind == "rotary":
        z = torch.polar(torch.full_like(s["inv_freq"], s["amplitude"]).expand(c["T"], -1), torch.outer(s["positions"].double(), s["inv_freq"]))[:, None]
        out = {}
        for n in ("q", "k", "dq", "dk"):
            if n not in s:
                continue
            y = s[n].double()
            pairs = y[..., :c["R"]].unflatten(-1, (-1, 2)) if c["interleaved"] else y[..., :c["R"]].unflatten(-1, (2, -1)).transpose(-1, -2)
            turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * (z.conj() if n[0] == "d" else z))
            y[..., :c["R"]] = turned.flatten(-2) if c["interleaved"] else turned.transpose(-1, -2).flatten(-2)
            out[n] = y.float() if y.numel() > 2 ** 27 else y
        return out
    if kind == "append":
        return {n: _exact_append(s, n) for n in ("k", "v")}
    outs, lses = [], []
    at, G = s["starts_host"], c["H"] // c["kv"]
    for i, (L, m) in enumerate(zip(s["lens"], s["new"])):
        place = torch.arange(L, device="cuda")
        pg, slot = s["tables"][i].long()[place // c["page"]], place % c["page"]
        K, V = [torch.mul(s["cache"][n + "_codes"][0][pg, :, slot].double() - 128, s["cache"][n + "_scale"][0][pg, :, slot // c["block"]].double()[..., None])
                for n in ("k", "v")]
        y, z = torch.empty(m, c["H"], c["D"], dtype=torch.float64, device="cuda"), torch.empty(m, c["H"], dtype=torch.float64, device="cuda")
        step = max(1, 2 ** 28 // L)
        for h in range(c["H"]):
            for a in range(0, m, step):
                at_q = torch.arange(L - m + a, L - m + min(m, a + step), device="cuda")
                x = torch.mm(s["q"][at[i] + a:at[i] + a + len(at_q), h].double(), K[:, h // G].t()) / c["D"] ** 0.5
                ago = at_q[:, None] - place
                x[(ago < 0) | ((ago >= c["window"]) if c["window"] else (ago < 0))] = -math.inf
                z[a:a + len(at_q), h] = torch.logsumexp(x, dim=1)
                y[a:a + len(at_q), h] = torch.softmax(x, dim=1) @ V[:, h // G]
        outs.append(y)
        lses.append(z)
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}


def _exact_append(s, n):
    """Sequence by sequence and block by block.  Scales, ratios and quotients are fp32 numbers by definition: 64 bits, rounded to them."""
    c = s["case"]
    page, block = c["page"], c["block"]
    nearest = lambda t: t.float().double()  # noqa: E731
    codes, scale, x = s["cache"][n + "_codes"][0], s["cache"][n + "_scale"][0].double(), s[n].double()
    parts = []
    for i, (L, m) in enumerate(zip(s["lens"], s["new"])):
        first = (L - m) // block * block
        place = torch.arange(first, L, device="cuda")
        pg, slot = s["tables"][i].long()[place // page], place % page
        v = codes[pg, :, slot].double() - 128
        old = scale[pg, :, slot // block]
        mine = x[s["starts_host"][i]:s["starts_host"][i + 1]]
        is_new = place >= L - m
        fill = -len(place) % block
        rows = torch.zeros(len(place), *mine.shape[1:], dtype=torch.float64, device="cuda")
        rows[is_new] = mine
        by = torch.nn.functional.pad(rows, (0, 0, 0, 0, 0, fill)).unflatten(0, (-1, block))
        peak = nearest(by.abs().amax(dim=(1, 3)) / 127)
        had = old[::block].clone()
        had[is_new[::block]] = 0.0  # the block starts with a new token
        now = torch.maximum(had, peak)
        shrink = torch.where(had > 0, nearest(had / now.clamp(min=1e-300)), torch.ones_like(now))
        each = lambda t: t.repeat_interleave(block, dim=0)[:len(place), :, None]  # noqa: E731
        kept = torch.round(nearest(v * each(shrink)))
        put = torch.round(nearest(rows / each(now).clamp(min=1e-300))).clamp(-127, 127)
        parts.append(torch.where(is_new[:, None, None], put, kept) * each(now))
    return torch.cat(parts)
