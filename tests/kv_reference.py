"""Plain definitions of the 8-bit key/value cache's operators, in 64 bits, and
caches to try them on.  Nothing of the package is used."""
import math
import random

import torch


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def starts_of(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return i32(out)


class Cache:
    """Buffers of a cache with arbitrary contents, and tables of scattered pages for given lengths."""

    def __init__(self, seed, lens, kv=2, D=64, page=64, block=16, layers=1, spare=3, extra_entries=2, poison=True):
        g, r = gen(seed), random.Random(seed)
        need = [-(-n // page) for n in lens]
        self.n_pages = sum(need) + spare
        self.kv, self.D, self.page, self.block, self.layers, self.lens = kv, D, page, block, layers, lens
        shape = (layers, self.n_pages, kv, page, D)
        self.k_codes = torch.randint(1, 256, shape, generator=g, device="cuda").to(torch.uint8)
        self.v_codes = torch.randint(1, 256, shape, generator=g, device="cuda").to(torch.uint8)
        sc = shape[:3] + (page // block,)
        self.k_scale = torch.exp2(3 * torch.rand(sc, generator=g, device="cuda") - 8)
        self.v_scale = torch.exp2(8 * torch.rand(sc, generator=g, device="cuda") - 12)
        order = list(range(self.n_pages))
        r.shuffle(order)
        width = max(need + [1]) + extra_entries
        rows, at = [], 0
        for n in need:
            rows.append(order[at:at + n] + [-1] * (width - n))
            at += n
        self.rows = rows
        if poison:   # what is behind the sequences' ends may hold anything, and the tables may name anything there
            for i, (n, pages) in enumerate(zip(lens, need)):
                if pages < width:
                    rows[i][pages] = [-1, self.n_pages, 2 ** 31 - 1, -2 ** 31][i % 4]
                if n % page:
                    used = -(-(n % page) // block)
                    p = rows[i][pages - 1]
                    self.k_scale[:, p, :, used:] = math.nan
                    self.v_scale[:, p, :, used:] = [math.nan, math.inf][i % 2]
            for p in order[at:]:
                self.k_scale[:, p] = math.nan
                self.v_scale[:, p] = math.nan
        self.tables = i32(rows)
        self.lengths = i32(lens)

    def buffers(self):
        return dict(k_codes=self.k_codes, v_codes=self.v_codes, k_scale=self.k_scale, v_scale=self.v_scale)

    def values(self, which, layer, s, n=None):
        """Row s's first n tokens: n x kv x D in 64 bits."""
        codes, scale = (self.k_codes, self.k_scale) if which == "k" else (self.v_codes, self.v_scale)
        n = self.lens[s] if n is None else n
        at = torch.arange(n, device="cuda")
        pg, slot = self.tables[s].long()[at // self.page], at % self.page
        return (codes[layer][pg, :, slot].double() - 128) * scale[layer][pg, :, slot // self.block].double()[..., None]


def attention(q, K, V, L, window, causal, scale):
    """One sequence: q m x H x D, K, V L x kv x D.  Outputs, log sums, and what the
    tolerances need: sum_j p_j |v_j|, the largest sum |q||k| of a row's scores."""
    m, H, D = q.shape
    kv = K.shape[1]
    q = q.double().view(m, kv, H // kv, D)
    at = torch.arange(L - m, L, device="cuda")[:, None]
    key = torch.arange(L, device="cuda")
    seen = (key <= at) if causal else torch.ones(m, L, dtype=torch.bool, device="cuda")
    if window:
        seen = seen & (key > at - window)
    s = torch.einsum("mkgd,lkd->mkgl", q, K) * scale
    s = s.masked_fill(~seen[:, None, None, :], -math.inf)
    lse = torch.logsumexp(s, -1) if L else torch.full(s.shape[:-1], -math.inf, dtype=torch.float64, device="cuda")
    p = torch.exp(s - lse[..., None]).nan_to_num(0.0)
    out = torch.einsum("mkgl,lkd->mkgd", p, V)
    mag = torch.einsum("mkgl,lkd->mkgd", p, V.abs())
    big = torch.einsum("mkgd,lkd->mkgl", q.abs(), K.abs()).amax(-1) * abs(scale) if L else torch.zeros_like(lse)
    return out.reshape(m, H, D), lse.reshape(m, H), mag.reshape(m, H, D), big.reshape(m, H)


def append(codes, scale, x, first, table, page, block):
    """One sequence's new tokens (n x kv x D) at positions first .. into one layer's
    codes and scales, in place, block by block.  Scales, ratios, products and
    quotients are fp32 numbers by definition: formed in 64 bits, rounded to them
    (a quotient or product of two fp32 numbers is not changed by the double rounding)."""
    n = x.shape[0]
    x = x.double()
    f = lambda t: t.float().double()   # noqa: E731
    for p0 in range(first // block * block, first + n, block):
        a, b = max(first, p0), min(first + n, p0 + block)
        pg = int(table[p0 // page])
        slot = p0 % page
        new = x[a - first:b - first].transpose(0, 1)                    # kv x tokens x D
        top = new.abs().amax(dim=(1, 2))
        before = scale[pg, :, slot // block].double() if a > p0 else torch.zeros_like(top)
        now = torch.maximum(before, f(top / 127))
        bad = ~torch.isfinite(top) | torch.isnan(before)
        now = torch.where(bad, torch.full_like(now, math.nan), now)
        if a > p0:
            kept = codes[pg, :, slot:slot + a - p0]
            ratio = f(before / now)
            moved = torch.round(f((kept.double() - 128) * ratio[:, None, None])) + 128
            grew = (now > before) & (before > 0)
            codes[pg, :, slot:slot + a - p0] = torch.where(grew[:, None, None], moved.nan_to_num(128.0).to(torch.uint8), kept)
        q = torch.round(f(new / now[:, None, None])).clamp(-127, 127) + 128
        q = torch.where((now > 0)[:, None, None], q, torch.full_like(q, 128.0))
        codes[pg, :, slot + a - p0:slot + b - p0] = q.to(torch.uint8)
        scale[pg, :, slot // block] = now.float()
