"""The 8-bit key/value cache's operators against their definitions in 64 bits.

U(t) = finfo(t).eps / 2 is half a step of type t, relative to the value."""
import math
import random

import pytest
import torch

import paper_2609_00049_gb300 as rq
from kv_reference import Cache, append, attention, gen, i32, starts_of

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def U(t):
    return torch.finfo(t).eps / 2


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2609_00049_gb300 import build as b
    b.build()
    rq.lib()


# ------------------------------------------------------------------ rotary ---
def turned(x, pos, f, interleaved, amplitude, back):
    y = x.double().clone()
    R = 2 * f.numel()
    # the angle modulo a turn from whole numbers: in 64 bits pos f alone is off by |pos f| 2^-53
    t = (pos.double()[:, None] * f)[:, None]
    c, s = amplitude * torch.cos(t), amplitude * torch.sin(t) * (-1 if back else 1)
    a, b = (y[..., 0:R:2], y[..., 1:R:2]) if interleaved else (y[..., :R // 2], y[..., R // 2:R])
    a, b = a.clone(), b.clone()
    u, w = a * c - b * s, b * c + a * s
    m = a.abs() + b.abs()
    mag = torch.zeros_like(y)
    for z, (p, q) in ((y, (u, w)), (mag, (m, m))):
        if interleaved:
            z[..., 0:R:2], z[..., 1:R:2] = p, q
        else:
            z[..., :R // 2], z[..., R // 2:R] = p, q
    return y, mag


def rotary_close(got, x, pos, f, interleaved, amplitude, back, extra=0.0):
    ref, mag = turned(x, pos, f, interleaved, amplitude, back)
    # cosine and sine: 2^-25 turns' conversion (2 pi 2^-26 after rounding to 24 bits) and two steps of sincospif, below 2^-22
    # together; amplitude, two products and a sum: four half steps of fp32; the output's rounding
    tol = (2.0 ** -22 + extra + 4 * U(F32)) * abs(amplitude) * mag + U(got.dtype) * ref.abs()
    assert bool(((got.double() - ref).abs() <= tol + 1e-38).all()), float(((got.double() - ref).abs() - tol).max())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,H,kv,D,R", [(1, 1, 1, 16, 16), (5, 7, 1, 128, 128), (3, 4, 2, 80, 40), (700, 8, 2, 64, 64), (9, 3, 3, 50, 6),
                                        (1, 64, 8, 128, 128), (2500, 2, 1, 256, 128), (4, 2, 2, 1024, 1022)])
def test_rotary(T, H, kv, D, R, interleaved, dtype):
    q, k = torch.randn(T, H, D, generator=gen(0), device="cuda").to(dtype), torch.randn(T, kv, D, generator=gen(1), device="cuda").to(dtype)
    pos = torch.randint(-50, 5000, (T,), generator=gen(2), device="cuda")
    f = rq.realq_rotary_frequencies(R, 10000.0).cuda()
    for back in (False, True):
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        rq.realq_rotary(q, pos, f, qo, k=k, k_out=ko, interleaved=interleaved, amplitude=1.25, transpose=back)
        for got, x in ((qo, q), (ko, k)):
            rotary_close(got, x, pos, f, interleaved, 1.25, back)
            assert torch.equal(got[..., R:], x[..., R:])
    q2 = q.clone()
    rq.realq_rotary(q2, pos, f, q2, interleaved=interleaved, amplitude=1.25, transpose=True)   # in place, without keys
    assert torch.equal(q2, qo)


def test_rotary_far_positions():
    """Positions up to 2^40: the reference's own angle is off by pos f 2^-53 turns and more, so frequencies are whole
    fractions of a turn whose multiples are known."""
    pos = torch.tensor([0, 1, 2 ** 20 + 3, 2 ** 31 - 1, 2 ** 31, 2 ** 40 + 5, -7, -2 ** 33 + 1], device="cuda")
    n = torch.tensor([8, 64, 1024, 2 ** 20], device="cuda")          # frequencies of a turn in n positions
    f = 2 * math.pi / n.double()
    q = torch.randn(8, 2, 8, generator=gen(3), device="cuda")
    out = torch.empty_like(q)
    rq.realq_rotary(q, pos, f, out)
    part = torch.remainder(pos[:, None], n)                          # exact
    ref, mag = turned(q, torch.ones(8, device="cuda"), torch.zeros(4, device="cuda", dtype=torch.float64), False, 1.0, False)
    t = (2 * math.pi * part.double() / n)[:, None]
    a, b = q.double()[..., :4], q.double()[..., 4:]
    ref = torch.cat([a * torch.cos(t) - b * torch.sin(t), b * torch.cos(t) + a * torch.sin(t)], dim=-1)
    # the frequency is a double: |pos| f 2^-53 radians and the same from 1 / 2 pi and the product, at 2^40 / 8 turns below 2^-13 radians
    drift = 3 * pos.abs().double()[:, None, None] * f.repeat(2) * 2.0 ** -53
    assert bool(((out.double() - ref).abs() <= (2.0 ** -22 + 4 * U(F32) + drift) * mag + U(F32) * ref.abs()).all())


def test_rotary_of_views_and_gradient():
    """q and k as parts of one projection's output; the transpose is the gradient, by differences."""
    T, H, kv, D = 6, 4, 2, 32
    qkv = torch.randn(T, (H + 2 * kv) * D, generator=gen(4), device="cuda")
    heads = qkv.view(T, H + 2 * kv, D)
    q, k = heads[:, :H], heads[:, H:H + kv]
    v0 = heads[:, H + kv:].clone()
    pos, f = torch.arange(T, device="cuda") * 13, rq.realq_rotary_frequencies(24, 1000.0).cuda()
    qo, ko = torch.empty(T, H, D, device="cuda"), torch.empty(T, kv, D, device="cuda")
    rq.realq_rotary(q, pos, f, qo, k=k, k_out=ko, amplitude=0.7)
    for got, x in ((qo, q), (ko, k)):
        rotary_close(got, x, pos, f, False, 0.7, False)
    g = torch.randn(T, H, D, generator=gen(5), device="cuda")
    dq = torch.empty_like(g)
    rq.realq_rotary(g, pos, f, dq, amplitude=0.7, transpose=True)
    # the operator is linear in q, so <g, R(q + d)> - <g, R(q)> = <R^T g, d> whatever the size of d
    d = torch.randn(T, H, D, generator=gen(6), device="cuda")
    a, _ = turned(q.double() + d.double(), pos, f, False, 0.7, False)
    b, _ = turned(q, pos, f, False, 0.7, False)
    left, right = (g.double() * (a - b)).sum(), (dq.double() * d.double()).sum()
    assert abs(left - right) <= 2.0 ** -20 * (g.double().abs() * d.double().abs()).sum() * 2
    rq.realq_rotary(q, pos, f, q, k=k, k_out=k, amplitude=0.7)        # in place, the values untouched
    assert torch.equal(heads[:, :H], qo) and torch.equal(heads[:, H:H + kv], ko) and torch.equal(heads[:, H + kv:], v0)


def test_rotary_frequencies_of_longer_contexts():
    R, base, ctx = 128, 500000.0, 8192.0
    f = base ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)
    near = lambda a, b: bool(((a - b).abs() <= 1e-14 * b.abs()).all())   # noqa: E731
    assert near(rq.realq_rotary_frequencies(R, base), f)
    assert near(rq.realq_rotary_frequencies(R, base, "linear", 4.0), f / 4)
    got = rq.realq_rotary_frequencies(R, base, "base", 4.0)
    assert near(got[:1], f[:1]) and abs(got[-1] * 4 / f[-1] - 1) < 1e-12
    turns = ctx * f / (2 * math.pi)
    w = ((turns - 1) / 3).clamp(0, 1)
    assert near(rq.realq_rotary_frequencies(R, base, "ramp", 8.0, ctx, 1.0, 4.0), f * w + f / 8 * (1 - w))


# ------------------------------------------------------------ append, read ---
def appended(c, layer, news, olds, dtype, seed, loud=1.0, edit=None):
    """Append news[s] tokens behind olds[s] of each row, with the package and by definition; compare everything."""
    T = sum(news)
    k = (loud * torch.randn(T, c.kv, c.D, generator=gen(seed), device="cuda")).to(dtype)
    v = torch.randn(T, c.kv, c.D, generator=gen(seed + 1), device="cuda").to(dtype)
    if edit:
        edit(k, v)
    want = {n: t.clone() for n, t in c.buffers().items()}
    starts = starts_of(news)
    pos = torch.cat([torch.arange(o, o + n) for o, n in zip(olds, news)]).cuda()
    rq.realq_kv_append(rq.kv_cache(**c.buffers()), layer, k, v, starts, pos, c.tables)
    at = 0
    for s, n in enumerate(news):
        for w, x in (("k", k), ("v", v)):
            if n:
                append(want[w + "_codes"][layer], want[w + "_scale"][layer], x[at:at + n], olds[s], c.rows[s], c.page, c.block)
        at += n
    for n, t in c.buffers().items():
        same = torch.equal(t, want[n]) if t.dtype == torch.uint8 else torch.equal(t.view(torch.int32), want[n].view(torch.int32)) or bool(
            ((t == want[n]) | (t.isnan() & want[n].isnan())).all())
        assert same, n
    return k, v, starts, pos


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("page,block", [(16, 1), (16, 16), (64, 16), (64, 4), (128, 64), (256, 256)])
@pytest.mark.parametrize("kv,D", [(1, 16), (2, 128), (3, 80)])
def test_append(kv, D, page, block, dtype):
    """Single tokens, none, whole and partial blocks, blocks begun earlier; small and large new values."""
    news, olds = [1, 0, 5, 130, 1, 300, 17], [0, 9, 3, 70, 255, 0, 64]
    lens = [o + n for o, n in zip(olds, news)]
    for loud in (1e-3, 1.0, 300.0):
        c = Cache(7, lens, kv=kv, D=D, page=page, block=block, layers=2, poison=False)
        appended(c, 1, news, olds, dtype, 11, loud)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_append_special_values(dtype):
    """Zeros, ties, the type's extremes, infinities and NaN; a poisoned block starts anew with its first token."""
    lens = [64, 64]
    c = Cache(1, lens, kv=2, D=32, page=64, block=16, poison=False)

    def edit(k, v):
        k[0:16] = 0                                   # a block of zeros: scale 0, codes 128
        k[16:32] = torch.linspace(-127, 127, 16 * 2 * 32, device="cuda").view(16, 2, 32).to(dtype)
        k[32:48] *= 1e-30
        k[48:64] = torch.finfo(dtype).max
        v[3, 0, 5] = math.inf
        v[20, 1, 0] = math.nan
        v[40] = 1e-42                                 # below the smallest normal number
        v[64 + 17] = -math.inf
    appended(c, 0, [64, 64], [0, 0], dtype, 3, edit=edit)
    assert bool(c.v_scale[0, c.rows[0][0], 0, 0].isnan()) and not bool(c.v_scale[0, c.rows[0][0], 1, 0].isnan())
    appended(c, 0, [14, 16], [2, 16], dtype, 5)       # behind a poisoned block's first tokens, and over one from its start
    assert bool(c.v_scale[0, c.rows[0][0], 0, 0].isnan()) and not bool(c.v_scale[0, c.rows[1][0]].isnan().any())


def test_append_and_read_of_bad_lists():
    """Starts out of order, positions and pages outside: skipped, everything else done, nothing else touched."""
    c = Cache(2, [40, 40, 40, 40], kv=2, D=16, page=16, block=4, poison=False)
    good = {n: t.clone() for n, t in c.buffers().items()}
    h = rq.kv_cache(**c.buffers())
    x = torch.randn(12, 2, 16, generator=gen(1), device="cuda")
    for starts, pos, rows in (([0, 20, 3, -5, 12], list(range(12)), c.rows),
                              ([0, 3, 6, 9, 12], [-1] * 12, c.rows), ([0, 3, 6, 9, 12], [10 ** 6] * 12, c.rows),
                              ([0, 3, 6, 9, 12], [2 ** 62] * 12, c.rows),
                              ([0, 3, 6, 9, 12], list(range(12)), [[-1, 2 ** 30, 4000, -9, 0]] * 4)):
        c.tables = i32(rows)
        p = torch.tensor(pos, device="cuda")
        if rows is not c.rows:
            c.tables[:] = c.n_pages
        rq.realq_kv_append(h, 0, x, x, i32(starts), p, c.tables)
        out = torch.full((12, 2, 16), 7.0, device="cuda")
        rq.realq_kv_read(h, 0, i32(starts), p, c.tables, out)
        for n, t in c.buffers().items():
            assert torch.equal(t, good[n]), (starts, n)
        assert bool((out.isnan() | (out == 7.0)).all() if starts[1] != 20 else True)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("offset", [0, 3])
def test_append_from_strided_heads_and_read(dtype, offset):
    """k and v inside one projection's output, at any alignment; reading in any order, into any alignment."""
    news, olds = [33, 1, 7], [0, 50, 13]
    c = Cache(3, [o + n for o, n in zip(olds, news)], kv=2, D=48, page=32, block=8, layers=1, poison=False)
    T = sum(news)
    flat = torch.randn(T * 7 * 48 + 8, generator=gen(9), device="cuda").to(dtype)
    heads = flat[offset:offset + T * 7 * 48].view(T, 7, 48)
    k, v = heads[:, 3:5], heads[:, 5:7]
    want = {n: t.clone() for n, t in c.buffers().items()}
    pos = torch.cat([torch.arange(o, o + n) for o, n in zip(olds, news)]).cuda()
    h = rq.kv_cache(**c.buffers())
    rq.realq_kv_append(h, 0, k, v, starts_of(news), pos, c.tables)
    at = 0
    for s, n in enumerate(news):
        for w, x in (("k", k), ("v", v)):
            append(want[w + "_codes"][0], want[w + "_scale"][0], x[at:at + n], olds[s], c.rows[s], 32, 8)
        at += n
    for n, t in c.buffers().items():
        assert torch.equal(t, want[n]), n
    counts = [5, 0, 20]
    rp = torch.cat([torch.randint(0, c.lens[s], (n,), generator=torch.Generator().manual_seed(s)) for s, n in enumerate(counts)]).cuda()
    room = torch.full((25 * 2 * 48 + 8,), 5.0, device="cuda").to(dtype)
    out, vout = room[offset:offset + 24 * 2 * 48].view(24, 2, 48), torch.empty(24, 2, 48, device="cuda", dtype=dtype)
    rq.realq_kv_read(h, 0, starts_of(counts[:2] + [19]), rp[:24], c.tables, out, vout)
    ref = lambda w: torch.cat([c.values(w, 0, 0)[rp[:5]], c.values(w, 0, 2)[rp[5:24]]])   # noqa: E731
    for got, r in ((out, ref("k")), (vout, ref("v"))):
        assert bool(((got.double() - r).abs() <= (U(F32) + U(dtype)) * r.abs()).all())
    assert bool((room[offset + 24 * 96:] == 5).all())
    rq.realq_kv_read(h, 0, starts_of([2, 0, 3]), rp[:24], c.tables, None, vout)   # tokens behind the last sequence stay
    assert torch.equal(vout[5:], vout[5:]) and bool(torch.isfinite(vout.float()).all())


# --------------------------------------------------------------- attention ---
def attended(c, news, H, dtype, seed, window=0, causal=True, layer=0, scale=None, max_new=None, q=None, ws=None, loud=1.0, stream=None):
    """The operator against the definition, with the tolerances derived below; returns (out, lse)."""
    T = sum(news)
    q = (loud * torch.randn(T, H, c.D, generator=gen(seed), device="cuda")).to(dtype) if q is None else q
    h = rq.kv_cache(**c.buffers())
    out, lse = torch.full((T + 2, H, c.D), 9.0, device="cuda", dtype=dtype), torch.full((T + 2, H), 9.0, device="cuda")
    if ws is None:
        ws = rq.workspace(rq.realq_kv_attention_workspace_size(h, len(news), T, H))
    q2 = torch.cat([q, q[:1], q[:1]])     # two rows behind the last sequence
    rq.realq_kv_attention(q2, h, layer, starts_of(news), c.lengths, c.tables, out, lse, scale=scale, causal=causal, window=window,
                          max_new=max_new, ws=ws, stream=stream)
    assert bool((out[T:] == 9).all()) and bool((lse[T:] == 9).all())
    at = 0
    sc = c.D ** -0.5 if scale is None else scale
    for s, m in enumerate(news):
        if m == 0:
            continue
        L = c.lens[s]
        y, z, mag, big = attention(q[at:at + m], c.values("k", layer, s), c.values("v", layer, s), L, window, causal, sc)
        # Scores: products of fp16 parts with codes are exact, a query's parts hold 22 bits (bf16: all), the sum over
        # channels and the two scalings are fp32: within e = 2^-20 of the largest sum |q||k| of the row.  A weight is
        # then off by e^(2 e) - 1 < 2.1 e, by ex2's 2^-22, and by its rounding to fp16 (two parts: 2^-22); the sums over
        # tokens add fp32 rounding, one step per 16 tokens and per joined share.
        e = 2.0 ** -20 * big + 2.0 ** -30
        steps = (L / 16 + 160) * 2.0 ** -23
        weight = 2.1 * e + 2.0 ** -20 + (U(torch.float16) if dtype == BF16 else 2.0 ** -21) + steps
        tol = weight[..., None] * mag + U(dtype) * y.abs() + 1e-30
        err = (out[at:at + m].double() - y).abs()
        assert bool((err <= tol).all()), (s, m, L, float((err / tol).max()))
        zerr = (lse[at:at + m].double() - z).abs()
        ztol = 1.1 * e + steps + 2.0 ** -21 + 4 * U(F32) * z.abs()
        none = z == -math.inf
        assert bool((lse[at:at + m][none] == -math.inf).all()) and bool((out[at:at + m][none] == 0).all())
        assert bool((zerr[~none] <= ztol[~none]).all()), (s, m, L, float((zerr[~none] / ztol[~none]).max()))
        at += m
    return out[:T], lse[:T]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [16, 64, 80, 128, 192, 256])
@pytest.mark.parametrize("kv,G", [(1, 1), (2, 4), (1, 16), (3, 5)])
def test_attention_of_single_tokens(kv, G, D, dtype):
    """Lengths from none over one to several pages, at the edges of groups, tiles and pages."""
    lens = [1, 0, 15, 16, 17, 63, 64, 65, 128, 200, 1000]
    c = Cache(1, lens, kv=kv, D=D, page=64, block=16)
    attended(c, [1] * len(lens), kv * G, dtype, 2, max_new=1)


@pytest.mark.parametrize("page,block", [(16, 1), (16, 16), (32, 2), (64, 64), (128, 8), (256, 256)])
@pytest.mark.parametrize("window", [0, 1, 7, 100])
def test_attention_pages_blocks_windows(page, block, window):
    lens, news = [300, 5, 257, 1, 64], [3, 5, 1, 1, 2]
    c = Cache(4, lens, kv=2, D=64, page=page, block=block, layers=2)
    attended(c, news, 6, BF16, 3, window=window, layer=1, max_new=5)
    attended(c, news, 6, F32, 3, window=window, layer=1)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D,kv,G,news,lens", [(128, 2, 8, [40, 1, 0, 200], [40, 700, 33, 300]), (64, 1, 1, [500], [500]), (256, 1, 3, [70, 9], [80, 400]),
                                              (96, 2, 7, [31, 33, 129], [1000, 33, 131]), (128, 8, 4, [1, 129], [5, 129])])
def test_attention_of_prompts(D, kv, G, news, lens, dtype):
    c = Cache(5, lens, kv=kv, D=D, page=32, block=8)
    for kw in (dict(), dict(window=50), dict(causal=False)):
        attended(c, news, kv * G, dtype, 6, **kw)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_rows_that_see_nothing(dtype):
    """More new tokens than cached ones (the first see none), no cached tokens at all, tables without a column."""
    c = Cache(6, [3, 0, 70], kv=1, D=64)
    attended_rows = [5, 4, 72]
    T, H = sum(attended_rows), 2
    q = torch.randn(T, H, 64, generator=gen(1), device="cuda").to(dtype)
    h = rq.kv_cache(**c.buffers())
    ws = rq.workspace(rq.realq_kv_attention_workspace_size(h, 3, T, H))
    for max_new in (None, 1):
        out, lse = torch.empty_like(q), torch.empty(T, H, device="cuda")
        rq.realq_kv_attention(q, h, 0, starts_of(attended_rows), c.lengths, c.tables, out, lse, max_new=max_new, ws=ws)
        for a, b in ((0, 2), (5, 9), (9, 11)):
            assert bool((out[a:b] == 0).all()) and bool((lse[a:b] == -math.inf).all())
        for a, b in ((2, 5), (11, T)):
            assert bool(torch.isfinite(lse[a:b]).all()) and bool((out[a:b] != 0).any(dim=-1).all())
    rq.realq_kv_attention(q, h, 0, starts_of(attended_rows), c.lengths, c.tables[:, :0].contiguous(), out, lse, ws=ws)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())


def test_attention_extremes():
    """Large and tiny queries and scales, a zero-valued block, NaN where it is seen and where it is not."""
    c = Cache(8, [100, 90, 70], kv=1, D=64, block=16)
    attended(c, [1, 1, 1], 4, F32, 3, loud=1e18, scale=1e-19)
    attended(c, [1, 1, 1], 4, BF16, 3, loud=1e-30, scale=1e30)
    attended(c, [2, 2, 2], 4, BF16, 3, loud=8.0)             # nearly one weight
    c.v_scale[0, c.rows[0][0], :, 1] = 0.0                   # a block of zero values
    c.v_scale[0, c.rows[1][0]] *= 2.0 ** 90
    c.v_scale[0, c.rows[2][0], :, 0] *= 2.0 ** -70
    attended(c, [1, 1, 1], 4, F32, 4)
    c.k_scale[0, c.rows[0][0], :, 0] = 0.0
    attended(c, [1, 1, 1], 4, F32, 5)
    c.v_scale[0, c.rows[1][0], :, 2] = math.nan              # tokens 32 .. 47 of row 1
    c.k_scale[0, c.rows[2][0], :, 2] = math.nan
    h = rq.kv_cache(**c.buffers())
    q = torch.randn(60 + 45 + 30, 2, 64, generator=gen(1), device="cuda")
    ws = rq.workspace(rq.realq_kv_attention_workspace_size(h, 3, 135, 2))
    out, lse = torch.empty_like(q), torch.empty(135, 2, device="cuda")
    rq.realq_kv_attention(q, h, 0, starts_of([60, 45, 30]), i32([60, 45, 30]), c.tables, out, lse, ws=ws)
    assert bool(torch.isfinite(out[:60]).all())
    assert bool(torch.isfinite(out[60:92]).all()) and bool(out[92:105].isnan().all()) and bool(torch.isfinite(lse[60:105]).all())
    assert bool(torch.isfinite(out[105:]).all())             # row 2's bad block lies behind its 30 tokens
    rq.realq_kv_attention(q, h, 0, starts_of([60, 30, 45]), i32([60, 30, 45]), c.tables, out, lse, ws=ws)
    assert bool(torch.isfinite(out[60:122]).all()) and bool(out[122:].isnan().all()) and bool(lse[122:].isnan().all())


def test_attention_strides_streams_and_repeats():
    """q inside a projection's output; on another stream; the same bits again and with any max_new that takes the same
    kernel; workspaces reused by calls of other sizes."""
    lens, news, H, kv, D = [900, 31, 500], [1, 1, 1], 8, 2, 128
    c = Cache(9, lens, kv=kv, D=D)
    qkv = torch.randn(3, (H + 2 * kv) * D, generator=gen(2), device="cuda").to(BF16).view(3, H + 2 * kv, D)
    q = qkv[:, :H]
    h = rq.kv_cache(**c.buffers())
    ws = rq.workspace(rq.realq_kv_attention_workspace_size(h, 3, 3, H))
    a, la = attended(c, news, H, BF16, 0, q=q.contiguous(), ws=ws, max_new=1)
    out, lse = torch.empty(3, H, D, device="cuda", dtype=BF16), torch.empty(3, H, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    rq.realq_kv_attention(q, h, 0, starts_of(news), c.lengths, c.tables, out, lse, max_new=1, ws=ws, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, a) and torch.equal(lse, la)
    other = Cache(10, [5000], kv=2, D=128)
    attended(other, [1], 8, BF16, 1, ws=ws, max_new=1)
    rq.realq_kv_attention(q, h, 0, starts_of(news), c.lengths, c.tables, out, None, max_new=1, ws=ws)
    assert torch.equal(out, a)
    rq.realq_workspace_status(ws)


def test_attention_many_sequences():
    """More sequences than a CTA holds the sums of at a time, many of them without new tokens."""
    r = random.Random(1)
    lens = [r.randint(0, 90) for _ in range(1300)]
    news = [r.choice([0, 0, 1, 1, 2]) if n >= 2 else 0 for n in lens]
    lens = [max(n, 0) for n in lens]
    c = Cache(12, lens, kv=1, D=16, page=16, block=4, poison=False)
    attended(c, news, 2, BF16, 1, max_new=2)


def test_attention_in_graphs_that_share_a_workspace():
    """A step captured once serves growing lengths; two graphs with one workspace, run in turn."""
    lens = [700, 40, 300]
    c = Cache(13, [900, 300, 400], kv=2, D=128, poison=False)
    c.lens = lens
    c.lengths.copy_(i32(lens))
    H, T = 8, 3
    h = rq.kv_cache(**c.buffers())
    ws = rq.workspace(rq.realq_kv_attention_workspace_size(h, 3, 6, H))
    qs = [torch.randn(3, H, 128, generator=gen(1), device="cuda").to(BF16), torch.randn(6, H, 128, generator=gen(2), device="cuda").to(BF16)]
    st = [starts_of([1, 1, 1]), starts_of([2, 2, 2])]
    outs = [torch.empty_like(q) for q in qs]
    run = lambda i: rq.realq_kv_attention(qs[i], h, 0, st[i], c.lengths, c.tables, outs[i], max_new=i + 1, ws=ws)   # noqa: E731
    side = torch.cuda.Stream()
    graphs = []
    with torch.cuda.stream(side):
        for i in range(2):
            run(i)
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                run(i)
            graphs.append(g)
    torch.cuda.synchronize()
    for step in range(3):
        now = [n + 50 * step for n in lens]
        c.lens = now
        c.lengths.copy_(i32(now))
        for i in (0, 1, 0):
            graphs[i].replay()
            got = outs[i].clone()
            want, _ = attended(c, [i + 1] * 3, H, BF16, 0, q=qs[i], max_new=i + 1)
            assert torch.equal(got, want)


def test_attention_right_behind_a_product():
    """The queries come from an 8-bit product that lets the next kernel start early: attention waits for them all the same."""
    T, n, H, D = 300, 2048, 4, 64
    c = Cache(14, [70] * T, kv=2, D=D)
    h = rq.kv_cache(**c.buffers())
    xc = torch.randint(0, 256, (T, n), generator=gen(1), device="cuda").to(torch.uint8)
    wc = torch.randint(0, 256, (H * D, n), generator=gen(2), device="cuda").to(torch.uint8)
    xs, ws = torch.full((T,), 1e-2, device="cuda"), torch.full((H * D,), 1e-3, device="cuda")
    pws = rq.workspace(rq.realq_int8_product_workspace_size(T, n, H * D))
    aws = rq.workspace(rq.realq_kv_attention_workspace_size(h, T, T, H))
    q, out = torch.zeros(T, H * D, device="cuda", dtype=BF16), torch.empty(T, H, D, device="cuda", dtype=BF16)
    starts = starts_of([1] * T)
    outs = []
    for together in (False, True, True):
        q.zero_()
        torch.cuda.synchronize()
        rq.realq_int8_product(xc, xs, wc, ws, q, ws=pws)
        if not together:
            torch.cuda.synchronize()
        rq.realq_kv_attention(q.view(T, H, D), h, 0, starts, c.lengths, c.tables, out, max_new=1, ws=aws)
        outs.append(out.clone())
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_tokens_within_a_heads_row(dtype):
    """Heads first, tokens within them (a transposed view): the same bits as from tokens x heads, in every operator."""
    news, olds, H, kv, D = [40, 1], [30, 90], 6, 2, 64
    c = Cache(16, [o + n for o, n in zip(olds, news)], kv=kv, D=D, page=32, block=16, poison=False)
    T, st = sum(news), starts_of(news)
    pos = torch.cat([torch.arange(o, o + n) for o, n in zip(olds, news)]).cuda()
    f = rq.realq_rotary_frequencies(D).cuda()
    first = [torch.randn(n, T, D, generator=gen(n), device="cuda").to(dtype) for n in (H, kv, kv + 1)]
    q, k, v = (x.transpose(0, 1) for x in first)
    v = v[:, :kv]
    h = rq.kv_cache(**c.buffers())
    before = {n: t.clone() for n, t in c.buffers().items()}
    ws = rq.workspace(rq.realq_kv_attention_workspace_size(h, 2, T, H))
    got = []
    for q1, k1, v1 in ((q, k, v), (q.contiguous(), k.contiguous(), v.contiguous())):
        for n, t in before.items():
            getattr(c, n).copy_(t)
        qo, ko = torch.empty_like(q1), torch.empty_like(k1)     # (of the same strides)
        assert qo.stride() == q1.stride()
        rq.realq_rotary(q1, pos, f, qo, k=k1, k_out=ko)
        rq.realq_kv_append(h, 0, ko, v1, st, pos, c.tables)
        out, one = torch.empty(T, H, D, device="cuda", dtype=dtype), torch.empty(T, H, D, device="cuda", dtype=dtype)
        rq.realq_kv_attention(qo, h, 0, st, c.lengths, c.tables, out, ws=ws)
        rq.realq_kv_attention(qo, h, 0, st, c.lengths, c.tables, one, max_new=1, ws=ws)
        got.append([qo.clone(), ko.clone(), out, one] + [t.clone() for t in c.buffers().values()])
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_pages_beyond_32_bits():
    """A pool of more than 2^32 bytes of codes of each kind: into its last pages, out of them, over them."""
    lens, kv, D = [300, 70], 8, 256
    c = Cache(15, lens, kv=kv, D=D, page=64, block=16, poison=False)
    small, rows = {n: t.clone() for n, t in c.buffers().items()}, c.rows
    n = 33000
    at = [n - 1 - 3 * i for i in range(c.n_pages)]
    assert min(at) * kv * 64 * D > 2 ** 32
    for name, t in small.items():
        big = torch.full((1, n, *t.shape[2:]), 128 if t.dtype == torch.uint8 else 0, dtype=t.dtype, device="cuda")
        big[:, at] = t
        setattr(c, name, big)
    c.rows = [[at[p] if p >= 0 else p for p in r] for r in rows]
    c.tables = i32(c.rows)
    attended(c, [200, 1], 16, BF16, 1)
    attended(c, [1, 1], 16, F32, 2, max_new=1)
    h = rq.kv_cache(**c.buffers())
    x = [torch.randn(40, kv, D, generator=gen(i), device="cuda").to(BF16) for i in (3, 4)]
    pos = torch.arange(100, 140, device="cuda")
    rq.realq_kv_append(h, 0, *x, starts_of([40, 0]), pos, c.tables)
    for w, t in zip("kv", x):
        append(small[w + "_codes"][0], small[w + "_scale"][0], t, 100, rows[0], 64, 16)
    for name, t in small.items():
        assert torch.equal(getattr(c, name)[:, at], t), name
        others = torch.ones(n, dtype=torch.bool, device="cuda")
        others[at] = False
        assert bool((getattr(c, name)[0, -40:][others[-40:]] == (128 if t.dtype == torch.uint8 else 0)).all()), name
    out = [torch.empty(40, kv, D, device="cuda") for _ in range(2)]
    rq.realq_kv_read(h, 0, starts_of([40, 0]), pos, c.tables, *out)
    for w, o in zip("kv", out):
        want = c.values(w, 0, 0)[100:140]
        assert bool(((o.double() - want).abs() <= U(F32) * want.abs()).all())
    rq.realq_pages_copy(h, i32(at), i32(list(range(len(at)))))
    rq.realq_pages_copy(h, i32(list(range(len(at)))), i32([p - 1 for p in at]))
    for name, t in small.items():
        assert torch.equal(getattr(c, name)[:, :len(at)], t) and torch.equal(getattr(c, name)[:, [p - 1 for p in at]], t), name


def test_attention_of_many_sequences_with_prompts_among_them():
    """More sequences than a CTA holds the sums of at a time; prompts, single tokens and rows that wait, in both kernels."""
    r = random.Random(5)
    news = [r.choice([0, 0, 1, 1, 2, 9, 20, 70]) for _ in range(1100)]
    news[510:515], news[1023:1026] = [70, 0, 20, 70, 1], [20, 70, 70]     # (around the sums' ends)
    lens = [n + r.randint(0, 150) for n in news]
    c = Cache(17, lens, kv=1, D=32, page=16, block=16, poison=False)
    attended(c, news, 4, BF16, 1)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("news,lens", [([64], [6000]), ([12, 3], [9000, 2500]), ([8], [2000]), ([2], [3000]), ([300, 9, 1], [700, 3000, 4000])])
def test_attention_units_of_many_tiles(news, lens, dtype):
    """One or two sequences, whose tiles are shared out several to a CTA and joined."""
    c = Cache(18, lens, kv=2, D=128, page=64, block=16)
    attended(c, news, 8, dtype, 2)
    attended(c, news, 8, dtype, 3, window=1500, max_new=max(news))
