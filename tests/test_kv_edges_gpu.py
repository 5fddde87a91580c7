"""The 8-bit key/value cache's operators at the edges of what their arguments allow,
against the definitions in 64 bits."""
import math

import pytest
import torch

import paper_2609_00049_gb300 as rq
from kv_reference import Cache, attention, gen, i32, starts_of

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def U(t):
    return torch.finfo(t).eps / 2


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2609_00049_gb300 import build as b
    b.build()
    rq.lib()


def run(q, h, starts, lengths, tables, max_new=None, **kw):
    """Attention into buffers that hold 9 before: outputs and log sums."""
    T, H = q.shape[:2]
    out, lse = torch.full_like(q, 9.0), torch.full((T, H), 9.0, device="cuda")
    ws = rq.workspace(rq.realq_kv_attention_workspace_size(h, len(lengths), T, H))
    rq.realq_kv_attention(q, h, 0, starts, lengths, tables, out, lse, max_new=max_new, ws=ws, **kw)
    rq.realq_workspace_status(ws)
    return out, lse


def one_page(values, D, kv=1, page=256, block=256):
    """A cache of the given pages: each (k code, k scale, v code, v scale), the same for all tokens and heads."""
    n = len(values)
    buf = [torch.empty(1, n, kv, page, D, dtype=torch.uint8, device="cuda") for _ in range(2)]
    sc = [torch.empty(1, n, kv, page // block, device="cuda") for _ in range(2)]
    for i, (kc, ks, vc, vs) in enumerate(values):
        buf[0][:, i], sc[0][:, i], buf[1][:, i], sc[1][:, i] = kc, ks, vc, vs
    return rq.kv_cache(buf[0], buf[1], sc[0], sc[1])


# ------------------------------------------- long contexts of zero values ---
# Scale 0 and codes 128 are what appending zeros leaves.  The tables name one page again and again.
# The softmax's sum of n equal weights: fp32 additions, one for every 16 tokens of a share and every joined share.
def sum_error(n):
    return (n / 16 + 160) * 2.0 ** -23


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("m,n", [(1, 20000), (1, 3000000), (40, 20000), (40, 5000000)])
def test_log_sums_over_zero_values(m, n, dtype):
    """All scores equal, all values zero: the log of the number of tokens seen, and zeros."""
    h = one_page([(128, 1.0, 128, 0.0)], 16)
    table = torch.zeros(1, -(-n // 256), dtype=torch.int32, device="cuda")
    q = torch.randn(m, 2, 16, generator=gen(1), device="cuda").to(dtype)
    out, lse = run(q, h, starts_of([m]), i32([n]), table)
    want = torch.log(torch.arange(n - m + 1, n + 1, dtype=torch.float64, device="cuda"))[:, None]
    assert bool((out == 0).all())
    assert bool(((lse.double() - want).abs() <= sum_error(n) + 2.0 ** -21 + 4 * U(F32) * want).all()), float(lse.max())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("m", [1, 40])
def test_log_sums_where_the_maximum_lags(m, dtype):
    """A first page whose scores are a little below the others', so that a running maximum that moves rarely stays behind
    by as much; a head to a CTA, so that whole contexts are summed by one."""
    kv, n, low = 160, 40000, 5.4                         # (5.4 < 8 ln 2)
    ks = torch.tensor(low / 16, dtype=F32).item()
    h = one_page([(128, 1.0, 128, 0.0), (127, ks, 128, 0.0)], 16, kv)
    table = torch.zeros(1, -(-n // 256), dtype=torch.int32, device="cuda")
    table[0, 0] = 1
    q = torch.ones(m, kv, 16, device="cuda", dtype=dtype)
    out, lse = run(q, h, starts_of([m]), i32([n]), table, scale=1.0)
    seen = torch.arange(n - m + 1, n + 1, dtype=torch.float64, device="cuda")[:, None]
    want = torch.log(256 * math.exp(-16 * ks) + seen - 256)
    assert bool((out == 0).all())
    # (scores within 2^-20 of themselves)
    assert bool(((lse.double() - want).abs() <= sum_error(n) + 2.0 ** -19 * low + 2.0 ** -21 + 4 * U(F32) * want).all()), float(lse.max())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("m", [1, 12])
def test_zero_values_before_others(m, dtype):
    """Many sequences whose values are zero but for the last page's: whole shares see nothing but zeros, and the output
    is the last page's all the same."""
    S, kv, G, n = 64, 8, 4, 256 * 157
    h = one_page([(128, 1.0, 128, 0.0), (128, 1.0, 128, 1.0)], 16, kv)
    kc, vc = (torch.randint(1, 256, (kv, 256, 16), generator=gen(i), device="cuda").to(torch.uint8) for i in (1, 2))
    h.tensors[0][0, 1], h.tensors[1][0, 1] = kc, vc
    h.tensors[2][0, 1] = 0.01
    table = torch.zeros(S, n // 256, dtype=torch.int32, device="cuda")
    table[:, -1] = 1
    T = S * m
    q = torch.randn(T, kv * G, 16, generator=gen(3), device="cuda").to(dtype)
    out, lse = run(q, h, starts_of([m] * S), i32([n] * S), table, max_new=m)
    # the definition: n - 256 tokens of score 0 and value 0, then the last page
    K, V = (kc.double() - 128).transpose(0, 1) * torch.tensor(0.01, dtype=F32).double().item(), (vc.double() - 128).transpose(0, 1)
    x = torch.einsum("smkgd,lkd->smkgl", q.double().view(S, m, kv, G, 16), K) * 0.25
    later = torch.arange(256, device="cuda") > (256 - m + torch.arange(m, device="cuda"))[:, None]
    w = torch.exp(x.masked_fill(later[None, :, None, None], -math.inf))
    total = n - 256 + w.sum(-1)
    y = torch.einsum("smkgl,lkd->smkgd", w, V) / total[..., None]
    mag = torch.einsum("smkgl,lkd->smkgd", w, V.abs()) / total[..., None]
    big = (q.double().abs().view(S, m, kv, G, 16).sum(-1) * 1.27 * 0.25).reshape(T, kv * G)
    y, mag, z = y.reshape(out.shape), mag.reshape(out.shape), torch.log(total).reshape(lse.shape)
    # as in the attention tests: scores within e, weights by 2.1 e, ex2 and their rounding, sums by additions
    e = 2.0 ** -20 * big + 2.0 ** -30
    weight = 2.1 * e + 2.0 ** -20 + (U(torch.float16) if dtype == BF16 else 2.0 ** -21) + sum_error(n)
    tol = weight[..., None] * mag + U(dtype) * y.abs() + 1e-30
    assert bool(((out.double() - y).abs() <= tol).all()), float(((out.double() - y).abs() / tol).max())
    assert bool(((lse.double() - z).abs() <= 1.1 * e + sum_error(n) + 2.0 ** -21 + 4 * U(F32) * z).all()), float(lse.max())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("m", [1, 40])
@pytest.mark.parametrize("n,block", [(300, 16), (300, 4), (3000, 16)])
@pytest.mark.parametrize("power", [110, 60, 20, -60])
def test_values_of_any_size(power, n, block, m, dtype):
    """Outputs of very large and very small values, with zero and far smaller ones among them: their tokens' weights count
    all the same, within a tile, over tiles and over shares."""
    c = Cache(30, [n], kv=1, D=32, page=16, block=block, poison=False)
    c.v_scale *= 2.0 ** power
    c.v_scale[0, c.rows[0][3]] = 0.0
    c.v_scale[0, c.rows[0][5:7]] *= 2.0 ** (-80 if power > 0 else -10)
    if n > 2000:
        c.v_scale[0, c.rows[0][40:130]] = 0.0
    q = torch.randn(m, 4, 32, generator=gen(4), device="cuda").to(dtype)
    out, lse = run(q, rq.kv_cache(**c.buffers()), starts_of([m]), c.lengths, c.tables)
    y, z, mag, big = attention(q, c.values("k", 0, 0), c.values("v", 0, 0), n, 0, True, 32 ** -0.5)
    e = 2.0 ** -20 * big + 2.0 ** -30
    weight = 2.1 * e + 2.0 ** -20 + (U(torch.float16) if dtype == BF16 else 2.0 ** -21) + sum_error(n)
    # (a zero value counts as 127 x 2^-88 at most in the kernel of many rows)
    tol = weight[..., None] * mag + U(dtype) * y.abs() + 2.0 ** -81
    assert bool(((out.double() - y).abs() <= tol).all()), float(((out.double() - y).abs() / tol).max())
    assert bool(((lse.double() - z).abs() <= 1.1 * e + sum_error(n) + 2.0 ** -21 + 4 * U(F32) * z.abs()).all())


# ------------------------------------------------------- lists with faults ---
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_reading_beside_a_sequence_that_ends_outside(dtype):
    """A sequence that ends behind the call's tokens takes no part; those before it are read, and nothing else is written."""
    c = Cache(31, [40, 40, 40], kv=2, D=32, page=16, block=4, poison=False)
    h, pos = rq.kv_cache(**c.buffers()), torch.arange(12, device="cuda")
    for starts, good in (([0, 3, 20, 20], 3), ([0, 3, 7, 13], 7), ([0, 12, 12, 12], 12), ([0, 4, 4, 9], 9), ([0, 0, 0, 13], 0), ([0, 2, 5, 5], 5)):
        got = [torch.full((12, 2, 32), 7.0, device="cuda", dtype=dtype) for _ in range(2)]
        rq.realq_kv_read(h, 0, i32(starts), pos, c.tables, *got)
        for w, t in zip("kv", got):
            assert bool((t[good:] == 7).all()), starts
            for s in range(3):
                a, b = starts[s], min(starts[s + 1], good)
                if a < b:
                    want = c.values(w, 0, s)[a:b]
                    assert bool(((t[a:b].double() - want).abs() <= (U(F32) + U(dtype)) * want.abs()).all()), starts


def expected(q, K, V, there, L, window, causal, scale):
    """Attention of a sequence of L tokens of which the first len(there) can be in the table and those that `there` names
    are; as kv_reference.attention."""
    m, H, D = q.shape
    kv, n = K.shape[1], len(there)
    q = q.double().view(m, kv, H // kv, D)
    at, key = torch.arange(L - m, L, device="cuda")[:, None], torch.arange(n, device="cuda")
    seen = there.expand(m, n) & ((key <= at) if causal else (key < L))
    if window:
        seen = seen & (key > at - window)
    s = (torch.einsum("mkgd,lkd->mkgl", q, K) * scale).masked_fill(~seen[:, None, None], -math.inf)
    if n == 0:
        zero = torch.zeros(m, H, D, dtype=torch.float64, device="cuda")
        return zero, zero[..., 0] - math.inf, zero, zero[..., 0]
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - lse[..., None]).nan_to_num(0.0)
    y, mag = torch.einsum("mkgl,lkd->mkgd", p, V), torch.einsum("mkgl,lkd->mkgd", p, V.abs())
    big = torch.einsum("mkgd,lkd->mkgl", q.abs(), K.abs()).amax(-1) * scale
    return y.reshape(m, H, D), lse.reshape(m, H), mag.reshape(m, H, D), big.reshape(m, H)


def close(out, lse, y, z, mag, big, L):
    """The attention tests' tolerances."""
    dtype = out.dtype
    e, steps = 2.0 ** -20 * big + 2.0 ** -30, (L / 16 + 160) * 2.0 ** -23
    weight = 2.1 * e + 2.0 ** -20 + (U(torch.float16) if dtype == BF16 else 2.0 ** -21) + steps
    none = z == -math.inf
    assert bool((lse[none] == -math.inf).all()) and bool((out[none] == 0).all())
    err, tol = (out.double() - y).abs(), weight[..., None] * mag + U(dtype) * y.abs() + 1e-30
    assert bool((err <= tol).all()), float((err / tol).max())
    err, tol = (lse.double() - z).abs()[~none], (1.1 * e + steps + 2.0 ** -21 + 4 * U(F32) * z.abs())[~none]
    assert bool((err <= tol).all()), float((err / tol).max())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kw", [dict(), dict(window=70), dict(causal=False)])
@pytest.mark.parametrize("news", [[1, 2, 5], [40, 70, 90]])
def test_attention_of_sequences_beyond_their_table(news, kw, dtype):
    """lengths that the table's row has no entries for: the queries keep their positions, the tokens behind take no part."""
    lens, width = [100, 200, 128], 128
    c = Cache(32, [width] * 3, kv=2, D=64, page=16, block=8, extra_entries=0, poison=False)
    T, H = sum(news), 8
    q = torch.randn(T, H, 64, generator=gen(5), device="cuda").to(dtype)
    out, lse = run(q, rq.kv_cache(**c.buffers()), starts_of(news), i32(lens), c.tables, max_new=max(news), **kw)
    at = 0
    for s, m in enumerate(news):
        n = min(lens[s], width)
        want = expected(q[at:at + m], c.values("k", 0, s, n), c.values("v", 0, s, n), torch.ones(n, dtype=torch.bool, device="cuda"), lens[s],
                        kw.get("window", 0), kw.get("causal", True), 64 ** -0.5)
        close(out[at:at + m], lse[at:at + m], *want, n)
        at += m


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("m", [1, 3, 40])
@pytest.mark.parametrize("back", [0, 1, 17, 300])
def test_attention_of_the_last_tokens_that_lengths_can_name(m, back, dtype):
    """A sequence of 2^31 - 1 tokens (less `back`), whose table names a few pages again and again."""
    L, page, near, window = 2 ** 31 - 1 - back, 256, 1024, 200
    c = Cache(33, [7 * page], kv=1, D=16, page=page, block=16, spare=0, extra_entries=0, poison=False)
    table = (torch.arange(2 ** 31 // page, device="cuda") % 7).to(torch.int32)[None]
    q = torch.randn(m, 2, 16, generator=gen(6), device="cuda").to(dtype)
    out, lse = run(q, rq.kv_cache(**c.buffers()), starts_of([m]), i32([L]), table, window=window)
    at = torch.arange(L - near, L, device="cuda")
    pg, slot = table[0].long()[at // page], at % page
    K, V = ((codes[0, pg, :, slot].double() - 128) * scale[0, pg, :, slot // 16].double()[..., None]
            for codes, scale in ((c.k_codes, c.k_scale), (c.v_codes, c.v_scale)))
    close(out, lse, *attention(q, K, V, near, window, True, 0.25), near)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("block", [16, 4])
@pytest.mark.parametrize("m", [1, 150])
def test_a_nan_among_values_of_no_weight(m, block, dtype):
    """Tokens whose weight is too small for any number of fp32, with values that are NaN: the rows that see them are NaN,
    the log sums are not, whichever tile the rows' last tokens lie in; a window that passes them by leaves numbers."""
    n = 150
    c = Cache(34, [n], kv=1, D=64, page=16, block=block, poison=False)
    first = c.rows[0][0]
    c.k_codes[0, first], c.k_scale[0, first] = 1, 1.0           # -127 in every channel: a score of -8128 for a q of ones
    c.v_scale[0, first] = math.nan
    q = torch.ones(m, 2, 64, device="cuda", dtype=dtype)
    h = rq.kv_cache(**c.buffers())
    out, lse = run(q, h, starts_of([m]), c.lengths, c.tables, scale=1.0)
    p = torch.arange(n - m, n, device="cuda")
    assert bool(out.isnan().all()) and bool(torch.isfinite(lse).all())
    out, lse = run(q, h, starts_of([m]), c.lengths, c.tables, scale=1.0, window=20)
    assert bool(out[p < 35].isnan().all()) and bool(torch.isfinite(out[p >= 35]).all()) and bool(torch.isfinite(lse).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("starts,lens", [([45, 90, 0, 45], [90, 77, 60]),               # the second is out of order
                                         ([0, 45, 200, 200], [90, 77, 60]), ([-3, 45, 90, 90], [90, 95, 60]),
                                         ([0, 45, 46, 90], [90, -5, 0]), ([0, 3, 5, 6], [90, -2 ** 31, 1])])
def test_attention_with_faulty_lists(starts, lens, dtype):
    """Sequences whose starts are not in order or lie outside take no part: their rows stay as they were, the others' are
    right.  A length below zero is none: such rows see nothing."""
    c = Cache(35, [96] * 3, kv=2, D=64, page=16, block=16, poison=False)
    T = 90
    q = torch.randn(T, 4, 64, generator=gen(7), device="cuda").to(dtype)
    out, lse = run(q, rq.kv_cache(**c.buffers()), i32(starts), i32(lens), c.tables)
    touched = torch.zeros(T, dtype=torch.bool, device="cuda")
    for s in range(3):
        a, b, L = starts[s], starts[s + 1], max(0, lens[s])
        if not 0 <= a < b <= T:
            continue
        touched[a:b] = True
        want = expected(q[a:b], c.values("k", 0, s, L), c.values("v", 0, s, L), torch.ones(L, dtype=torch.bool, device="cuda"), L, 0, True, 0.125)
        close(out[a:b], lse[a:b], *want, 96)
    assert bool((out[~touched] == 9).all()) and bool((lse[~touched] == 9).all()) and bool(touched.any())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("block", [16, 2])
@pytest.mark.parametrize("news", [[1, 2], [60, 90]])
def test_attention_over_missing_pages(news, block, dtype):
    """Pages outside the pool inside a sequence: their tokens take no part."""
    lens = [300, 170]
    c = Cache(36, lens, kv=2, D=64, page=16, block=block, poison=False)
    gone = [[0, 3, 4, 11, 18], [9, 10]]
    for s, bad in enumerate([[-1, 10 ** 6, c.n_pages, -2 ** 31, 2 ** 31 - 1], [-7, c.n_pages + 1]]):
        c.tables[s, gone[s]] = i32(bad)
    q = torch.randn(sum(news), 4, 64, generator=gen(8), device="cuda").to(dtype)
    out, lse = run(q, rq.kv_cache(**c.buffers()), starts_of(news), c.lengths, c.tables, max_new=max(news))
    at = 0
    for s, (m, L) in enumerate(zip(news, lens)):
        there = ~torch.isin(torch.arange(L, device="cuda") // 16, torch.tensor(gone[s], device="cuda"))
        rows = torch.tensor(c.rows[s], device="cuda")[torch.arange(L, device="cuda") // 16]
        slot = torch.arange(L, device="cuda") % 16
        K, V = ((codes[0, rows, :, slot].double() - 128) * scale[0, rows, :, slot // block].double()[..., None]
                for codes, scale in ((c.k_codes, c.k_scale), (c.v_codes, c.v_scale)))
        close(out[at:at + m], lse[at:at + m], *expected(q[at:at + m], K, V, there, L, 0, True, 0.125), L)
        at += m


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("news", [[5, 9], [60, 90]])
def test_attention_of_the_largest_window(news, dtype):
    """A window that no sequence reaches is none, for queries without cached tokens as well."""
    c = Cache(37, [3, 70], kv=1, D=64, page=16, block=16, poison=False)
    q = torch.randn(sum(news), 2, 64, generator=gen(9), device="cuda").to(dtype)
    h = rq.kv_cache(**c.buffers())
    want = run(q, h, starts_of(news), c.lengths, c.tables, max_new=max(news))
    for window in (1000, 2 ** 31, 2 ** 40, 2 ** 63 - 1):
        got = run(q, h, starts_of(news), c.lengths, c.tables, max_new=max(news), window=window)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), window


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("m", [1, 40])
def test_attention_of_subnormal_queries(m, dtype):
    """Rows whose largest value is below the smallest normal number, under a scale that makes scores of them; a row of zeros."""
    c = Cache(38, [200], kv=2, D=64, page=16, block=16, poison=False)
    q = torch.randn(m, 4, 64, generator=gen(10), device="cuda").clamp(-4, 4) * 2e-39
    q[0, 1] = 0.0
    q = q.to(dtype)
    assert 0.0 < float(q.double().abs().max()) < 2.0 ** -126
    out, lse = run(q, rq.kv_cache(**c.buffers()), starts_of([m]), c.lengths, c.tables, scale=5e37)
    sc = torch.tensor(5e37, dtype=F32).double().item()
    # (values of the scaled rows are held to 2^-25 with a largest of 2^-2 and more: within the tolerance's 2^-20)
    close(out, lse, *attention(q, c.values("k", 0, 0), c.values("v", 0, 0), 200, 0, True, sc), 200)
