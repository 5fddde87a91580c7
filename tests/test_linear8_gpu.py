"""The 8-bit linear operators and the token log probabilities on the GPU
against their definitions in 64 bits.  Bounds: U = 2^-24 and
BF = 2^-8 are the unit roundoffs of fp32 (24 significant bits) and bf16 (8)."""
import math

import pytest
import torch

import paper_2609_00049_gb300 as rq

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
BF = 2.0 ** -8
INF = math.inf


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2609_00049_gb300 import build as b
    b.build()
    rq.lib()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def shifted(t, by):
    """A contiguous copy of t whose address is `by` elements off the allocation's."""
    flat = torch.empty(t.numel() + by, dtype=t.dtype, device="cuda")[by:]
    return flat.copy_(t.reshape(-1)).view(t.shape)


# -------------------------------------------------------------- product ---
def product_case(T, n, m, w_bits, zeros, seed=0, extreme=False):
    g = gen(seed)
    hi = 256
    xc = torch.randint(0, hi, (T, n), generator=g, device="cuda").to(torch.uint8)
    wc = torch.randint(0, 256, (m, n if w_bits == 8 else (n + 1) // 2), generator=g, device="cuda").to(torch.uint8)
    if extreme:   # every product at its largest, all of one sign
        xc.zero_()
        wc.zero_()
    xs = torch.rand(T, generator=g, device="cuda") * 0.1 + 1e-3
    ws = torch.rand(m, generator=g, device="cuda") * 0.01 + 1e-4
    wz = torch.randint(0, 256 if w_bits == 8 else 16, (m,), generator=g, device="cuda").to(torch.uint8) if zeros else None
    return xc, xs, wc, ws, wz


def product_exact(xc, xs, wc, ws, wz, w_bits):
    n = xc.shape[1]
    if w_bits == 4:
        w = torch.stack([wc & 15, wc >> 4], dim=2).reshape(wc.shape[0], -1)[:, :n].double()
    else:
        w = wc.double()
    z = wz.double()[:, None] if wz is not None else float(2 ** (w_bits - 1))
    N = (xc.double() - 128) @ (w - z).T
    return N, N * xs.double()[:, None] * ws.double()


def run_product(xc, xs, wc, ws, wz, w_bits, dtype, ws_buf=None, stream=None):
    T, n = xc.shape
    m = wc.shape[0]
    Y = torch.full((T, m), math.nan, dtype=dtype, device="cuda")
    buf = rq.workspace(rq.realq_int8_product_workspace_size(T, n, m, w_bits)) if ws_buf is None else ws_buf
    rq.realq_int8_product(xc, xs, wc, ws, Y, w_bits=w_bits, w_zero=wz, ws=buf, stream=stream)
    if buf is not None and stream is None:
        rq.realq_workspace_status(buf)
    return Y


def product_bound(N, ref, n, dtype):
    """Two roundings for the scales and one of the sum's conversion; sums past
    2^24 lose at most 2u of the largest partial sum at each of n/16 additions."""
    past = (N.abs().amax() > 2 ** 23).item()
    rel = 3 * U + (2 * U * (n / 16 + 2) if past else 0.0) + (BF if dtype == torch.bfloat16 else 0.0)
    return ref.abs() * rel * 1.01 + 1e-30


SHAPES = [(1, 1, 1), (1, 7, 5), (1, 1024, 2048), (1, 1000, 33), (1, 4099, 130), (2, 16, 3), (2, 31, 9), (3, 64, 64),
          (4, 515, 257), (5, 96, 40), (7, 2048, 515), (8, 4096, 300), (8, 129, 1001), (9, 64, 128), (13, 200, 77),
          (16, 1024, 256), (17, 1007, 129), (33, 640, 384), (64, 2048, 512), (65, 48, 1000), (100, 8192, 128),
          (128, 65, 65), (129, 1024, 1024), (200, 320, 2000), (257, 1111, 259), (300, 4096, 640), (513, 96, 96),
          (1025, 512, 768)]


@pytest.mark.parametrize("T,n,m", SHAPES)
@pytest.mark.parametrize("w_bits,zeros", [(8, False), (8, True), (4, False), (4, True)])
def test_product_matches_the_definition(T, n, m, w_bits, zeros):
    for dtype in (torch.float32, torch.bfloat16):
        c = product_case(T, n, m, w_bits, zeros, seed=T + n + m)
        N, ref = product_exact(*c, w_bits)
        Y = run_product(*c, w_bits, dtype).double()
        assert ((Y - ref).abs() <= product_bound(N, ref, n, dtype)).all()


@pytest.mark.parametrize("T", [1, 6, 40, 300])
@pytest.mark.parametrize("n", [4096, 30000, 131071])
def test_product_of_the_largest_codes(T, n):
    c = product_case(T, n, 130, 8, False, extreme=True)
    N, ref = product_exact(*c, 8)
    Y = run_product(*c, 8, torch.float32).double()
    assert ((Y - ref).abs() <= product_bound(N, ref, n, torch.float32)).all()


@pytest.mark.parametrize("T", [1, 8, 16, 40, 100, 200])
@pytest.mark.parametrize("w_bits", [8, 4])
@pytest.mark.parametrize("n", [64, 480, 512])
def test_product_is_exact_below_2_24(T, w_bits, n):
    """Large codes of one sign with single units among them: the sum is a whole
    number below 2^24 (512 x 255 x 127) and, with scales of one, the result."""
    g = gen(n)
    m = 200
    xc = torch.randint(228, 256, (T, n), generator=g, device="cuda")
    xc[torch.rand(T, n, generator=g, device="cuda") < 0.1] = 129      # x = 1
    hi = 255 if w_bits == 8 else 15
    w = torch.randint(hi - hi // 8, hi + 1, (m, n), generator=g, device="cuda")
    w[torch.rand(m, n, generator=g, device="cuda") < 0.1] = 1
    wc = w.to(torch.uint8) if w_bits == 8 else (w[:, 0::2] | (w[:, 1::2] << 4)).to(torch.uint8).contiguous()
    one = torch.ones
    Y = run_product(xc.to(torch.uint8), one(T, device="cuda"), wc, one(m, device="cuda"),
                    torch.zeros(m, dtype=torch.uint8, device="cuda"), w_bits, torch.float32)
    assert torch.equal(Y.double(), (xc.double() - 128) @ w.double().T)


@pytest.mark.parametrize("T", [1, 16, 20, 70])
@pytest.mark.parametrize("x,w,z", [(0, 255, 0), (255, 255, 0), (0, 0, 255), (255, 0, 255), (0, 255, 128)])
def test_product_past_32_bits(T, x, w, z):
    """The longest sums of one sign: 131071 x 255 x 128 is more than 2^31."""
    n, m = 131071, 40
    xc = torch.full((T, n), x, dtype=torch.uint8, device="cuda")
    wc = torch.full((m, n), w, dtype=torch.uint8, device="cuda")
    c = (xc, torch.ones(T, device="cuda"), wc, torch.ones(m, device="cuda"),
         torch.full((m,), z, dtype=torch.uint8, device="cuda"))
    N, ref = product_exact(*c, 8)
    Y = run_product(*c, 8, torch.float32).double()
    assert ((Y - ref).abs() <= product_bound(N, ref, n, torch.float32)).all()


@pytest.mark.parametrize("T", [1, 3, 8, 20, 150])
@pytest.mark.parametrize("bx,bw", [(0, 1), (1, 0), (2, 3), (8, 8), (5, 7)])
@pytest.mark.parametrize("w_bits", [8, 4])
def test_product_of_unaligned_codes(T, bx, bw, w_bits):
    xc, xs, wc, ws, wz = product_case(T, 352, 100, w_bits, True, seed=T)
    N, ref = product_exact(xc, xs, wc, ws, wz, w_bits)
    Y = run_product(shifted(xc, bx), shifted(xs, 1), shifted(wc, bw), shifted(ws, 1), shifted(wz, 3), w_bits,
                    torch.float32).double()
    assert ((Y - ref).abs() <= product_bound(N, ref, 352, torch.float32)).all()


@pytest.mark.parametrize("T,n,m", [(17, 4096, 6400), (40, 4096, 4200), (64, 5120, 5000), (2100, 320, 2500), (3, 256, 20000),
                                   (12, 320, 20003), (5, 33, 11000)])
@pytest.mark.parametrize("w_bits", [8, 4])
def test_product_of_many_tiles(T, n, m, w_bits):
    """Token tiles of every width, more tiles than SMs, and more rows than the streaming CTAs hold at once."""
    c = product_case(T, n, m, w_bits, True, seed=m)
    N, ref = product_exact(*c, w_bits)
    Y = run_product(*c, w_bits, torch.float32).double()
    assert ((Y - ref).abs() <= product_bound(N, ref, n, torch.float32)).all()


def test_product_of_the_sweeps_codes():
    """The sweep's 4-bit codes, scales and zero points (one group per row) run as
    they are and give the dequantized weights' product."""
    from paper_2609_00049_gb300 import layer
    g = gen(3)
    W0 = torch.randn(96, 128, generator=g, device="cuda")
    X = torch.randn(256, 128, generator=g, device="cuda")
    H, _, T = layer.accumulate([X], 128)
    q = layer.quantize(W0, layer.prepare(H, T), rq.quant_cfg(group_size=0))
    xc = torch.empty(256, 128, dtype=torch.uint8, device="cuda")
    xs = torch.empty(256, device="cuda")
    Xq = rq.realq_quantize_activations(X, 8, 1.0, codes=xc, scale=xs)
    Y = run_product(xc, xs, q.codes, q.scale.reshape(-1), q.zero.reshape(-1), 4, torch.float32)
    ref = Xq.double() @ q.W.double().T
    # X_q and the dequantized weights are themselves rounded (u each), and so are the scales' products (2u)
    bound = (Xq.double().abs() @ q.W.double().abs().T) * 2 * U + ref.abs() * 4 * U
    assert ((Y.double() - ref).abs() <= bound).all()


def test_product_repeats_bitwise_and_keeps_nothing():
    c1, c2 = product_case(200, 2048, 512, 8, False, 1), product_case(200, 2048, 512, 8, False, 2)
    buf = rq.workspace(rq.realq_int8_product_workspace_size(200, 2048, 512, 8))
    a = run_product(*c1, 8, torch.float32, ws_buf=buf)
    run_product(*c2, 8, torch.float32, ws_buf=buf)
    assert torch.equal(a, run_product(*c1, 8, torch.float32, ws_buf=buf))


def test_operators_on_another_stream():
    c = product_case(70, 640, 256, 8, False)
    _, ref = product_exact(*c, 8)
    x = torch.randn(70, 3000, generator=gen(0), device="cuda")
    y = torch.arange(70, device="cuda")
    lp = torch.empty(70, device="cuda")
    buf = rq.workspace(rq.realq_int8_product_workspace_size(70, 640, 256, 8))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    Y = run_product(*c, 8, torch.float32, ws_buf=buf, stream=s)
    rq.realq_token_logprobs(x, y, lp, stream=s)
    s.synchronize()
    assert ((Y.double() - ref).abs() <= ref.abs() * 4 * U + 1e-30).all()
    assert torch.isfinite(lp).all()


def test_operators_in_a_captured_graph():
    """A head step's operators recorded once and replayed on new inputs."""
    T, d, vocab = 96, 512, 3000
    W = 0.05 * torch.randn(vocab, d, generator=gen(1), device="cuda")
    wc, ws = torch.empty(vocab, d, dtype=torch.uint8, device="cuda"), torch.empty(vocab, device="cuda")
    rq.realq_quantize_activations(W, 8, 1.0, codes=wc, scale=ws)
    xc, xs = torch.empty(T, d, dtype=torch.uint8, device="cuda"), torch.empty(T, device="cuda")
    h, y = torch.empty(T, d, device="cuda"), torch.randint(0, vocab, (T,), generator=gen(2), device="cuda")
    hq = torch.empty_like(h)
    logits, lp, norm = torch.empty(T, vocab, device="cuda"), torch.empty(T, device="cuda"), torch.empty(T, 2, device="cuda")
    codes, exps = torch.empty(T, d, dtype=torch.int8, device="cuda"), torch.empty(T, d // 32, dtype=torch.uint8, device="cuda")
    g, dW = torch.full((T,), -1.0 / T, device="cuda"), torch.empty(vocab, d, device="cuda")
    b1 = rq.workspace(rq.realq_int8_product_workspace_size(T, d, vocab))
    b2 = rq.workspace(rq.realq_checkpoint_weight_grad_workspace_size(T, vocab, d, torch.float32))

    def step(s):
        rq.realq_quantize_activations(h, 8, 1.0, X_q=hq, codes=xc, scale=xs, stream=s)
        rq.realq_int8_product(xc, xs, wc, ws, logits, ws=b1, stream=s)
        rq.realq_token_logprobs(logits, y, lp, norm, stream=s)
        rq.realq_checkpoint_pack(h, codes, exps, stream=s)
        rq.realq_token_logprobs_grad(logits, y, norm, logits, d_logprob=g, stream=s)
        rq.realq_checkpoint_weight_grad(logits, codes, exps, dW, ws=b2, stream=s)

    s = torch.cuda.Stream()
    h.normal_(generator=gen(3))
    s.wait_stream(torch.cuda.current_stream())
    step(s)
    s.synchronize()
    rq.realq_graph_begin(s)
    step(s)
    graph = rq.realq_graph_end(s)
    for seed in (4, 5):
        h.normal_(generator=gen(seed))
        s.wait_stream(torch.cuda.current_stream())
        step(s)
        s.synchronize()
        want = [v.clone() for v in (lp, norm, logits, dW)]
        for v in (lp, norm, logits, dW):
            v.fill_(math.nan)
        s.wait_stream(torch.cuda.current_stream())
        graph.launch(s)
        s.synchronize()
        for v, w in zip((lp, norm, logits, dW), want):
            assert torch.equal(v, w)


# ------------------------------------------------------ log probabilities ---
def forward(x, y, k):
    T = x.shape[0]
    new = lambda *s, dtype=torch.float32: torch.full(s, -7, dtype=dtype, device="cuda")  # noqa: E731
    out = dict(logprob=new(T), norm=new(T, 2), entropy=new(T), top_ids=new(T, k, dtype=torch.int64) if k else None,
               top_logprob=new(T, k) if k else None)
    rq.realq_token_logprobs(x, y, **out)
    return out


def forward_exact(x, y, k):
    """Rows without NaN or +inf."""
    v = x.double()
    m = v.amax(dim=1)
    s = torch.where(torch.isinf(m)[:, None], torch.zeros_like(v), torch.exp(v - m[:, None])).sum(dim=1)
    empty = torch.isinf(m)
    ls = torch.where(empty, torch.zeros_like(s), torch.log(s))
    lp = (v - torch.where(empty, torch.zeros_like(m), m)[:, None]) - ls[:, None]
    p = torch.exp(lp)
    H = -torch.special.xlogy(p, p).sum(dim=1)
    at = y.clamp(min=0, max=v.shape[1] - 1)
    logprob = torch.where(y >= 0, lp.gather(1, at[:, None])[:, 0], torch.zeros_like(H))
    kk = min(k, v.shape[1])
    by = torch.sort(v, dim=1, descending=True, stable=True)
    ids = torch.full((len(v), k), -1, dtype=torch.int64, device="cuda")
    top = torch.full((len(v), k), -INF, dtype=torch.float64, device="cuda")
    if kk:
        none = torch.isinf(by.values[:, :kk])
        ids[:, :kk] = by.indices[:, :kk].masked_fill(none, -1)
        top[:, :kk] = lp.gather(1, by.indices[:, :kk]).masked_fill(none, -INF)
    return dict(logprob=logprob, norm=torch.stack([m, ls], 1), entropy=H, top_ids=ids, top_logprob=top, p=p, lp=lp)


def sum_bound(V):
    """Relative error of s: V/512 + 40 sequential additions of a thread and its
    joins (u each), each term's exponential (2^-22 and the argument's two
    roundings, u |x - m| each, at most log V + 3 where the term counts)."""
    return (V / 512 + 40 + 4 + 2 * (math.log(V) + 3)) * U


def check_forward(out, ref, V, k):
    e = sum_bound(V)
    def near(a, b, tol):
        a = a.double()
        assert torch.equal(torch.isinf(a), torch.isinf(b)) and torch.equal(torch.isnan(a), torch.isnan(b))
        fine = torch.isfinite(b)
        assert torch.equal(a[~fine & ~torch.isnan(b)], b[~fine & ~torch.isnan(b)])
        assert ((a - b).abs()[fine] <= (tol + 4 * U * b.abs() if not torch.is_tensor(tol) else tol + 4 * U * b.abs())[fine]).all()
    near(out["logprob"], ref["logprob"], e)
    near(out["norm"], ref["norm"], e)
    near(out["entropy"], ref["entropy"], e * (2 + 2 * (math.log(V) + 3)))
    if k:
        assert torch.equal(out["top_ids"], ref["top_ids"])
        near(out["top_logprob"], ref["top_logprob"], e)


def logits_case(T, V, dtype, masked, seed=0):
    g = gen(seed)
    x = 3 * torch.randn(T, V, generator=g, device="cuda")
    if masked == "inf":
        x[:, torch.randperm(V, generator=g, device="cuda")[: V // 2]] = -INF
    elif masked == "lowest":
        x[:, torch.randperm(V, generator=g, device="cuda")[: V // 2]] = torch.finfo(dtype).min
    elif masked == "few":       # three tokens left, in the middle
        x[:, : V // 2] = -INF
        x[:, V // 2 + 3:] = -INF
    elif masked == "few_lowest":
        x[:, : V // 2] = torch.finfo(dtype).min
        x[:, V // 2 + 3:] = torch.finfo(dtype).min
    elif masked == "ties":
        x = torch.round(x / 4) * 4
    elif masked == "equal":
        x.fill_(1.25)
    y = torch.randint(0, V, (T,), generator=g, device="cuda")
    if T > 2:
        y[1] = -100
    return x.to(dtype), y


@pytest.mark.parametrize("T,V", [(1, 1), (2, 3), (1, 31), (3, 512), (5, 1000), (1, 50257), (7, 32003), (1, 128256),
                                 (33, 8191), (150, 20000), (400, 4097)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("masked", ["", "inf", "lowest", "few", "few_lowest", "ties", "equal"])
def test_logprobs_match_the_definition(T, V, dtype, masked):
    x, y = logits_case(T, V, dtype, masked, seed=V)
    for k in (0, 1, 5, 32):
        check_forward(forward(x, y, k), forward_exact(x, y, k), V, k)


@pytest.mark.parametrize("T,V", [(700, 8), (700, 1001), (1300, 4099), (900, 16384), (650, 32768)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("masked", ["", "few", "ties"])
def test_logprobs_of_many_short_rows(T, V, dtype, masked):
    x, y = logits_case(T, V, dtype, masked, seed=V)
    for k in (0, 7, 32):
        check_forward(forward(x, y, k), forward_exact(x, y, k), V, k)


def test_logprobs_of_a_vocabulary_past_the_notes():
    """Rows so long that a thread's run maxima are merged."""
    x, y = logits_case(2, 1_500_003, torch.float32, "")
    x[0, 7], x[0, 1_500_002], x[1, 750_000] = 40.0, 40.0, 41.0
    check_forward(forward(x, y, 20), forward_exact(x, y, 20), 1_500_003, 20)


def test_logprobs_of_rows_that_lie_apart():
    for dtype in (torch.float32, torch.bfloat16):
        for V, ld in ((1000, 1003), (50257, 50304), (8, 16)):
            big = 3 * torch.randn(6, ld, generator=gen(1), device="cuda").to(dtype)
            big[:, V:] = 100.0   # what lies between the rows is not read
            y = torch.randint(0, V, (6,), generator=gen(2), device="cuda")
            x = big[:, :V]
            check_forward(forward(x, y, 5), forward_exact(x.contiguous(), y, 5), V, min(5, V))


def test_logprobs_past_32_bits_of_offset():
    V, T = 32768, 70000      # 2.29e9 logits
    x = torch.zeros(T, V, dtype=torch.bfloat16, device="cuda")
    rows = torch.tensor([0, 40000, 65535, 65536, 69999], device="cuda")
    x[rows] = (3 * torch.randn(5, V, generator=gen(4), device="cuda")).to(torch.bfloat16)
    y = torch.randint(0, V, (T,), generator=gen(5), device="cuda")
    out = forward(x, y, 3)
    got = {n: v[rows] for n, v in out.items()}
    check_forward(got, forward_exact(x[rows], y[rows], 3), V, 3)
    d = torch.empty_like(x)
    rq.realq_token_logprobs_grad(x, y, out["norm"], d, d_logprob=torch.ones(T, device="cuda"))
    ref = -forward_exact(x[rows], y[rows], 0)["p"]
    ref[torch.arange(5, device="cuda"), y[rows]] += 1
    assert ((d[rows].double() - ref).abs() <= ref.abs() * (BF + 1e-5) + 1e-6).all()


@pytest.mark.parametrize("V", [1, 40, 5000, 128256])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_without_a_distribution(V, dtype):
    x = torch.randn(5, V, generator=gen(0), device="cuda").to(dtype)
    x[0] = -INF
    x[1, V // 2] = math.nan
    x[2, V - 1] = INF
    x[3, 0] = math.nan
    y = torch.tensor([0, 0, 0, -1, V], device="cuda")
    out = forward(x, y, 3)
    lp = out["logprob"].cpu()
    assert lp[0] == -INF and math.isnan(lp[1]) and math.isnan(lp[2]) and lp[3] == 0 and math.isnan(lp[4])
    assert out["norm"][0].tolist() == [-INF, 0.0] and out["entropy"][0] == 0
    assert torch.isnan(out["norm"][1:4]).all() and torch.isnan(out["entropy"][1:4]).all()
    assert (out["top_ids"][:4] == -1).all() and (out["top_logprob"][0] == -INF).all()
    assert torch.isnan(out["top_logprob"][1:4]).all()
    d = torch.full_like(x, 9.0)
    one = torch.ones(5, device="cuda")
    rq.realq_token_logprobs_grad(x, y, out["norm"], d, d_logprob=one, entropy=out["entropy"], d_entropy=one,
                                 top_ids=out["top_ids"], d_top=torch.ones(5, 3, device="cuda"))
    assert (d[0] == 0).all() and torch.isnan(d[1]).all() and torch.isnan(d[4]).all()


def test_logprobs_write_only_what_is_asked():
    x, y = logits_case(4, 700, torch.float32, "")
    ref = forward_exact(x, y, 0)
    H = torch.empty(4, device="cuda")
    rq.realq_token_logprobs(x, None, entropy=H)
    assert ((H.double() - ref["entropy"]).abs() <= 1e-5).all()
    rq.realq_token_logprobs(x[:0], y[:0], torch.empty(0, device="cuda"))   # no rows


def grad_exact(x, y, g, gH, ids, gt):
    r = forward_exact(x, y, 0)
    p, lp, H = r["p"], r["lp"], r["entropy"]
    c = torch.where(y >= 0, g.double(), torch.zeros_like(H))
    add = torch.zeros_like(p)
    add.scatter_add_(1, y.clamp(min=0)[:, None], c[:, None])
    if ids is not None:
        t = torch.where(ids >= 0, gt.double(), torch.zeros_like(gt.double()))
        add.scatter_add_(1, ids.clamp(min=0), t)
        c = c + t.sum(dim=1)
    lpz = torch.where(p > 0, lp, torch.zeros_like(lp))
    dense = -p * (c[:, None] + gH.double()[:, None] * (lpz + H[:, None]))
    size = p * (c.abs()[:, None] + gH.double().abs()[:, None] * (lpz.abs() + H[:, None])) + add.abs()
    return dense + add, size


@pytest.mark.parametrize("T,V,ld,ldd", [(1, 5, 5, 5), (3, 1000, 1000, 1000), (4, 4099, 4099, 4099), (2, 50257, 50304, 50304),
                                        (5, 9000, 9001, 9000), (2, 40000, 40000, 40008), (300, 777, 777, 777)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("masked", ["", "inf", "lowest", "few_lowest"])
def test_logprobs_gradient_matches_the_formula(T, V, ld, ldd, dtype, masked):
    x0, y = logits_case(T, V, dtype, masked, seed=V)
    x = torch.zeros(T, ld, dtype=dtype, device="cuda")[:, :V].copy_(x0)
    k = min(V, 4)
    out = forward(x, y, k)
    if V > 8:
        out["top_ids"][0, 0] = y[0]       # the target is among the alternatives
        if T > 2:
            out["top_ids"][2, 1] = out["top_ids"][2, 0]   # one listed twice
    g = gen(9)
    w, wH, wt = (torch.randn(T, generator=g, device="cuda"), torch.randn(T, generator=g, device="cuda"),
                 torch.randn(T, k, generator=g, device="cuda"))
    ref, size = grad_exact(x0, y, w, wH, out["top_ids"], wt)
    whole = torch.full((T, ldd), 5.0, dtype=dtype, device="cuda")
    d = whole[:, :V]
    rq.realq_token_logprobs_grad(x, y, out["norm"], d, d_logprob=w, entropy=out["entropy"], d_entropy=wH,
                                 top_ids=out["top_ids"], d_top=wt)
    # p: the log's error (the sum's, and |x - m| u) and the exponential's; then a handful of roundings
    lp = torch.where(torch.isfinite(x0.double()), (x0.double() - x0.double().amax(dim=1, keepdim=True)).abs(), torch.zeros_like(ref))
    rel = sum_bound(V) * (4 + 2 * math.log(V + 1)) + 16 * U + 4 * U * lp.clamp(max=100.0)
    bound = size * rel + (ref.abs() * BF if dtype == torch.bfloat16 else 0.0) + 1e-37
    if dtype == torch.bfloat16:
        bound = bound * (1 + 2 * BF)
    assert ((d.double() - ref).abs() <= bound).all()
    assert (whole[:, V:] == 5.0).all()
    if ld == ldd:                          # in place
        want = d.clone()
        rq.realq_token_logprobs_grad(x, y, out["norm"], x, d_logprob=w, entropy=out["entropy"], d_entropy=wH,
                                     top_ids=out["top_ids"], d_top=wt)
        assert torch.equal(x.view(torch.int32 if dtype == torch.float32 else torch.int16),
                           want.view(torch.int32 if dtype == torch.float32 else torch.int16))


def test_logprobs_gradient_parts_alone():
    x, y = logits_case(6, 900, torch.float32, "inf")
    out = forward(x, y, 3)
    w = torch.randn(6, generator=gen(1), device="cuda")
    zero = torch.zeros(6, device="cuda")
    for part in ("logprob", "entropy", "top"):
        d = torch.empty_like(x)
        wt = torch.randn(6, 3, generator=gen(2), device="cuda")
        if part == "logprob":
            rq.realq_token_logprobs_grad(x, y, out["norm"], d, d_logprob=w)
            ref, size = grad_exact(x, y, w, zero, None, None)
        elif part == "entropy":
            rq.realq_token_logprobs_grad(x, None, out["norm"], d, entropy=out["entropy"], d_entropy=w)
            ref, size = grad_exact(x, y, zero, w, None, None)
        else:
            rq.realq_token_logprobs_grad(x, None, out["norm"], d, top_ids=out["top_ids"], d_top=wt)
            ref, size = grad_exact(x, y, zero, zero, out["top_ids"], wt)
        assert ((d.double() - ref).abs() <= size * (sum_bound(900) * 20 + 128 * U) + 1e-37).all()


def test_logprobs_gradient_against_differences():
    """Central differences of the forward call's own outputs: the loss changes
    by at most e^3 |f'''| / 6 beyond its slope, and is known to the forward's
    bound."""
    x, y = logits_case(3, 32, torch.float32, "")
    y = y.clamp(min=0)
    w, wH = torch.tensor([1.0, -0.5, 0.7], device="cuda"), torch.tensor([0.3, 0.6, -1.0], device="cuda")
    out = forward(x, y, 2)
    wt = torch.tensor([[0.2, -0.4]] * 3, device="cuda")
    d = torch.empty_like(x)
    rq.realq_token_logprobs_grad(x, y, out["norm"], d, d_logprob=w, entropy=out["entropy"], d_entropy=wH,
                                 top_ids=out["top_ids"], d_top=wt)

    def loss(v):
        o = forward(v, y, 32)
        lp = torch.full_like(v, 0).double()
        lp.scatter_(1, o["top_ids"], o["top_logprob"].double())   # all 32 log probabilities
        return (w.double() * o["logprob"].double() + wH.double() * o["entropy"].double()
                + (wt.double() * lp.gather(1, out["top_ids"])).sum(dim=1))

    e = 0.03
    for j in range(0, 32, 3):
        up, dn = x.clone(), x.clone()
        up[:, j] += e
        dn[:, j] -= e
        step = (up[:, j].double() - dn[:, j].double())
        slope = (loss(up) - loss(dn)) / step
        # third derivatives of log p and H along one logit are at most 1 and 2 + 2 log 32
        bound = e * e / 6 * (1.0 + 0.6 + 1.0 * (2 + 2 * math.log(32))) + 4 * 2.6 * sum_bound(32) * 12 / (2 * e)
        assert ((slope - d[:, j].double()).abs() <= bound).all()


# ------------------------------------------------------------ checkpoints ---
def pack_exact(x):
    """Codes and bytes from the definition, in 64 bits."""
    T, n = x.shape
    nb = -(-n // 32)
    v = torch.nn.functional.pad(x.double(), (0, nb * 32 - n)).reshape(T, nb, 32)
    amax = torch.nn.functional.pad(x.float(), (0, nb * 32 - n)).reshape(T, nb, 32).abs().view(torch.int32).amax(dim=2)
    byte = amax >> 23
    step = torch.ldexp(torch.ones_like(byte, dtype=torch.float64, device="cpu"), (byte.cpu() - 133)).cuda()
    q = torch.clamp(torch.round(v / step[:, :, None]), -127, 127)
    bad = byte == 255
    q = torch.where(bad[:, :, None], torch.zeros_like(q), q)
    val = torch.where(bad[:, :, None], torch.full_like(q, math.nan), q * step[:, :, None])
    return q.reshape(T, -1)[:, :n].to(torch.int8), byte.to(torch.uint8), val.reshape(T, -1)[:, :n]


@pytest.mark.parametrize("T,n", [(1, 1), (1, 32), (3, 31), (2, 33), (5, 64), (7, 100), (64, 4096), (17, 1111), (3, 28672)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shift", [0, 1])
def test_checkpoint_matches_the_definition(T, n, dtype, shift):
    g = gen(n)
    x = torch.randn(T, n, generator=g, device="cuda") * torch.exp2(torch.randint(-40, 40, (T, n), generator=g, device="cuda").float())
    x[0, : n // 2] = 0
    x = shifted(x.to(dtype), shift)
    codes = shifted(torch.empty(T, n, dtype=torch.int8, device="cuda"), shift)
    exps = torch.empty(T, -(-n // 32), dtype=torch.uint8, device="cuda")
    rq.realq_checkpoint_pack(x, codes, exps)
    q, byte, val = pack_exact(x)
    assert torch.equal(codes, q) and torch.equal(exps, byte)
    for out_dtype in (torch.float32, torch.bfloat16):
        y = shifted(torch.empty(T, n, dtype=out_dtype, device="cuda"), shift)
        rq.realq_checkpoint_unpack(codes, exps, y)
        assert torch.equal(y.double(), val)
    assert ((val - x.double()).abs() <= torch.exp2(byte.double() - 133).repeat_interleave(32, 1)[:, :n]).all()


def test_checkpoint_of_the_ends_of_the_range():
    big, tiny = torch.finfo(torch.float32).max, 2.0 ** -149
    rows = [[big, -big, 1.0], [tiny, -3 * tiny, 0.0], [2.0 ** -126, -2.0 ** -133, 0.0], [0.0, -0.0, 0.0], [1.0, INF, 2.0],
            [1.0, math.nan, 2.0], [-INF, 0.0, 0.0], [127.5, -127.5, 1.0], [127.0, 63.5, 0.5]]
    x = torch.zeros(len(rows), 64, device="cuda")
    for i, r in enumerate(rows):
        x[i, :3] = torch.tensor(r)
    x[:, 32:] = 1.5      # the neighbouring block is not touched
    codes, exps, y = torch.empty(len(rows), 64, dtype=torch.int8, device="cuda"), torch.empty(len(rows), 2, dtype=torch.uint8, device="cuda"), torch.empty_like(x)
    rq.realq_checkpoint_pack(x, codes, exps)
    q, byte, val = pack_exact(x)
    assert torch.equal(codes, q) and torch.equal(exps, byte)
    rq.realq_checkpoint_unpack(codes, exps, y)
    assert torch.equal(torch.isnan(y), torch.isnan(val))
    assert torch.equal(torch.nan_to_num(y.double()), torch.nan_to_num(val))
    assert (y[:, 32:] == 1.5).all() and exps[4:7, 0].tolist() == [255] * 3


def test_checkpoint_of_tiny_and_huge_bf16():
    """Blocks whose scale is no bf16 number, and subnormal values beside the smallest that is."""
    g = gen(0)
    x = torch.randn(64, 256, generator=g, device="cuda")
    e = torch.arange(64, device="cuda")
    x[:32] *= torch.exp2(-133.0 + 0.5 * e[:32, None])     # 2^-133 .. 2^-117
    x[32:] *= torch.exp2(94.0 + e[32:, None].clamp(max=62) - 32)
    x = x.clamp(-3e38, 3e38).to(torch.bfloat16)
    codes = torch.empty(64, 256, dtype=torch.int8, device="cuda")
    exps = torch.empty(64, 8, dtype=torch.uint8, device="cuda")
    rq.realq_checkpoint_pack(x, codes, exps)
    q, byte, val = pack_exact(x)
    assert torch.equal(codes, q) and torch.equal(exps, byte)
    for out_dtype in (torch.float32, torch.bfloat16):
        y = torch.empty(64, 256, dtype=out_dtype, device="cuda")
        rq.realq_checkpoint_unpack(codes, exps, y)
        assert torch.equal(y.double(), val)


# ------------------------------------------------------- weight gradients ---
def weight_grad_case(T, m, n, dtype, seed=0):
    g = gen(seed)
    x = torch.randn(T, n, generator=g, device="cuda")
    x[:, :: max(1, n // 3)] *= 30
    codes = torch.empty(T, n, dtype=torch.int8, device="cuda")
    exps = torch.empty(T, -(-n // 32), dtype=torch.uint8, device="cuda")
    rq.realq_checkpoint_pack(x, codes, exps)
    dy = (1e-3 * torch.randn(T, m, generator=g, device="cuda")).to(dtype)
    X = torch.empty(T, n, device="cuda")
    rq.realq_checkpoint_unpack(codes, exps, X)
    return dy, codes, exps, X


def weight_grad(dy, codes, exps, dW=None, accumulate=False):
    T, m = dy.shape
    n = codes.shape[1]
    dW = torch.full((m, n), math.nan, device="cuda") if dW is None else dW
    ws = rq.workspace(rq.realq_checkpoint_weight_grad_workspace_size(T, m, n, dy.dtype))
    rq.realq_checkpoint_weight_grad(dy, codes, exps, dW, accumulate=accumulate, ws=ws)
    rq.realq_workspace_status(ws)
    return dW


def weight_grad_bound(T, dy, X):
    """Per element: 64 accumulations to a promoted part, two units each of its
    partial sums, then one rounding per part (at most T/256 + 8 of them)."""
    return (dy.double().abs().T @ X.double().abs()) * ((64 * 2 + T / 256 + 8) * U) + 1e-37


@pytest.mark.parametrize("T,m,n", [(1, 1, 1), (1, 64, 64), (3, 5, 7), (17, 100, 31), (63, 130, 257), (64, 128, 256),
                                   (65, 129, 300), (200, 8, 1024), (513, 256, 512), (1000, 333, 777), (1999, 512, 1024),
                                   (2048, 1000, 264), (5000, 64, 96)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_weight_grad_matches_the_definition(T, m, n, dtype):
    dy, codes, exps, X = weight_grad_case(T, m, n, dtype, seed=T + m)
    ref = dy.double().T @ X.double()
    got = weight_grad(dy, codes, exps)
    assert ((got.double() - ref).abs() <= weight_grad_bound(T, dy, X)).all()
    # added to what is there: one rounding more
    base = torch.randn(m, n, generator=gen(8), device="cuda")
    both = weight_grad(dy, codes, exps, base.clone(), accumulate=True)
    assert ((both.double() - (ref + base.double())).abs() <= weight_grad_bound(T, dy, X) + 2 * U * (ref.abs() + base.double().abs())).all()
    assert torch.equal(got, weight_grad(dy, codes, exps))   # bitwise repeatable


@pytest.mark.parametrize("T,m,n", [(300, 2600, 2200), (700, 64, 20000), (129, 20001, 70)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_weight_grad_of_many_tiles(T, m, n, dtype):
    dy, codes, exps, X = weight_grad_case(T, m, n, dtype, seed=T)
    ref = dy.double().T @ X.double()
    assert ((weight_grad(dy, codes, exps).double() - ref).abs() <= weight_grad_bound(T, dy, X)).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_weight_grad_against_differences(dtype):
    """The loss sum(dY * (X W^T)) is linear in W: its change along any direction
    is the gradient's inner product with it."""
    T, m, n = 300, 70, 90
    dy, codes, exps, X = weight_grad_case(T, m, n, dtype)
    dW = weight_grad(dy, codes, exps).double()
    W = torch.randn(m, n, generator=gen(1), device="cuda").double()
    E = torch.randn(m, n, generator=gen(2), device="cuda").double()
    loss = lambda w: (dy.double() * (X.double() @ w.T)).sum()  # noqa: E731
    bound = (weight_grad_bound(T, dy, X) * E.abs()).sum()
    assert ((loss(W + E) - loss(W)) - (dW * E).sum()).abs() <= bound


def test_weight_grad_keeps_what_is_not_finite():
    dy, codes, exps, X = weight_grad_case(100, 40, 96, torch.float32)
    dy[7, 3] = INF
    dy[9, 5] = math.nan
    exps[50, 1] = 255        # a block that held an infinity or a NaN
    got = weight_grad(dy, codes, exps)
    rq.realq_checkpoint_unpack(codes, exps, X)
    ref = dy.double().T @ X.double()
    assert torch.equal(torch.isfinite(got), torch.isfinite(ref))


def test_weight_grad_of_no_tokens():
    dW = torch.ones(4, 8, device="cuda")
    none = [torch.empty(0, 4, device="cuda"), torch.empty(0, 8, dtype=torch.int8, device="cuda"), torch.empty(0, 1, dtype=torch.uint8, device="cuda")]
    rq.realq_checkpoint_weight_grad(*none, dW, accumulate=True)
    assert (dW == 1).all()
    rq.realq_checkpoint_weight_grad(*none, dW)
    assert (dW == 0).all()


# ------------------------------------------------------ together: the head ---
@pytest.mark.parametrize("T,d,vocab,dtype", [(1, 128, 1000, torch.bfloat16), (5, 96, 777, torch.float32),
                                             (130, 256, 4096, torch.bfloat16), (300, 1024, 5001, torch.float32)])
def test_head_scores_and_trains(T, d, vocab, dtype):
    from paper_2609_00049_gb300.head import Head8
    g = gen(T)
    W = 0.05 * torch.randn(vocab, d, generator=g, device="cuda")
    h = torch.randn(T, d, generator=g, device="cuda")
    y = torch.randint(0, vocab, (T,), generator=g, device="cuda")
    if T > 2:
        y[2] = -1
    head = Head8(W, logits_dtype=dtype)
    step = head.forward(h, y, k=min(5, vocab))
    # the codes' own values give the logits exactly, up to the scales' roundings and the logits' type
    x8, w8 = torch.empty_like(h), torch.empty_like(W)
    xc, xs = torch.empty(T, d, dtype=torch.uint8, device="cuda"), torch.empty(T, device="cuda")
    rq.realq_quantize_activations(h, 8, 1.0, X_q=x8, codes=xc, scale=xs)
    rq.realq_quantize_activations(W, 8, 1.0, X_q=w8)
    logits = x8.double() @ w8.double().T
    tol = (x8.double().abs() @ w8.double().abs().T) * 2 * U + logits.abs() * (4 * U + (BF if dtype == torch.bfloat16 else 0.0))
    assert ((step.logits.double() - logits).abs() <= tol).all()
    # scores and gradient are those of the logits as they were stored
    stored = step.logits.clone()
    ref = forward_exact(stored, y, 5)
    check_forward(dict(logprob=step.logprob, norm=step.norm, entropy=step.entropy, top_ids=step.top_ids,
                       top_logprob=step.top_logprob), ref, vocab, 5)
    scored = y >= 0
    assert abs(step.perplexity() / math.exp(-ref["logprob"][scored].mean().item()) - 1) <= sum_bound(vocab) + 40 * U
    w = torch.where(scored, -1.0 / scored.sum(), 0.0).float()
    dW = head.weight_grad(step, w)
    X = torch.empty(T, d, device="cuda")
    rq.realq_checkpoint_unpack(step.codes, step.exps, X)
    dl, size = grad_exact(stored, y, w, torch.zeros(T, device="cuda"), None, None)
    err = size * (sum_bound(vocab) * (4 + 2 * math.log(vocab)) + 16 * U + 400 * U) + (dl.abs() * BF if dtype == torch.bfloat16 else 0.0) * (1 + BF) + 1e-37
    bound = err.T @ X.double().abs() + weight_grad_bound(T, (dl.abs() + err).float(), X)
    assert ((dW.double() - dl.T @ X.double()).abs() <= bound * 1.01).all()
    # (checkpoints of h, not of its 8-bit row codes: half a step of 1/64 of a block's largest value)
    assert ((X - h).abs() <= h.abs().amax(dim=1, keepdim=True) / 64).all()
    with pytest.raises(ValueError):
        head.weight_grad(step, w)
