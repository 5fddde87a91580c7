"""What the 8-bit linear operators promise beyond their values at ordinary
inputs: status words that outlive a call, and the sums' accuracy at the ends of
the codes' range.  U = 2^-24 is the unit roundoff of fp32."""
import pytest
import torch

import paper_2609_00049_gb300 as rq

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2609_00049_gb300 import build as b
    b.build()
    rq.lib()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


# ------------------------------------------------------------ status words ---
def gave_up(ws):
    """What a bounded wait that gave up leaves in a workspace."""
    ws[:4].view(torch.int32).fill_(4)


def raises_timeout(ws):
    with pytest.raises(rq.RealqError) as e:
        rq.realq_workspace_status(ws)
    assert e.value.status == rq.REALQ_ERR_TIMEOUT
    rq.realq_workspace_status(ws)     # reading it clears it


@pytest.mark.parametrize("T,n,m,w_bits", [(1, 1024, 300, 8), (12, 96, 200, 4), (40, 31, 50, 8), (300, 640, 256, 8),
                                          (300, 200, 256, 4), (300, 101, 77, 8)])
def test_a_product_keeps_an_earlier_calls_status(T, n, m, w_bits):
    xc = torch.randint(0, 256, (T, n), generator=gen(0), device="cuda").to(torch.uint8)
    wc = torch.randint(0, 256, (m, n if w_bits == 8 else (n + 1) // 2), generator=gen(1), device="cuda").to(torch.uint8)
    Y = torch.empty(T, m, device="cuda")
    ws = rq.workspace(rq.realq_int8_product_workspace_size(T, n, m, w_bits))
    gave_up(ws)
    rq.realq_int8_product(xc, torch.ones(T, device="cuda"), wc, torch.ones(m, device="cuda"), Y, w_bits=w_bits, ws=ws)
    raises_timeout(ws)
    rq.realq_int8_product(xc, torch.ones(T, device="cuda"), wc, torch.ones(m, device="cuda"), Y, w_bits=w_bits, ws=ws)
    rq.realq_workspace_status(ws)


@pytest.mark.parametrize("T,m,n", [(1, 64, 64), (300, 333, 777)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_weight_gradient_keeps_an_earlier_calls_status(T, m, n, dtype):
    dy = torch.randn(T, m, generator=gen(0), device="cuda").to(dtype)
    codes = torch.randint(-127, 128, (T, n), generator=gen(1), device="cuda").to(torch.int8)
    exps = torch.full((T, -(-n // 32)), 127, dtype=torch.uint8, device="cuda")
    dW = torch.empty(m, n, device="cuda")
    ws = rq.workspace(rq.realq_checkpoint_weight_grad_workspace_size(T, m, n, dtype))
    gave_up(ws)
    rq.realq_checkpoint_weight_grad(dy, codes, exps, dW, ws=ws)
    raises_timeout(ws)


def test_a_head_reports_a_pass_that_gave_up():
    """By check(), and by perplexity(), also after the workspace was replaced by a larger one."""
    from paper_2609_00049_gb300.head import Head8
    d, vocab = 64, 500
    head = Head8(torch.randn(vocab, d, generator=gen(0), device="cuda"))
    h = torch.randn(400, d, generator=gen(1), device="cuda")
    y = torch.randint(0, vocab, (400,), generator=gen(2), device="cuda")
    step = head.forward(h[:70].contiguous(), y[:70].contiguous())
    small = head._ws["product"]
    gave_up(small)
    larger = head.forward(h, y)
    assert head._ws["product"] is not small
    for call in (step.perplexity, head.check):
        with pytest.raises(rq.RealqError) as e:
            call()
        assert e.value.status == rq.REALQ_ERR_TIMEOUT
        larger.perplexity()
        gave_up(head._ws["product"])
    head.weight_grad(larger, torch.full((400,), -1.0 / 400, device="cuda"))
    with pytest.raises(rq.RealqError):
        head.check()
    gave_up(head._ws["grad"])
    with pytest.raises(rq.RealqError):
        head.check()
    head.check()


# ------------------------------------------------------------------- sums ---
def exact_sums(xc, w, z):
    return (xc.double() - 128) @ (w.double() - z).T


def largest_running_sum(xc, w, z, step=16):
    """The largest magnitude of a sum over consecutive columns, taken 16 columns
    at a time (their products' magnitudes added for what lies inside a step)."""
    x, v = xc.double() - 128, w.double() - z
    lo = hi = total = torch.zeros(x.shape[0], v.shape[0], dtype=torch.float64, device="cuda")
    inside = torch.zeros_like(lo)
    for j in range(0, x.shape[1], step):
        a, b = x[:, j:j + step], v[:, j:j + step]
        total = total + a @ b.T
        inside = torch.maximum(inside, a.abs() @ b.abs().T)
        lo, hi = torch.minimum(lo, total), torch.maximum(hi, total)
    return hi - lo + 2 * inside


def check_sums(T, xc, w, wc, z, w_bits):
    """With scales of one.  Up to 16 tokens the integer sum is exact and rounded
    once; above, each 16 columns may lose 2 U of the largest running sum once
    that passes 2^24 (and the parts of a split sum, at most 16, as much again)."""
    n, m = xc.shape[1], w.shape[0]
    Y = torch.empty(T, m, device="cuda")
    ws = rq.workspace(rq.realq_int8_product_workspace_size(T, n, m, w_bits))
    zero = torch.full((m,), z, dtype=torch.uint8, device="cuda")
    rq.realq_int8_product(xc, torch.ones(T, device="cuda"), wc, torch.ones(m, device="cuda"), Y, w_bits=w_bits,
                          w_zero=zero, ws=ws)
    rq.realq_workspace_status(ws)
    N = exact_sums(xc, w, z)
    if T <= 16:
        assert torch.equal(Y, N.float())
    else:
        run = largest_running_sum(xc, w, z)
        lost = torch.where(run < 2.0 ** 24, torch.zeros_like(run), 2 * U * (n / 16 + 16) * run)
        assert ((Y.double() - N).abs() <= lost + U * N.abs()).all()


def packed(w):
    if w.shape[1] % 2:
        w = torch.cat([w, torch.zeros_like(w[:, :1])], dim=1)
    return (w[:, 0::2] | (w[:, 1::2] << 4)).contiguous()


@pytest.mark.parametrize("T", [1, 16, 17, 40, 200, 300])
@pytest.mark.parametrize("n", [4096, 8192, 20001])
def test_sums_that_cancel_past_2_24(T, n):
    """The first half of the columns adds up to far more than 2^24, the second
    half takes it away again but for a few units."""
    m = 70
    xc = torch.full((T, n), 255, dtype=torch.uint8, device="cuda")
    xc[:, n // 2:] = 1
    w = torch.full((m, n), 255, dtype=torch.uint8, device="cuda")
    w[:, : m] -= torch.eye(m, dtype=torch.uint8, device="cuda") * 7
    check_sums(T, xc, w, w, 0, 8)


@pytest.mark.parametrize("T", [1, 8, 16, 20, 150])
@pytest.mark.parametrize("n", [131071, 131040])
@pytest.mark.parametrize("x,c,z", [(255, 15, 0), (0, 15, 0), (0, 0, 15), (255, 0, 15)])
def test_longest_sums_of_4_bit_codes(T, n, x, c, z):
    m = 40
    xc = torch.full((T, n), x, dtype=torch.uint8, device="cuda")
    w = torch.full((m, n), c, dtype=torch.uint8, device="cuda")
    check_sums(T, xc, w, packed(w), z, 4)


@pytest.mark.parametrize("T", [1, 9, 40, 300])
@pytest.mark.parametrize("n", [96, 1003])
@pytest.mark.parametrize("z", [16, 100, 255])
def test_4_bit_zero_points_beyond_the_codes(T, n, z):
    """A zero point is a byte, whatever the width of the codes."""
    m = 130
    xc = torch.randint(0, 256, (T, n), generator=gen(n), device="cuda").to(torch.uint8)
    w = torch.randint(0, 16, (m, n), generator=gen(z), device="cuda").to(torch.uint8)
    check_sums(T, xc, w, packed(w), z, 4)
