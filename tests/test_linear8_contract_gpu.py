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
