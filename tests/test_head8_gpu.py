"""The LM head on 8-bit codes on the GPU: streams of the caller's choice, and
hidden states that a pass has to carry through."""
import math

import pytest
import torch

import paper_2609_00049_gb300 as rq
from paper_2609_00049_gb300.head import Head8

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2609_00049_gb300 import build as b
    b.build()
    rq.lib()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def inputs(T, d, vocab, seed=0):
    g = gen(seed)
    h = torch.randn(T, d, generator=g, device="cuda")
    y = torch.randint(0, vocab, (T,), generator=g, device="cuda")
    return h, y, torch.full((T,), -1.0 / T, device="cuda")


def scores(step):
    return [step.logprob, step.entropy, step.top_ids, step.top_logprob, step.norm, step.codes, step.exps]


@pytest.mark.parametrize("T", [1, 12, 200])
def test_a_pass_on_a_side_stream_gives_the_same_bits(T):
    """With allocations and writes on the default stream all the while, and with
    passes of several sizes on two streams that share the head's workspaces."""
    d, vocab = 512, 4099
    W = 0.05 * torch.randn(vocab, d, generator=gen(1), device="cuda")
    cases = [inputs(t, d, vocab, seed=t) for t in (T, 3 * T, T)]
    plain, want = Head8(W), []
    for h, y, w in cases:
        step = plain.forward(h, y, k=3)
        got = [v.clone() for v in scores(step)]
        want.append((got, step.perplexity(), plain.weight_grad(step, w)))
    torch.cuda.synchronize()
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    head = Head8(W)
    for _ in range(5):
        for i, (h, y, w) in enumerate(cases):
            step = head.forward(h.clone(), y, k=3, stream=side if i % 2 else other)
            for n in (T * d, T * vocab, 4096, T * 4):   # memory that a pass may have given back too early
                torch.empty(n, device="cuda").fill_(math.nan)
            ppl = step.perplexity()
            kept = scores(step)
            dW = head.weight_grad(step, w.clone(), stream=side)
            for n in (T * d, T * vocab, 2 * T * vocab):
                torch.empty(n, device="cuda").fill_(math.nan)
            torch.cuda.current_stream().wait_stream(side)
            assert ppl == want[i][1]
            for a, b in zip(kept + [dW], want[i][0] + [want[i][2]]):
                assert torch.equal(a, b)


BAD = [math.nan, math.inf, -math.inf]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("n", [1, 31, 64, 515])
def test_quantized_activations_show_what_is_not_finite(dtype, bits, n):
    """A token with an infinity or a NaN: NaN scale and values; the others are as without it."""
    x = torch.randn(9, n, generator=gen(n), device="cuda").to(dtype)

    def run(v):
        codes = torch.empty(9, (n + 1) // 2 if bits <= 4 else n, dtype=torch.uint8, device="cuda")
        scale = torch.empty(9, device="cuda")
        return rq.realq_quantize_activations(v, bits, 0.9, codes=codes, scale=scale), codes, scale

    want = run(x)
    bad = x.clone()
    for i, v in enumerate(BAD):
        bad[2 * i + 1, (n // 2 + i) % n] = v
    got = run(bad)
    rows = torch.arange(9, device="cuda")
    hit = (rows % 2 == 1) & (rows < 6)
    assert torch.isnan(got[0][hit]).all() and torch.isnan(got[2][hit]).all()
    packed = 128 if bits == 8 else 0x88
    assert (got[1][hit][:, : n // 2] == packed).all()
    for a, b in zip(got, want):
        assert torch.equal(a[~hit], b[~hit])


@pytest.mark.parametrize("T", [5, 40])     # both sides of the product's dispatch
@pytest.mark.parametrize("logits", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("value", BAD)
def test_a_hidden_state_that_is_not_finite_shows(T, logits, value):
    """Its log probability and entropy are NaN, the other tokens' are untouched,
    and the weight gradient of the same step is NaN where it takes part."""
    d, vocab = 1024, 30011
    h, y, w = inputs(T, d, vocab)
    head = Head8(0.05 * torch.randn(vocab, d, generator=gen(2), device="cuda"), logits_dtype=logits)
    want = head.forward(h, y, k=4)
    h = h.clone()
    h[3, 700] = value
    step = head.forward(h, y, k=4)
    rows = torch.arange(T, device="cuda") != 3
    assert torch.isnan(step.logits[3]).all() and torch.isnan(step.logprob[3]) and torch.isnan(step.entropy[3])
    assert (step.top_ids[3] == -1).all()
    assert math.isnan(step.perplexity())
    for a, b in ((step.logprob, want.logprob), (step.entropy, want.entropy), (step.top_ids, want.top_ids)):
        assert torch.equal(a[rows], b[rows])
    dW = head.weight_grad(step, w)
    assert torch.isnan(dW).all()


def test_a_pass_of_no_tokens():
    head = Head8(torch.randn(300, 64, generator=gen(0), device="cuda"))
    h, y, w = torch.empty(0, 64, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda")
    step = head.forward(h, y, k=2)
    assert step.logprob.shape == (0,) and step.top_ids.shape == (0, 2) and math.isnan(step.perplexity())
    dW = torch.ones(300, 64, device="cuda")
    assert (head.weight_grad(step, w, dW=dW) == 1).all()
    assert (head.weight_grad(head.forward(h, y), w) == 0).all()
