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
