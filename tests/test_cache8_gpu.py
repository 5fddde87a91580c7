"""Sequences generated with the 8-bit cache against attention over all of their
tokens in 64 bits: prompts, single tokens, forks, leavers and compaction together."""
import pytest
import torch

import paper_2609_00049_gb300 as rq
from kv_reference import attention, gen

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2609_00049_gb300 import build as b
    b.build()
    rq.lib()


def turned(x, pos, f):
    R = 2 * f.numel()
    t = (pos.double()[:, None] * f)[:, None]
    a, b = x[..., :R // 2].double(), x[..., R // 2:R].double()
    return torch.cat([a * torch.cos(t) - b * torch.sin(t), b * torch.cos(t) + a * torch.sin(t), x[..., R:].double()], dim=-1)


@pytest.mark.parametrize("dtype,D,page,block", [(torch.bfloat16, 128, 64, 16), (torch.float32, 64, 16, 1)])
def test_generation(dtype, D, page, block):
    from paper_2609_00049_gb300.cache import Cache8
    rows, kv, H, layers = 5, 2, 8, 2
    f = rq.realq_rotary_frequencies(D // 2, 500000.0, "ramp", 8.0).cuda()
    cache = Cache8(layers, 200 * 16 // page, rows, 700, kv, D, page_size=page, scale_block=block, inv_freq=f)
    held = [[(torch.zeros(0, kv, D, dtype=torch.float64, device="cuda"),) * 2 for _ in range(layers)] for _ in range(rows)]
    worst = 0.0
    g = gen(1)
    plan = [[130, 7, 0, 1, 40], [1, 1, 0, 1, 1], ("fork", [0, 1], [2, 3]), [1, 1, 1, 1, 1], [1, 3, 9, 0, 1], ("release", [1]), ("compact",),
            [1, 33, 1, 1, 0], ("fork", [2, 0, 4], [0, 2, 4]), [2, 1, 1, 2, 60], [1, 1, 1, 1, 1]]
    for what in plan:
        if isinstance(what, tuple):
            if what[0] == "fork":
                cache.fork(what[1], what[2])
                old = [list(h) for h in held]
                for s, d in zip(what[1], what[2]):
                    held[d] = list(old[s])
            elif what[0] == "release":
                cache.release(what[1])
                for s in what[1]:
                    held[s] = [(torch.zeros(0, kv, D, dtype=torch.float64, device="cuda"),) * 2 for _ in range(layers)]
            else:
                cache.compact()
            continue
        step = cache.begin(what)
        T = sum(what)
        pos = torch.cat([torch.arange(len(held[s][0][0]), len(held[s][0][0]) + n) for s, n in enumerate(what)]).cuda()
        assert torch.equal(step.positions, pos)
        for la in range(layers):
            q, k, v = (torch.randn(T, n, D, generator=g, device="cuda").to(dtype) for n in (H, kv, kv))
            q0, k0 = q.clone(), k.clone()
            out = cache.attend(step, la, q, k, v)
            u = torch.finfo(dtype).eps / 2
            for x, x0 in ((q, q0), (k, k0)):      # turned in place, rounded once
                ref = turned(x0, pos, f)
                assert bool(((x.double() - ref).abs() <= u * ref.abs() + 2.0 ** -20 * x0.double().norm(dim=-1, keepdim=True)).all())
            at = 0
            for s, n in enumerate(what):
                K, V = (torch.cat([a, b[at:at + n].double()]) for a, b in zip(held[s][la], (k, v)))
                held[s][la] = (K, V)
                if n:
                    L = len(K)
                    y, _, mag, _ = attention(q[at:at + n], K, V, L, 0, True, D ** -0.5)
                    # Against the values themselves: a code is off by half a step of 1/127 of its block's largest value, and by
                    # another half for every time its block's scale grew (a block of b tokens: at most b - 1 times).
                    # The largest of a block's normal values is below 6, so a value is off by d = 6 b / 254 at most (its kept
                    # codes included); a score by sqrt(D) d |q| / sqrt(D), its weight by e to that, both signs.
                    d = 6.0 * (1 + 0.5 * (block - 1)) / 254
                    ds = (d * q[at:at + n].double().abs().sum(-1) * D ** -0.5).repeat_interleave(1, dim=1)
                    tol = d + (torch.expm1(2 * ds)[..., None]) * (mag + y.abs()) + 2.0 ** -8 * y.abs() + 2.0 ** -8
                    err = (out[at:at + n].double() - y).abs()
                    assert bool((err <= tol).all())
                    worst = max(worst, float(err.square().mean().sqrt() / y.square().mean().sqrt()))
                at += n
    cache.check()
    # the codes' own error, typically a step of 6 / 127 uniform: 0.014 of a value of size 1, less its mean over tokens
    assert worst < 0.06
    with pytest.raises(rq.RealqError) as e:
        cache.begin([700, 700, 700, 700, 700])
        cache.check()
    assert e.value.status == rq.REALQ_ERR_NO_PAGES
    with pytest.raises(ValueError):
        cache.begin([1, 2])


def test_a_refused_step_changes_nothing():
    """Attending after a refused step neither writes nor faults; the next step goes on as if it had not been."""
    from paper_2609_00049_gb300.cache import Cache8
    cache = Cache8(1, 4, 2, 160, 1, 64, page_size=16, scale_block=16)
    def through(counts, seed):
        step = cache.begin(counts)
        T = sum(counts)
        q, k, v = (torch.randn(T, n, 64, generator=gen(seed + i), device="cuda") for i, n in enumerate((2, 1, 1)))
        return cache.attend(step, 0, q, k, v)
    through([20, 10], 1)
    before = [t.clone() for t in cache.cache.tensors] + [cache.tables.clone(), cache.lengths.clone()]
    through([40, 5], 5)
    for a, b in zip(before, list(cache.cache.tensors) + [cache.tables, cache.lengths]):
        assert torch.equal(a, b)
    with pytest.raises(rq.RealqError):
        cache.check()
    out = through([5, 5], 9)
    cache.check()
    assert bool(torch.isfinite(out).all()) and cache.lengths.tolist() == [25, 15]


def two_caches(**kw):
    from paper_2609_00049_gb300.cache import Cache8
    return [Cache8(2, 40, 3, 300, 2, 64, page_size=16, **kw) for _ in range(2)]


def tokens(T, seed):
    return [torch.randn(T, n, 64, generator=gen(seed + i), device="cuda").to(torch.bfloat16) for i, n in enumerate((8, 2, 2))]


def test_calls_on_other_streams():
    """Calls handed from stream to stream, their lists freed at once and the memory reused, give what one stream gives."""
    here, there = two_caches()
    streams = [torch.cuda.Stream() for _ in range(3)] + [None]
    plan = [[70, 3, 0], ("fork", [0], [2]), [1, 1, 1], ("compact",), [1, 40, 2], ("release", [1]), [1, 0, 5], ("fork", [2], [1]), [2, 2, 2]]
    for turn in range(3):
        at = 0
        for i, what in enumerate(plan):
            if isinstance(what, tuple):
                for c, kw in ((here, {}), (there, dict(stream=streams[(at := at + 1) % 4]))):
                    getattr(c, what[0])(*what[1:], **kw)
                torch.full((4096,), 7, dtype=torch.int32, device="cuda")     # (what lists' memory might become)
                continue
            steps = [here.begin(what), there.begin(what, stream=streams[(at := at + 1) % 4])]
            for la in range(2):
                x = tokens(sum(what), 100 * turn + 10 * i + la)
                want = here.attend(steps[0], la, *[t.clone() for t in x])
                s = streams[(at := at + 1) % 4]
                y = [t.clone() for t in x]
                got = there.attend(steps[1], la, *y, stream=s)
                del y
                torch.full((4096, 64), 7.0, device="cuda")
                if s is not None:
                    torch.cuda.current_stream().wait_stream(s)
                assert torch.equal(got, want), (turn, i, la)
        for c in (here, there):
            c.check()
            c.release([0, 1, 2])
    assert there.used.sum().item() == 0


def test_a_captured_token():
    """`attend` captured once and replayed for the tokens after it, the first call of its cache among them."""
    eager, captured = two_caches()
    for c in (eager, captured):
        c.begin([20, 7, 1])
    step = captured.begin([1, 1, 1])
    eager.begin([1, 1, 1])
    buf, out = tokens(3, 0), torch.empty(3, 8, 64, device="cuda", dtype=torch.bfloat16)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        captured.attend(step, 1, *buf, out=out)
    for t in range(5):
        x = tokens(3, 10 + t)
        a, b = eager.begin([1, 1, 1]), captured.begin([1, 1, 1])
        want = eager.attend(a, 1, *[v.clone() for v in x])
        for to, v in zip(buf, x):
            to.copy_(v)
        step.starts.copy_(b.starts)
        step.positions.copy_(b.positions)
        g.replay()
        assert torch.equal(out, want)
    for a, b in zip(eager.cache.tensors, captured.cache.tensors):
        assert torch.equal(a, b)
    captured.check()
