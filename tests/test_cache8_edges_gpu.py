"""What Cache8 does with errors, refusals, streams and the host's time."""
import pytest
import torch

import paper_2609_00049_gb300 as rq
from kv_reference import gen

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2609_00049_gb300 import build as b
    b.build()
    rq.lib()


def caches(n, **kw):
    from paper_2609_00049_gb300.cache import Cache8
    return [Cache8(2, 40, 3, 300, 2, 64, page_size=16, **kw) for _ in range(n)]


def tokens(T, seed, dtype=torch.bfloat16):
    return [torch.randn(T, n, 64, generator=gen(seed + i), device="cuda").to(dtype) for i, n in enumerate((8, 2, 2))]


TIMEOUT_BIT, NO_PAGES_BIT = 4, 8      # of a workspace's status word


def test_going_on_after_a_wait_that_gave_up():
    """A status and arrival counters as a call that gave up leaves them: check raises once, and what follows is as in a
    cache that never saw it."""
    bad, good = caches(2)
    for c in (bad, good):
        step = c.begin([250, 100, 33])
        c.attend(step, 0, *tokens(383, 1))
    torch.cuda.synchronize()
    # (those of the kernel of few rows begin 256 bytes behind the status)
    bad._attend_ws.view(torch.int32)[64:128] = 30          # (of a join of some 50 shares)
    bad._attend_ws.view(torch.int32)[0] = TIMEOUT_BIT
    with pytest.raises(rq.RealqError) as e:
        bad.check()
    assert e.value.status == rq.REALQ_ERR_TIMEOUT
    bad.check()
    for i, counts in enumerate([[1, 1, 1], [2, 0, 20], [1, 1, 1]]):
        got, want = (c.attend(c.begin(counts), 0, *tokens(sum(counts), 10 + i)) for c in (bad, good))
        assert torch.equal(got, want), counts
    bad.check()


def test_check_reports_both_errors():
    """Too few pages and a wait that gave up since the last check: both are raised, and nothing is left behind."""
    c, = caches(1)
    c._pages_ws.view(torch.int32)[0] = NO_PAGES_BIT
    c._attend_ws.view(torch.int32)[0] = TIMEOUT_BIT
    with pytest.raises(rq.RealqError) as e:
        c.check()
    assert e.value.status == rq.REALQ_ERR_TIMEOUT and e.value.__cause__.status == rq.REALQ_ERR_NO_PAGES
    c.check()
    assert not bool(c._attend_ws.any())
    c._pages_ws.view(torch.int32)[0] = NO_PAGES_BIT
    with pytest.raises(rq.RealqError) as e:
        c.check()
    assert e.value.status == rq.REALQ_ERR_NO_PAGES
    c.check()


def test_a_refused_attend_changes_nothing():
    """Whatever attend refuses, q and k are not turned and nothing is cached."""
    c, = caches(1)
    step = c.begin([5, 1, 0])
    q, k, v = tokens(6, 3)
    before = [t.clone() for t in (q, k, *c.cache.tensors)]
    out = torch.empty_like(q)
    for bad in (dict(layer=2), dict(layer=-1), dict(v=v[:5]), dict(v=v.float()), dict(v=v.cpu()), dict(v=v[:, :1].expand(6, 2, 64)), dict(v=v[:, :1]),
                dict(k=k[:, :1].contiguous()), dict(q=q[:, :7]), dict(out=out[:5]), dict(out=out.float()), dict(out=out.cpu()),
                dict(lse=torch.empty(6, 7, device="cuda")), dict(lse=torch.empty(6, 8, device="cuda", dtype=torch.float64)),
                dict(window=-1), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=q[:5])):
        a = dict(layer=0, q=q, k=k, v=v) | bad
        with pytest.raises((ValueError, rq.RealqError)):
            c.attend(step, a.pop("layer"), a.pop("q"), a.pop("k"), a.pop("v"), **a)
        for t, want in zip((q, k, *c.cache.tensors), before):
            assert torch.equal(t, want), bad
    c.attend(step, 0, q, k, v, out=out, lse=torch.empty(6, 8, device="cuda"), window=3, scale=0.2)
    assert bool(torch.isfinite(out.float()).all())


def test_steps_do_not_wait_for_the_gpu():
    """begin, fork and release return while what was enqueued before them is still running."""
    c, = caches(1)
    calls = [lambda: c.begin([3, 1, 0]), lambda: c.fork([0], [2]), lambda: c.release([1])]
    for _ in range(2):                   # (host memory, kernels and streams are there)
        for f in calls:
            f()
    torch.cuda.synchronize()
    done = torch.cuda.Event()
    torch.cuda._sleep(2 * 10 ** 9)       # about a second
    done.record()
    for f in calls:
        f()
    waited = done.query()
    torch.cuda.synchronize()
    assert not waited
    assert c.lengths.tolist() == [9, 0, 9]


def test_a_captured_token_on_a_stream_given_by_name():
    """attend captured with `stream` the stream that is being captured."""
    eager, captured = caches(2)
    for c in (eager, captured):
        c.begin([20, 7, 1])
    steps = [c.begin([1, 1, 1]) for c in (eager, captured)]
    x = tokens(3, 5)
    buf, out = [t.clone() for t in x], torch.empty(3, 8, 64, device="cuda", dtype=torch.bfloat16)
    want = eager.attend(steps[0], 1, *[t.clone() for t in x])
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        captured.attend(steps[1], 1, *buf, out=out, stream=side)
    g.replay()
    assert torch.equal(out, want)


def test_a_step_of_another_stream_keeps_its_memory():
    """Two steps at a time, the first from another stream: its lists are not handed on while attention on this one reads them."""
    c, = caches(1)
    side = torch.cuda.Stream()
    c.begin([5, 0, 0])
    for warm in (True, False):           # (a kernel's first launch waits for the GPU)
        first = c.begin([3, 0, 0], stream=side)
        second = c.begin([0, 4, 0])
        x, y = tokens(3, 1), tokens(4, 9)
        torch.cuda.synchronize()
        held, done = {first.starts.data_ptr(), first.positions.data_ptr()}, torch.cuda.Event()
        if not warm:
            torch.cuda._sleep(2 * 10 ** 9)           # about a second
        done.record()
        c.attend(second, 0, *y)
        c.attend(first, 0, *x)
        del first
        with torch.cuda.stream(side):
            new = [torch.empty(4, dtype=torch.int32, device="cuda") for _ in range(200)]
        handed_on, waited = held & {t.data_ptr() for t in new}, done.query()
        torch.cuda.synchronize()
        if not warm:
            assert not waited and not handed_on
        del new
