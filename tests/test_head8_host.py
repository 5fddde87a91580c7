"""The LM head on 8-bit codes, its order of work and its refusals, without a GPU:
the operators and torch's streams are stood in for by recorders."""
import contextlib

import pytest
import torch

from paper_2609_00049_gb300 import head as head_module


class FakeEvent:
    def __init__(self):
        self.after = None

    def record(self, stream):
        self.after = (stream, len(stream.log))


class FakeStream:
    def __init__(self, name, log):
        self.name, self.log, self.cuda_stream = name, log, hash(name)

    def wait_stream(self, other):
        self.log.append(("wait_stream", self.name, other.name))

    def wait_event(self, event):
        self.log.append(("wait_event", self.name, event.after[0].name))

    def record_event(self, event=None):
        event = event or FakeEvent()
        event.record(self)
        return event


@pytest.fixture
def world(monkeypatch):
    """Streams `main` and `side`, `main` current; a log of waits, allocations,
    operator calls (with the stream that was current and the stream they ran on)
    and recorded uses."""
    log = []
    main, side = FakeStream("main", log), FakeStream("side", log)
    current = [main]

    @contextlib.contextmanager
    def on(stream):
        current.append(stream)
        yield
        current.pop()

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current[-1])
    monkeypatch.setattr(torch.cuda, "Event", FakeEvent)
    monkeypatch.setattr(head_module, "_stream", lambda s: (s or current[-1]).cuda_stream, raising=False)
    monkeypatch.setattr(torch.Tensor, "record_stream",
                        lambda t, s: log.append(("record", id(t), s.name)), raising=False)
    keep = []   # tensors stay alive, so that an id names one of them

    def allocates(fn):
        def call(*a, **k):
            t = fn(*a, **k)
            log.append(("alloc", id(t), current[-1].name))
            keep.append(t)
            return t
        return call

    monkeypatch.setattr(torch, "empty", allocates(torch.empty))
    monkeypatch.setattr(head_module, "workspace",
                        allocates(lambda nbytes, device=None: torch.zeros(int(nbytes), dtype=torch.uint8)))

    def operator(name, result=None):
        def call(*a, stream=None, **k):
            log.append(("op", name, (stream or current[-1]).name))
            return a[result] if result is not None else None
        return call

    monkeypatch.setattr(head_module, "realq_quantize_activations", operator("quantize"))
    monkeypatch.setattr(head_module, "realq_int8_product", operator("product"))
    monkeypatch.setattr(head_module, "realq_token_logprobs", operator("logprobs"))
    monkeypatch.setattr(head_module, "realq_token_logprobs_grad", operator("logprobs_grad"))
    monkeypatch.setattr(head_module, "realq_checkpoint_pack", operator("pack"))
    monkeypatch.setattr(head_module, "realq_workspace_status", operator("status"), raising=False)
    monkeypatch.setattr(head_module, "realq_checkpoint_weight_grad", operator("weight_grad", result=3))
    monkeypatch.setattr(head_module, "realq_int8_product_workspace_size", lambda T, n, m: 256 * T)
    monkeypatch.setattr(head_module, "realq_checkpoint_weight_grad_workspace_size", lambda T, m, n, dt: 256 * T)
    return main, side, log


def kept(log, t, stream):
    """The allocator does not hand t's memory on while `stream` may use it: it
    belongs to that stream or its use there has been recorded."""
    return ("alloc", id(t), stream) in log or ("record", id(t), stream) in log


def waits(log, stream, other):
    return ("wait_stream", stream, other) in log or ("wait_event", stream, other) in log


def results(step):
    return [step.logprob, step.entropy, step.top_ids, step.top_logprob, step.logits, step.norm, step.codes, step.exps]


def test_a_head_on_another_stream_is_ordered_and_keeps_its_memory(world):
    """Everything that a pass on a side stream allocates belongs to that stream;
    the side stream waits for the caller's and for the stream that made the head
    before its first kernel; what crosses streams is recorded, so that the
    allocator hands nothing of it on while it is in use."""
    main, side, log = world
    head = head_module.Head8(torch.zeros(12, 8))
    h, y, g = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    built = len(log)
    step = head.forward(h, y, k=2, stream=side)
    done = len(log)
    first = next(i for i in range(built, done) if log[i][0] in ("op", "alloc"))
    assert waits(log[built:first], "side", "main")
    assert {e[2] for e in log[built:done] if e[0] == "op"} == {"side"}
    assert {e[2] for e in log[built:done] if e[0] == "alloc"} == {"side"}
    for t in (h, y, head.codes, head.scale, head._ws["product"]):
        assert kept(log[built:done], t, "side")
    for t in results(step):
        assert kept(log[built:done], t, "main")

    logits = step.logits
    dW = head.weight_grad(step, g, stream=side)
    assert {e[2] for e in log[done:] if e[0] == "op"} == {"side"}
    assert {e[2] for e in log[done:] if e[0] == "alloc"} == {"side"}
    first = next(i for i in range(done, len(log)) if log[i][0] in ("op", "alloc"))
    assert waits(log[done:first], "side", "main")
    for t in (g, y, logits, step.norm, step.codes, step.exps, head._ws["grad"]):
        assert kept(log, t, "side")
    assert kept(log[done:], dW, "main")


def test_a_head_used_on_two_streams_orders_its_workspaces(world):
    """A second pass on another stream waits for the first one's use of the
    shared workspaces, and a workspace that is replaced has been recorded."""
    main, side, log = world
    head = head_module.Head8(torch.zeros(12, 8))
    head.forward(torch.zeros(2, 8), torch.zeros(2, dtype=torch.int64), stream=side)
    old, at = head._ws["product"], len(log)
    assert kept(log, old, "side")
    step = head.forward(torch.zeros(9, 8), torch.zeros(9, dtype=torch.int64))   # larger: the workspace is replaced
    first = next(i for i in range(at, len(log)) if log[i][0] == "op")
    assert waits(log[at:first], "main", "side")
    assert head._ws["product"] is not old and kept(log, old, "main")
    assert {e[2] for e in log[at:] if e[0] == "op"} == {"main"}
    at = len(log)
    logits = step.logits
    head.weight_grad(step, torch.zeros(9), stream=side)
    first = next(i for i in range(at, len(log)) if log[i][0] == "op")
    assert waits(log[at:first], "side", "main")
    for t in (logits, step.norm, step.codes, step.exps):   # (the forward pass was on main)
        assert kept(log, t, "side")


def test_perplexity_waits_for_the_pass(world):
    main, side, log = world
    head = head_module.Head8(torch.zeros(12, 8))
    step = head.forward(torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64), stream=side)
    at = len(log)
    step.perplexity()
    assert waits(log[at:], "main", "side")


def test_a_refused_backward_pass_keeps_the_logits():
    """A backward pass whose arguments are refused has not used the step's
    logits: it can be called again with the right ones."""
    head = head_module.Head8.__new__(head_module.Head8)   # (no GPU: the fields that the checks read)
    head.vocab, head.d = 12, 8
    head.codes, head.scale, head._handle = torch.zeros(12, 8, dtype=torch.uint8), torch.zeros(12), 0
    logits, f = torch.zeros(4, 12), torch.zeros(4)
    step = head_module.HeadStep(f, f, None, None, logits, torch.zeros(4, 2), torch.zeros(4, dtype=torch.int64),
                                torch.zeros(4, 8, dtype=torch.int8), torch.zeros(4, 1, dtype=torch.uint8))
    for bad in (dict(d_logprob=torch.zeros(5)), dict(d_logprob=torch.zeros(4, dtype=torch.float64)),
                dict(d_logprob=f, d_entropy=torch.zeros(3)), dict(d_logprob=f, dW=torch.zeros(12, 9)),
                dict(d_logprob=f, dW=torch.zeros(12, 8, dtype=torch.bfloat16)),
                dict(d_logprob=f, dW=torch.zeros(8, 12).t())):
        with pytest.raises(ValueError):
            head.weight_grad(step, **bad)
        assert step.logits is logits


def test_passes_on_the_callers_own_stream_add_no_waits(world):
    main, side, log = world
    head = head_module.Head8(torch.zeros(12, 8))
    step = head.forward(torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64), k=2)
    head.weight_grad(step, torch.zeros(4), stream=main)
    assert {e[0] for e in log} == {"alloc", "op"}
