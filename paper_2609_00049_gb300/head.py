"""The LM head on 8-bit codes: a model's hidden states scored against the next
tokens (perplexity, entropy, alternatives) and the head's weight gradient.

    head = Head8(W)                      # W: vocab x d, bf16 or fp32
    step = head.forward(h, targets)      # h: tokens x d
    step.perplexity()
    dW = head.weight_grad(step, d_logprob)

The forward pass quantizes each hidden state to 8 bits
(realq_quantize_activations), multiplies the codes with the head's
(realq_int8_product) and scores the logits (realq_token_logprobs).  What it
keeps for the backward pass is the logits, the rows' normalisers and the hidden
states in 8 bits with a scale per 32 values (realq_checkpoint_pack); the
backward pass turns the logits into their gradient in place
(realq_token_logprobs_grad) and takes the weight gradient from the checkpoint
(realq_checkpoint_weight_grad).  The paper evaluates perplexities (Sec. 5) and
takes its Fisher from the gradient of the token log probabilities at the head
(App. "Pre-computation of the aggregated Fisher and last-transformer-block
handling"); it has no 8-bit head.  The logits are kept in bf16
(logits_dtype), whose rounding a perplexity of more than three digits shows;
torch.float32 avoids it.  Buffers are allocated with torch; no
arithmetic happens here beyond the mean of the scored log probabilities.
"""
from __future__ import annotations

import contextlib
from dataclasses import dataclass
from typing import Optional

import torch

from . import (realq_checkpoint_pack, realq_checkpoint_weight_grad, realq_checkpoint_weight_grad_workspace_size,
               realq_int8_product, realq_int8_product_workspace_size, realq_quantize_activations,
               realq_token_logprobs, realq_token_logprobs_grad, realq_workspace_status, workspace, _stream)


@dataclass
class HeadStep:
    """One forward pass: what it returns, and what the backward pass reads."""
    logprob: torch.Tensor                 # tokens
    entropy: torch.Tensor                 # tokens
    top_ids: Optional[torch.Tensor]       # tokens x k
    top_logprob: Optional[torch.Tensor]
    logits: Optional[torch.Tensor]        # tokens x vocab; the backward pass puts their gradient here
    norm: torch.Tensor                    # tokens x 2
    targets: torch.Tensor
    codes: torch.Tensor                   # the hidden states' checkpoint
    exps: torch.Tensor
    stream: Optional[torch.cuda.Stream] = None   # the pass's
    head: Optional["Head8"] = None

    def perplexity(self) -> float:
        """exp of minus the mean log probability of the scored tokens (synchronizes).
        Raises RealqError if a pass of the head since its last check gave up."""
        if self.stream is not None:
            current = torch.cuda.current_stream(self.logprob.device)
            if current != self.stream:
                current.wait_stream(self.stream)
        if self.head is not None:
            self.head.check()
        scored = self.targets >= 0
        return float(torch.exp(-self.logprob[scored].double().mean()))


_HERE = contextlib.nullcontext()


def _used_on(stream, *tensors: Optional[torch.Tensor]) -> None:
    """Keep the tensors' memory from being handed on before `stream` is done with it."""
    for t in tensors:
        if t is not None:
            t.record_stream(stream)


class Head8:
    """An LM head of 8-bit channel codes with one scale per output token.

    Any stream: a pass on a stream other than the current one (`stream`) starts
    after what the current stream holds and takes its memory from its own
    stream; its results are there once that stream has run, and the current
    stream has to wait for it before it reads them, as with any operator.  The
    head's workspaces are reused from call to call, so its passes run one after
    the other, whatever their streams."""

    def __init__(self, W: torch.Tensor, logits_dtype=torch.bfloat16):
        self.vocab, self.d = W.shape
        self.logits_dtype = logits_dtype
        self.codes = torch.empty((self.vocab, self.d), dtype=torch.uint8, device=W.device)
        self.scale = torch.empty(self.vocab, dtype=torch.float32, device=W.device)
        realq_quantize_activations(W, 8, 1.0, codes=self.codes, scale=self.scale)   # a row's symmetric 8-bit grid
        self._ws = {}
        self._stream = torch.cuda.current_stream(W.device)   # the latest pass's
        self._handle = self._stream.cuda_stream

    def _workspace(self, key: str, nbytes: int, device) -> Optional[torch.Tensor]:
        have = self._ws.get(key)
        if have is None or have.numel() < nbytes:
            new = workspace(nbytes, device)
            if have is not None:
                new[:4].copy_(have[:4])   # the status word
            self._ws[key] = have = new
        return have

    def _begin(self, stream):
        """A pass on `stream` (None: the current one) begins: after the caller's
        work and the head's latest pass.  The stream for the pass's operators, and
        the caller's where that is another (the pass is then run with its own
        current, so that allocations belong to it)."""
        handle = _stream(stream)
        if handle == self._handle and (stream is None or handle == _stream(None)):
            return stream, None   # (nothing to order; making stream objects would take as long as a small kernel)
        caller = torch.cuda.current_stream(self.codes.device)
        s = caller if stream is None else stream
        if handle != self._handle:
            s.wait_stream(self._stream)
            _used_on(s, self.codes, self.scale, *self._ws.values())
            self._stream, self._handle = s, handle
        if s == caller:
            return s, None
        s.wait_stream(caller)
        return s, caller

    def check(self) -> None:
        """Raises RealqError if a bounded wait gave up in a pass since the last
        check, whose results then hold NaN (synchronizes)."""
        s, _ = self._begin(None)
        for ws in self._ws.values():
            if ws is not None:
                realq_workspace_status(ws, stream=s)

    def forward(self, h: torch.Tensor, targets: torch.Tensor, k: int = 0, stream=None) -> HeadStep:
        """Score the next tokens (negative targets are not scored) with the k
        likeliest alternatives of each position."""
        T, dev = h.shape[0], h.device
        new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=dev)  # noqa: E731
        s, caller = self._begin(stream)
        with _HERE if caller is None else torch.cuda.stream(s):
            if caller is not None:
                _used_on(s, h, targets)
            xc, xs = new(T, self.d, dtype=torch.uint8), new(T)
            realq_quantize_activations(h, 8, 1.0, codes=xc, scale=xs, stream=s)
            logits = new(T, self.vocab, dtype=self.logits_dtype)
            ws = self._workspace("product", realq_int8_product_workspace_size(T, self.d, self.vocab), dev)
            realq_int8_product(xc, xs, self.codes, self.scale, logits, ws=ws, stream=s)
            out = dict(logprob=new(T), norm=new(T, 2), entropy=new(T),
                       top_ids=new(T, k, dtype=torch.int64) if k else None, top_logprob=new(T, k) if k else None)
            realq_token_logprobs(logits, targets, **out, stream=s)
            codes, exps = new(T, self.d, dtype=torch.int8), new(T, (self.d + 31) // 32, dtype=torch.uint8)
            realq_checkpoint_pack(h, codes, exps, stream=s)
            if caller is not None:
                _used_on(caller, logits, codes, exps, *out.values())
        return HeadStep(**out, logits=logits, targets=targets, codes=codes, exps=exps, stream=self._stream, head=self)

    def weight_grad(self, step: HeadStep, d_logprob: torch.Tensor, d_entropy: Optional[torch.Tensor] = None,
                    dW: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """dL/dW of the head for a loss with the given derivatives with respect to
        the log probabilities (and entropies), added to dW where it is given.
        The step's logits become their gradient: a step takes one backward pass."""
        if step.logits is None:
            raise ValueError("this step's logits have been used by a backward pass")
        T, dev = step.codes.shape[0], step.codes.device
        for name, t, shape in (("d_logprob", d_logprob, (T,)), ("d_entropy", d_entropy, (T,)),
                               ("dW", dW, (self.vocab, self.d))):   # before the logits are used up
            if t is not None and (t.dtype != torch.float32 or t.shape != shape or t.device != dev
                                  or not t.is_contiguous()):
                raise ValueError(f"{name}: expected a contiguous float32 tensor of shape {shape} on {dev}, got "
                                 f"{t.dtype} {tuple(t.shape)} on {t.device}")
        d_logits, step.logits = step.logits, None
        s, caller = self._begin(stream)
        with _HERE if caller is None else torch.cuda.stream(s):
            if caller is not None:
                _used_on(s, step.targets, d_logprob, d_entropy, dW)
            if self._stream is not step.stream:
                _used_on(self._stream, d_logits, step.targets, step.norm, step.entropy, step.codes, step.exps)
            realq_token_logprobs_grad(d_logits, step.targets, step.norm, d_logits, d_logprob=d_logprob,
                                      entropy=step.entropy if d_entropy is not None else None, d_entropy=d_entropy,
                                      stream=s)
            accumulate = dW is not None
            if dW is None:
                dW = torch.empty((self.vocab, self.d), dtype=torch.float32, device=dev)
                if caller is not None:
                    _used_on(caller, dW)
            ws = self._workspace("grad", realq_checkpoint_weight_grad_workspace_size(T, self.vocab, self.d,
                                                                                     d_logits.dtype), dev)
            return realq_checkpoint_weight_grad(d_logits, step.codes, step.exps, dW, accumulate=accumulate, ws=ws,
                                                stream=s)
