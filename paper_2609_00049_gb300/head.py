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
handling"); it has no 8-bit head.  Buffers are allocated with torch; no
arithmetic happens here beyond the mean of the scored log probabilities.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Optional

import torch

from . import (realq_checkpoint_pack, realq_checkpoint_weight_grad, realq_checkpoint_weight_grad_workspace_size,
               realq_int8_product, realq_int8_product_workspace_size, realq_quantize_activations,
               realq_token_logprobs, realq_token_logprobs_grad, workspace)


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

    def perplexity(self) -> float:
        """exp of minus the mean log probability of the scored tokens (synchronizes)."""
        scored = self.targets >= 0
        return float(torch.exp(-self.logprob[scored].double().mean()))


class Head8:
    """An LM head of 8-bit channel codes with one scale per output token.  Its
    workspaces are reused from call to call, so use one stream at a time."""

    def __init__(self, W: torch.Tensor, logits_dtype=torch.bfloat16):
        self.vocab, self.d = W.shape
        self.logits_dtype = logits_dtype
        self.codes = torch.empty((self.vocab, self.d), dtype=torch.uint8, device=W.device)
        self.scale = torch.empty(self.vocab, dtype=torch.float32, device=W.device)
        realq_quantize_activations(W, 8, 1.0, codes=self.codes, scale=self.scale)   # a row's symmetric 8-bit grid
        self._ws = {}

    def _workspace(self, key: str, nbytes: int, device) -> Optional[torch.Tensor]:
        have = self._ws.get(key)
        if have is None or have.numel() < nbytes:
            self._ws[key] = have = workspace(nbytes, device)
        return have

    def forward(self, h: torch.Tensor, targets: torch.Tensor, k: int = 0, stream=None) -> HeadStep:
        """Score the next tokens (negative targets are not scored) with the k
        likeliest alternatives of each position."""
        T, dev = h.shape[0], h.device
        new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device=dev)  # noqa: E731
        xc, xs = new(T, self.d, dtype=torch.uint8), new(T)
        realq_quantize_activations(h, 8, 1.0, codes=xc, scale=xs, stream=stream)
        logits = new(T, self.vocab, dtype=self.logits_dtype)
        ws = self._workspace("product", realq_int8_product_workspace_size(T, self.d, self.vocab), dev)
        realq_int8_product(xc, xs, self.codes, self.scale, logits, ws=ws, stream=stream)
        step = HeadStep(new(T), new(T), new(T, k, dtype=torch.int64) if k else None, new(T, k) if k else None, logits,
                        new(T, 2), targets, new(T, self.d, dtype=torch.int8),
                        new(T, (self.d + 31) // 32, dtype=torch.uint8))
        realq_token_logprobs(logits, targets, step.logprob, step.norm, step.entropy, step.top_ids, step.top_logprob,
                             stream=stream)
        realq_checkpoint_pack(h, step.codes, step.exps, stream=stream)
        return step

    def weight_grad(self, step: HeadStep, d_logprob: torch.Tensor, d_entropy: Optional[torch.Tensor] = None,
                    dW: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """dL/dW of the head for a loss with the given derivatives with respect to
        the log probabilities (and entropies), added to dW where it is given.
        The step's logits become their gradient: a step takes one backward pass."""
        if step.logits is None:
            raise ValueError("this step's logits have been used by a backward pass")
        T, dev = step.codes.shape[0], step.codes.device
        d_logits, step.logits = step.logits, None
        realq_token_logprobs_grad(d_logits, step.targets, step.norm, d_logits, d_logprob=d_logprob,
                                  entropy=step.entropy if d_entropy is not None else None, d_entropy=d_entropy,
                                  stream=stream)
        accumulate = dW is not None
        if dW is None:
            dW = torch.empty((self.vocab, self.d), dtype=torch.float32, device=dev)
        ws = self._workspace("grad", realq_checkpoint_weight_grad_workspace_size(T, self.vocab, self.d, d_logits.dtype),
                             dev)
        return realq_checkpoint_weight_grad(d_logits, step.codes, step.exps, dW, accumulate=accumulate, ws=ws,
                                            stream=stream)
