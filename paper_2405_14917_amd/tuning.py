"""The step that tunes what stays above the low widths: the norm in front of an 8-bit head and, if wanted, the head itself, against a
full-precision teacher's top logits.  Only the order of the library's calls: the norm, the 8-bit linear layer, the divergence with its
gradient, and both backward passes."""
from __future__ import annotations

from typing import Optional

import torch

from . import binding


def workspace_query(vocabulary: int, width: int, tokens: int, dtype: torch.dtype = torch.bfloat16, bias: bool = True,
                    head_grad: bool = True, num_cus: int = 0) -> int:
    """Bytes of workspace of a HeadTuning with up to `tokens` tokens a call, for a context under graph capture."""
    return max(binding.fp8_linear_workspace(vocabulary, width, tokens, dtype, num_cus),
               binding.fp8_linear_backward_workspace(vocabulary, width, tokens, True, head_grad, torch.float32, num_cus),
               binding.layer_norm_backward_workspace(tokens, width, bias, dtype, num_cus),
               binding.distill_workspace(tokens, vocabulary, dtype))          # (each of them is enough for fewer tokens too)


class HeadTuning:
    """Norm (weight, bias or None; without the mean with `rms`) and 8-bit head W (vocabulary x width, 16 bits or fp32) on hidden states.
    Where a call is captured into a graph, change weight and bias in place between the replays; store() does so with the head."""

    def __init__(self, slim: binding.Slim, W: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
                 rms: bool = False, tau: float = 1.0):
        self.slim, self.weight, self.bias, self.eps, self.rms, self.tau = slim, weight, bias, eps, rms, tau
        self.q, self.s, self.qt, self.st = slim.fp8_quantize_weights(W)

    def store(self, W: torch.Tensor):
        """Takes new weights of the head, of the same shape, into the stored 8-bit form: in its place, where a captured graph reads it."""
        self.slim.fp8_quantize_weights(W, out=(self.q, self.s, self.qt, self.st))

    def logits(self, X: torch.Tensor) -> torch.Tensor:
        """Serving: the logits of hidden states X (t, width), one token or many."""
        return self.slim.fp8_linear(self.slim.layer_norm(X, self.weight, self.bias, self.eps, self.rms), self.q, self.s)

    def validate(self, X: torch.Tensor, index: torch.Tensor, teacher: torch.Tensor, lse: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The divergence from the teacher, token by token."""
        return self.slim.distill_loss(self.logits(X), index, teacher, self.tau, lse)

    def gradients(self, X: torch.Tensor, index: torch.Tensor, teacher: torch.Tensor, dloss: torch.Tensor, lse: Optional[torch.Tensor] = None,
                  head_grad: bool = True):
        """(loss per token, dict of the gradients of sum(dloss * loss)): X, weight, bias (None without one) and, with `head_grad`, head
        (float32, for the caller's copy of the weights in more bits)."""
        y, mean, rstd = self.slim.layer_norm(X, self.weight, self.bias, self.eps, self.rms, stats=True)
        S = self.slim.fp8_linear(y, self.q, self.s)
        loss, dS = self.slim.distill_loss_grad(S, index, teacher, dloss, self.tau, lse, dS=S)      # (in the logits' own memory)
        dy, dhead = self.slim.fp8_linear_backward(dS, y if head_grad else None, self.qt, self.st, torch.float32, dw=head_grad)
        dX, dweight, dbias = self.slim.layer_norm_backward(dy, X, self.weight, mean, rstd, bias=self.bias is not None)
        return loss, dict(X=dX, weight=dweight, bias=dbias, head=dhead)
