"""The steps that tune what stays above the low widths.  HeadTuning: the norm in front of an 8-bit head and, if wanted, the head itself, against a
full-precision teacher's top logits.  BlockTuning: a feed-forward block kept in 8 bits and the head behind it, against labels.  Only the order
of the library's calls: norms, 8-bit linear layers, a loss with its gradient, the backward passes, the clipping of the gradients."""
from __future__ import annotations

from typing import Optional, Tuple

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


def block_workspace_query(vocabulary: int, width: int, inner: int, tokens: int, dtype: torch.dtype = torch.bfloat16, num_cus: int = 0) -> int:
    """Bytes of workspace of a BlockTuning with up to `tokens` tokens a call, for a context under graph capture."""
    f32 = torch.float32
    return max(binding.fp8_linear_act_workspace(inner, width, tokens, True, dtype, num_cus),
               binding.fp8_linear_act_workspace(width, inner, tokens, False, dtype, num_cus),
               binding.fp8_linear_act_backward_workspace(inner, width, tokens, True, True, f32, True, num_cus),
               binding.fp8_linear_act_backward_workspace(width, inner, tokens, True, True, f32, True, num_cus),
               binding.head_loss_grad_workspace(vocabulary, width, tokens, True, True, f32, num_cus),
               binding.head_loss_workspace(vocabulary, width, tokens, num_cus),
               binding.fp8_linear_workspace(vocabulary, width, tokens, f32, num_cus),
               binding.layer_norm_backward_workspace(tokens, width, True, dtype, num_cus),
               binding.grad_norm_workspace(12, num_cus))


class BlockTuning:
    """The last feed-forward block of a model, in 8 bits, and the head behind it:

        h = x + r,  u = act(norm1(h) Up^T + up_bias),  h' = h + u Down^T + down_bias,  logits = norm2(h') Head^T

    Up (inner x width), Down (width x inner) and Head (vocabulary x width) of 16 bits or fp32; norm1, norm2 and the biases: (weight, bias or None) and
    vectors or None, of the activations' type or fp32.  Where a call is captured into a graph, change the vectors in place; store() does so with the
    matrices."""

    def __init__(self, slim: binding.Slim, up: torch.Tensor, down: torch.Tensor, head: torch.Tensor,
                 norm1: Tuple[torch.Tensor, Optional[torch.Tensor]], norm2: Tuple[torch.Tensor, Optional[torch.Tensor]],
                 up_bias: Optional[torch.Tensor] = None, down_bias: Optional[torch.Tensor] = None, act: str = "silu", eps: float = 1e-5,
                 rms: bool = False):
        self.slim, self.norm1, self.norm2, self.up_bias, self.down_bias = slim, norm1, norm2, up_bias, down_bias
        self.act, self.eps, self.rms = act, eps, rms
        self.up, self.down, self.head = (slim.fp8_quantize_weights(W) for W in (up, down, head))

    def store(self, up: Optional[torch.Tensor] = None, down: Optional[torch.Tensor] = None, head: Optional[torch.Tensor] = None):
        """Takes new matrices, of the same shapes, into the stored 8-bit forms, in their places."""
        for W, place in ((up, self.up), (down, self.down), (head, self.head)):
            if W is not None:
                self.slim.fp8_quantize_weights(W, out=place)

    def hidden(self, X: torch.Tensor, R: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Serving: h' of one token or many, from the stream R and what the layer before adds to it, X."""
        s, n = self.slim, self.slim.add_norm(X, R, *self.norm1, eps=self.eps, rms=self.rms, y=False, e4m3=True)
        u = s.fp8_linear_act((n.q, n.s), *self.up[:2], self.up_bias, self.act, dtype=X.dtype)
        return s.fp8_linear_act(u, *self.down[:2], self.down_bias, residual=n.H)

    def logits(self, X: torch.Tensor, R: Optional[torch.Tensor] = None) -> torch.Tensor:
        n = self.slim.add_norm(self.hidden(X, R), None, *self.norm2, eps=self.eps, rms=self.rms, y=False, e4m3=True)
        return self.slim.fp8_linear_act((n.q, n.s), *self.head[:2], dtype=torch.float32)

    def validate(self, X: torch.Tensor, R: Optional[torch.Tensor], labels: torch.Tensor) -> torch.Tensor:
        """The cross entropy of the labels, token by token."""
        n = self.slim.add_norm(self.hidden(X, R), None, *self.norm2, eps=self.eps, rms=self.rms)
        return self.slim.head_loss(n.Y, *self.head[:2], labels)

    def gradients(self, X: torch.Tensor, R: Optional[torch.Tensor], labels: torch.Tensor, dloss: torch.Tensor, limit: float = float("inf")):
        """(loss per token, dict of the gradients of sum(dloss * loss), their norm): X (and R alike), norm1, norm2 (weight, bias or None), up, down,
        head (float32, for the caller's copies in more bits), up_bias, down_bias (None without one).  Those of the parameters are scaled to
        `limit` together; the norm is the one before."""
        s, norm = self.slim, dict(eps=self.eps, rms=self.rms, stats=True)
        f32 = torch.float32
        n1 = s.add_norm(X, R, *self.norm1, e4m3=True, **norm)
        U, Z = s.fp8_linear_act((n1.q, n1.s), *self.up[:2], self.up_bias, self.act, dtype=X.dtype, keep=True)
        with torch.no_grad():                     # (the step's gradients are its results)
            H = s.fp8_linear_act(U, *self.down[:2], self.down_bias, residual=n1.H)
        n2 = s.add_norm(H, None, *self.norm2, **norm)
        loss, dY2, dhead = s.head_loss_grad(n2.Y, *self.head, labels, dloss, f32)
        dH, dw2, db2 = s.add_norm_backward(dY2, None, H, self.norm2[0], n2.mean, n2.rstd, bias=self.norm2[1] is not None)
        like = lambda b: None if b is None else b.dtype
        dU, ddown, ddown_bias = s.fp8_linear_act_backward(dH, None, None, U, *self.down[2:], f32, db_dtype=like(self.down_bias))
        dY1, dup, dup_bias = s.fp8_linear_act_backward(dU, Z, self.act, n1.Y, *self.up[2:], f32, db_dtype=like(self.up_bias))
        dX, dw1, db1 = s.add_norm_backward(dY1, dH, n1.H, self.norm1[0], n1.mean, n1.rstd, bias=self.norm1[1] is not None)
        grads = dict(norm1=(dw1, db1), norm2=(dw2, db2), up=dup, down=ddown, head=dhead, up_bias=dup_bias, down_bias=ddown_bias)
        of_all = s.clip_gradients([g for g in (dw1, db1, dw2, db2, dup, ddown, dhead, dup_bias, ddown_bias) if g is not None], limit)
        return loss, dict(grads, X=dX), of_all
