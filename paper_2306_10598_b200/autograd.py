"""The training operators as differentiable torch functions: each forward call and its backward pass are the calls of
``api`` of the same name.  Gradients have their input's type; for gradients summed in fp32 over micro-batches call
``api.embed_backward`` and ``api.vocab_loss_backward`` with ``accumulate=True`` (as ``drop_train`` does)."""
from __future__ import annotations

import torch

from . import api


def _rows(t: torch.Tensor) -> torch.Tensor:
    """A tensor as the library takes it: gradients of a sum or a mean are one value seen many times, and the rows of a slice
    of sequences need not be evenly spaced."""
    return t.contiguous()


class _Embed(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, ids, scale, pad_id):
        ids = _rows(ids)
        ctx.save_for_backward(ids)
        ctx.rest = (table.shape[0], scale, pad_id)
        return api.embed(table, ids, scale, pad_id)

    @staticmethod
    def backward(ctx, dout):
        (ids,) = ctx.saved_tensors
        V, scale, pad_id = ctx.rest
        return api.embed_backward(_rows(dout), ids, V, scale, pad_id), None, None, None


class _Gelu(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x):
        y, q, scales = api.gelu_save8(_rows(x))
        ctx.save_for_backward(q, scales)
        return y

    @staticmethod
    def backward(ctx, dy):
        return api.gelu_save8_backward(_rows(dy), *ctx.saved_tensors)


class _VocabLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, hidden, weight, targets, ignore_index, logit_scale):
        hidden, targets = _rows(hidden), _rows(targets)
        loss, lse = api.vocab_loss(hidden, weight, targets, ignore_index, logit_scale)
        ctx.save_for_backward(hidden, weight, targets, lse)
        ctx.rest = (ignore_index, logit_scale)
        return loss

    @staticmethod
    def backward(ctx, dloss):
        hidden, weight, targets, lse = ctx.saved_tensors
        need_h, need_w = ctx.needs_input_grad[:2]
        dh, dw = api.vocab_loss_backward(hidden, weight, targets, lse, _rows(dloss), *ctx.rest, want_dhidden=need_h, want_dweight=need_w)
        return dh, dw, None, None, None


def embed(table: torch.Tensor, ids: torch.Tensor, scale: float = 1.0, pad_id: int = -1) -> torch.Tensor:
    return _Embed.apply(table, ids, scale, pad_id)


def gelu(x: torch.Tensor) -> torch.Tensor:
    """gelu that keeps its input in 8 bits."""
    return _Gelu.apply(x)


def vocab_loss(hidden: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, ignore_index: int = -100,
               logit_scale: float = 1.0) -> torch.Tensor:
    """The loss of each row, fp32 (0 where targets == ignore_index)."""
    return _VocabLoss.apply(hidden, weight, targets, ignore_index, logit_scale)
