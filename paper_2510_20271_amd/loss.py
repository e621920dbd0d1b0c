"""Softmax cross entropy of a linear head, logits never kept, over the C ABI.

What a network does with the soft layer's curves [batch, T], or with the features of every voxel, is to score them
against classes: logits = hidden weight^T, then the cross entropy with a label for each row.  The logits would be the
largest tensor of the step (rows times classes); here they are formed in pieces of the classes, forward and backward.
``LinearCrossEntropy`` holds the head's weight, ``linear_cross_entropy`` is the functional form.

Inputs must live on the GPU; there is no CPU path.
"""
from __future__ import annotations

import math

import torch

from . import api
from .layer import _native_functions, _once, _plain


class LinearCrossEntropyFunction(torch.autograd.Function):
    """loss_i = log sum_v exp <hidden_i, weight_v> - <hidden_i, weight_label>, reduced; rows of ignore_index left out."""

    @staticmethod
    def forward(ctx, hidden, weight, labels, ignore_index: int, reduction: str):
        keep = any(ctx.needs_input_grad[:2])
        loss, stats, counted = api.ecc_xent_fwd(hidden.detach(), weight.detach(), labels, ignore_index, reduction, keep=keep)
        ctx.ignore_index, ctx.reduction = ignore_index, reduction
        if keep:
            ctx.save_for_backward(hidden, weight, labels, stats, counted)
        return loss

    @staticmethod
    @_once
    def backward(ctx, grad_loss):
        hidden, weight, labels, stats, counted = ctx.saved_tensors
        skip = [n for n, need in zip(("grad_hidden", "grad_weight"), ctx.needs_input_grad) if not need]
        with api._on_device_of(hidden):
            grads = api.ecc_xent_bwd(hidden, weight, labels, grad_loss.contiguous(), stats, counted, ctx.ignore_index,
                                     ctx.reduction, skip=skip)
        return *grads, None, None, None


def linear_cross_entropy(hidden, weight, labels, ignore_index: int = -100, reduction: str = "mean"):
    """hidden [..., dim] and weight [classes, dim] of one type (float32, float16 or bfloat16) on the GPU, labels [...]
    int64.  reduction "mean" (over the rows whose label is not ignore_index; 0 if there are none), "sum", or "none" (a
    loss for each label, 0 where it is ignore_index).  The loss is float32, and so are sums of products, the softmax and its
    gradient (held to twice the bits of a 16-bit type; float16: and to 2^-39 of the largest upstream gradient).  Any other label outside 0 .. classes - 1
    makes its row's loss and gradients NaN."""
    if not hidden.is_cuda or not weight.is_cuda or not labels.is_cuda:
        raise ValueError("hidden, weight and labels must be on the GPU")
    if not hidden.device == weight.device == labels.device:
        raise ValueError(f"tensors must be on one device, got {hidden.device}, {weight.device} and {labels.device}")
    api._one_of(api._REDUCTIONS, reduction, "reduction")
    api._one_of(api._OPERATOR_DTYPES, hidden.dtype, "the type of hidden")
    if hidden.dim() < 1 or weight.dim() != 2 or hidden.shape[-1] != weight.shape[1]:
        raise ValueError("hidden must be [..., dim] and weight [classes, dim]")
    if tuple(labels.shape) != tuple(hidden.shape[:-1]):
        raise ValueError(f"labels must have the shape {tuple(hidden.shape[:-1])}, got {tuple(labels.shape)}")
    if hidden.dtype != weight.dtype:
        raise ValueError(f"hidden and weight must have one type, got {hidden.dtype} and {weight.dtype}")
    if labels.dtype != torch.int64:
        raise ValueError(f"labels must be int64, got {labels.dtype}")
    if labels.numel() == 0:  # no row: no loss, gradients of zero
        nothing = (hidden.sum() * 0.0 + weight[:0].sum() * 0.0).float()
        return nothing if reduction != "none" else nothing + torch.zeros(labels.shape, device=hidden.device)
    rows = (hidden if hidden.dim() == 2 else hidden.reshape(-1, hidden.shape[-1])).contiguous()
    weight, flat = weight.contiguous(), labels.reshape(-1).contiguous()
    with api._on_device_of(hidden):
        if _plain(rows, weight, flat):
            loss = _native_functions().linear_xent(rows, weight, flat, int(ignore_index), api._REDUCTIONS[reduction])
        else:
            loss = LinearCrossEntropyFunction.apply(rows, weight, flat, int(ignore_index), reduction)
    return loss.reshape(labels.shape) if reduction == "none" else loss


class LinearCrossEntropy(torch.nn.Module):
    """A linear head without a bias and its cross entropy; weight [classes, dim]."""

    def __init__(self, classes: int, dim: int, ignore_index: int = -100, reduction: str = "mean",
                 dtype: torch.dtype = torch.float32):
        super().__init__()
        if classes < 1 or dim < 1:
            raise ValueError(f"classes and dim must be >= 1, got {classes} and {dim}")
        api._one_of(api._REDUCTIONS, reduction, "reduction")
        api._one_of(api._OPERATOR_DTYPES, dtype, "dtype")
        self.classes, self.dim, self.ignore_index, self.reduction = int(classes), int(dim), int(ignore_index), reduction
        self.weight = torch.nn.Parameter(torch.randn(classes, dim, dtype=torch.float32).mul_(1.0 / math.sqrt(dim)).to(dtype))

    def forward(self, hidden: torch.Tensor, labels: torch.Tensor) -> torch.Tensor:
        return linear_cross_entropy(hidden, self.weight, labels, self.ignore_index, self.reduction)
