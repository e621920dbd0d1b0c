"""Group normalisation with an activation for channels-last features, over the C ABI.

The soft layer takes its curves of a field [batch, (D,) H, W]; a network makes that field from features
[batch, (D,) H, W, channels], the same layout with the channels innermost, and this is the layer it is made of
between products.  The curves themselves, [batch, T], can be normalised over groups of thresholds the same way.
``GroupNormAct`` holds the scale and shift of every channel, ``group_norm_act`` is the functional form.

Inputs must live on the GPU; there is no CPU path.
"""
from __future__ import annotations

import torch

from . import api
from .layer import _native_functions, _once, _plain


class GroupNormActFunction(torch.autograd.Function):
    """y = act((x - mean) / sqrt(var + eps) * weight + bias), statistics over the points and channels of a group."""

    @staticmethod
    def forward(ctx, x, weight, bias, groups: int, eps: float, act: str):
        y, stats = api.ecc_norm_fwd(x.detach(), groups, weight, bias, eps, act, keep=any(ctx.needs_input_grad[:3]))
        ctx.groups, ctx.act = groups, act
        if stats is not None:
            ctx.save_for_backward(x, weight, bias, stats)
        return y

    @staticmethod
    @_once
    def backward(ctx, grad_y):
        x, weight, bias, stats = ctx.saved_tensors
        skip = [n for n, need in zip(("grad_x", "grad_weight", "grad_bias"), ctx.needs_input_grad) if not need]
        with api._on_device_of(x):
            grads = api.ecc_norm_bwd(x, grad_y.contiguous(), ctx.groups, stats, weight, bias, ctx.act, skip=skip)
        return *grads, None, None, None


def group_norm_act(x, groups: int, weight=None, bias=None, eps: float = 1e-5, act: str = "silu"):
    """x [batch, (D,) H, W, channels] or [batch, channels], float32, float16 or bfloat16 on the GPU; weight, bias
    [channels] or None; act "none", "relu" or "silu".  Statistics and parameters are float32 or better whatever the
    type of x; the result has the type of x."""
    if not x.is_cuda:
        raise ValueError("x must be on the GPU")
    if x.dim() < 2:
        raise ValueError("x must be [batch, (points,) channels]")
    channels = x.shape[-1]
    if channels < 1 or int(groups) < 1 or channels % int(groups):
        raise ValueError(f"groups must divide the {channels} channels, got {groups}")
    code = api._one_of(api._ACTS, act, "act")
    api._one_of(api._OPERATOR_DTYPES, x.dtype, "the type of x")
    for name, t in (("weight", weight), ("bias", bias)):
        if t is not None and tuple(t.shape) != (channels,):
            raise ValueError(f"{name} must have {channels} elements, got shape {tuple(t.shape)}")
        if t is not None and t.device != x.device:
            raise ValueError(f"{name} must be on {x.device}, got {t.device}")
    if x.numel() == 0:  # no item or no point: nothing to normalise, gradients of zero
        return x * 1.0 + sum(t.sum().to(x.dtype) * 0.0 for t in (weight, bias) if t is not None)
    weight = None if weight is None else weight.float().contiguous()
    bias = None if bias is None else bias.float().contiguous()
    x = x.contiguous()
    with api._on_device_of(x):
        if _plain(x, weight, bias):
            return _native_functions().norm_act(x, weight, bias, int(groups), float(eps), code)
        return GroupNormActFunction.apply(x, weight, bias, int(groups), float(eps), act)


class GroupNormAct(torch.nn.Module):
    """Group normalisation over channels-last features, a scale and a shift for every channel, an activation.

    groups must divide channels; affine=False leaves scale and shift out.
    """

    def __init__(self, groups: int, channels: int, eps: float = 1e-5, act: str = "silu", affine: bool = True):
        super().__init__()
        if groups < 1 or channels < 1 or channels % groups:
            raise ValueError(f"groups must divide the {channels} channels, got {groups}")
        api._one_of(api._ACTS, act, "act")
        self.groups, self.channels, self.eps, self.act = int(groups), int(channels), float(eps), act
        self.weight = torch.nn.Parameter(torch.ones(channels)) if affine else None
        self.bias = torch.nn.Parameter(torch.zeros(channels)) if affine else None

    def forward(self, x: torch.Tensor) -> torch.Tensor:
        if x.shape[-1] != self.channels:
            raise ValueError(f"x must have {self.channels} channels, got {x.shape[-1]}")
        return group_norm_act(x, self.groups, self.weight, self.bias, self.eps, self.act)
