"""What torch's differentiation does with the training operators: linear and group_norm record themselves where an
input requires a gradient, and their gradients are linear_backward and group_norm_backward. First derivatives only."""
from __future__ import annotations

import torch
from torch.autograd.function import once_differentiable

from . import train_ops as T


class Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, act, residual, save):
        y, z = T.linear(x, weight, bias, act, residual, True)
        ctx.act, ctx.bias_shape = act, None if bias is None else bias.shape
        ctx.save_for_backward(x, weight, z)
        if z is None or not save:
            return y
        ctx.mark_non_differentiable(z)
        return y, z

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, *_):
        x, weight, z = ctx.saved_tensors
        need_x, need_w, need_b, _, need_r, _ = ctx.needs_input_grad
        dx = dw = db = None
        if need_x or need_w or need_b:
            g = dy if dy.shape[1] <= 1 or dy.stride(1) == 1 else dy.contiguous()
            dx, dw, db = T.linear_backward(g, x, weight, z, ctx.act, need=(need_x, need_w, need_b))
        return dx, dw, None if db is None else db.view(ctx.bias_shape), None, dy if need_r else None, None


class GroupNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, groups, weight, bias, eps, act):
        y, mean, rstd = T.group_norm(x, groups, weight, bias, eps, act)
        ctx.groups, ctx.act = groups, act
        ctx.save_for_backward(x, mean, rstd, weight, bias)
        ctx.mark_non_differentiable(mean, rstd)
        return y, mean, rstd

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, *_):
        x, mean, rstd, weight, bias = ctx.saved_tensors
        need_x, _, need_w, need_b, _, _ = ctx.needs_input_grad
        dx, dw, db = T.group_norm_backward(dy.contiguous(), x, mean, rstd, ctx.groups, weight, bias, ctx.act)
        return dx if need_x else None, None, dw.view(weight.shape) if need_w else None, db.view(bias.shape) if need_b else None, None, None
