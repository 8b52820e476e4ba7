"""The operators of `head` with autograd, and a box head on them (MMDetection, arXiv 1906.07155,
§3.1 RoIHead, §3.2 losses).

`linear_act` and `class_logprob` wire the kernels into torch.autograd, and `BoxHead` takes what
roi_extract gives for each RoI through two shared dense layers to class scores and box deltas:

    head = BoxHead(256 * 7 * 7, classes=80).cuda()
    scores, deltas = head(rois_features)            # [K, 81], [K, 320]
    loss = head.loss(scores, labels)                # mean of -log p over the labels that count
    logp, classes = head.best(scores, 5)            # per RoI: the five likeliest classes

There are no second and no forward-mode derivatives: they are refused.

All of it can be captured into a HIP graph.  A captured `backward()` needs leaves of which no eager graph
lives any more (torch accumulates their gradients on that graph's stream); torch.autograd.grad does not.
"""
from __future__ import annotations

import torch
from torch import nn
from torch.nn.modules import module as modules

from . import head as ops
from .relation_head import differentiated, once


def _rows(x):
    """[..., columns] as rows with adjacent columns."""
    x = x if x.dim() == 2 else x.reshape(-1, x.shape[-1])
    return x if x.stride(1) == 1 or x.shape[1] == 1 else x.contiguous()


class LinearActFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, residual, act):
        y, saved = ops.linear_act_fwd(x, weight, bias, act=act, residual=residual, save=True)
        ctx.save_for_backward(x, weight, bias, saved)
        ctx.act = act
        return y

    @staticmethod
    @once("linear_act")
    def backward(ctx, grad_y):
        x, weight, bias, saved = ctx.saved_tensors
        want = ctx.needs_input_grad
        gx = gw = gb = None
        if any(want[:3]):
            gx, gw, gb = ops.linear_act_bwd(grad_y.contiguous(), x, weight, saved, bias=bias, act=ctx.act,
                                            want_x=want[0], want_weight=want[1], want_bias=want[2])
        return gx, gw, gb, grad_y if want[3] else None, None


class ClassLogprobFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, labels, scale, top):
        logp, entropy, stats, top_logp, top_index = ops.class_logprob_fwd(logits, labels, scale=scale, top=top)
        ctx.save_for_backward(logits, labels, stats, entropy)
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        ctx.mark_non_differentiable(*(t for t in (top_logp, top_index) if t is not None))
        return logp, entropy, top_logp, top_index

    @staticmethod
    @once("class_logprob")
    def backward(ctx, grad_logp, grad_entropy, *_):
        logits, labels, stats, entropy = ctx.saved_tensors
        if grad_logp is None and grad_entropy is None:
            return (None,) * 4
        grads = (None if g is None else g.contiguous() for g in (grad_logp, grad_entropy))
        return ops.class_logprob_bwd(*grads, logits, labels, stats, entropy, scale=ctx.scale), None, None, None


def linear_act(x, weight, bias=None, *, act: str = "none", residual=None):
    """act(x weight^T + bias) + residual of x [..., ins], with gradients for every tensor given."""
    shape = (*x.shape[:-1], weight.shape[0])
    if residual is not None and residual.shape != shape:
        raise ValueError("residual must have shape %s (got %s)" % (shape, tuple(residual.shape)))
    rows, added = _rows(x), None if residual is None else _rows(residual)
    given = (rows, _rows(weight), None if bias is None else bias.contiguous(), added)
    if differentiated(*given):
        y = LinearActFunction.apply(*given, act)
    else:
        y = ops.linear_act_fwd(*given[:3], act=act, residual=added)[0]
    return y.view(shape)


def class_logprob(logits, labels, *, scale: float = 1.0, top: int = 0):
    """head.class_logprob_fwd with gradients of logp and entropy for the logits.  Returns (logp,
    entropy, top_logp, top_index); the last two have no gradient (None where top is 0)."""
    logits = _rows(logits)
    if differentiated(logits):
        return ClassLogprobFunction.apply(logits, labels, scale, top)
    logp, entropy, _, top_logp, top_index = ops.class_logprob_fwd(logits, labels, scale=scale, top=top)
    return logp, entropy, top_logp, top_index


class Dense(nn.Linear):
    """nn.Linear in linear_act's kernels."""

    def forward(self, x, act: str = "none"):
        return linear_act(x, self.weight, self.bias, act=act)


def dense(layer, x, act: str = "none"):
    """A layer, called as a module, and an activation ("none" or "relu").  A Dense has it in its kernel, where
    no hook is there to see the result before it, as those of nn.Linear do."""
    if act == "none":
        return layer(x)
    seen = layer._forward_hooks or layer._backward_hooks or layer._backward_pre_hooks or modules._has_any_global_hook()
    return layer(x, act=act) if isinstance(layer, Dense) and not seen else torch.relu(layer(x))


class BoxHead(nn.Module):
    """Two shared dense layers of `hidden` channels, then scores of `classes` classes and background
    (the last) and four deltas for each class."""

    def __init__(self, in_features: int, classes: int, hidden: int = 1024):
        super().__init__()
        self.classes = classes
        self.fc1, self.fc2 = Dense(in_features, hidden), Dense(hidden, hidden)
        self.score, self.delta = Dense(hidden, classes + 1), Dense(hidden, 4 * classes)

    def forward(self, x):
        """x: [K, channels, height, width] (or [K, in_features]) of the parameters' type."""
        x = x.flatten(1)
        for fc in (self.fc1, self.fc2):
            x = dense(fc, x, "relu")
        return dense(self.score, x), dense(self.delta, x)

    def loss(self, scores, labels):
        """Mean of -log p over the labels in [0, classes]; others are not counted."""
        logp = class_logprob(scores, labels)[0]
        counted = ((labels >= 0) & (labels <= self.classes)).sum()
        return -logp.sum() / counted.clamp(min=1)

    def best(self, scores, top: int, scale: float = 1.0):
        """(log probabilities, classes) of each row's `top` likeliest classes, background among them."""
        labels = scores.new_full(scores.shape[:1], -1, dtype=torch.int64)
        with torch.no_grad():
            return class_logprob(scores.detach(), labels, scale=scale, top=top)[2:]
