"""A relation head on the operators of `relation`, with autograd: the boxes of an image attend
to each other and, in video, to the boxes of earlier frames (MMDetection, arXiv 1906.07155,
§2: attention modules; §3.1: it takes the place of a RoIHead's shared layers).

`box_attention` and `gated_norm` wire the kernels into torch.autograd, `BoxMemory` hands out
the pages of the 8-bit memory to streams, and `RelationHead` runs them together:

    head = RelationHead(256, heads=8).cuda()
    y = head(features, boxes, counts)                    # training: [images, boxes, channels]
    memory = head.memory(num_pages=4096, streams=4, max_pages=32)
    y = head(features, boxes, counts, memory=memory)     # video: recalls, then remembers
"""
from __future__ import annotations

from typing import List, Optional, Sequence

import torch
from torch import nn
from torch.autograd import forward_ad

from . import evict, relation


def box_head():
    from . import box_head as module                    # (which needs `once` of this module)
    return module


def differentiated(*tensors) -> bool:
    """Whether a call on these (None skipped) goes through autograd: one of them wants a gradient, or has a
    forward-mode tangent, which the functions here refuse (outside autograd it would be lost)."""
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors):
        return True
    # (0.05 us to see that there is no level, 0.3 to look at each tensor)
    return forward_ad._current_level >= 0 and any(
        t is not None and forward_ad.unpack_dual(t).tangent is not None for t in tensors)


class _Final(torch.autograd.Function):
    """Gradients of an operator that have no gradient themselves."""

    @staticmethod
    def forward(ctx, operator, _, *grads):
        ctx.operator = operator
        return tuple(g.view_as(g) for g in grads)

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("%s is once_differentiable: its gradients have none" % ctx.operator)


def once(operator):
    """Of an operator's backward: its results, under create_graph, fail where they are differentiated again
    instead of counting as constants (torch's once_differentiable does so only where the upstream gradient
    itself wants one)."""
    def wrap(backward):
        def wrapped(ctx, *upstream):
            with torch.no_grad():
                found = backward(ctx, *upstream)
            if not torch.is_grad_enabled():
                return found
            given = iter(_Final.apply(operator, torch.empty(0, requires_grad=True), *(g for g in found if g is not None)))
            return tuple(None if g is None else next(given) for g in found)
        return wrapped
    return wrap


class BoxAttnFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, bias, q_boxes, k_boxes, q_len, k_len, k_mask, cfg):
        geo = dict(bias=bias, q_boxes=q_boxes, k_boxes=k_boxes, q_len=q_len, k_len=k_len, k_mask=k_mask, **cfg)
        out, lse, out_f32 = relation.box_attn_fwd(q, k, v, save=True, **geo)
        ctx.save_for_backward(q, k, v, bias, q_boxes, k_boxes, q_len, k_len, k_mask, out, lse, out_f32)
        ctx.cfg = cfg
        ctx.mark_non_differentiable(lse)
        return out, lse

    @staticmethod
    @once("box_attention")
    def backward(ctx, grad_out, _):
        q, k, v, bias, q_boxes, k_boxes, q_len, k_len, k_mask, out, lse, out_f32 = ctx.saved_tensors
        grads = relation.box_attn_bwd(grad_out.contiguous(), q, k, v, out, lse, out_f32, bias=bias,
                                      q_boxes=q_boxes, k_boxes=k_boxes, q_len=q_len, k_len=k_len,
                                      k_mask=k_mask, **ctx.cfg)
        return (*grads, None, None, None, None, None, None)


class GatedNormFunction(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, branch, gate, post_weight, post_bias, pre_weight, pre_bias, cfg, second):
        args = dict(gate=gate, post_weight=post_weight, post_bias=post_bias, pre_weight=pre_weight,
                    pre_bias=pre_bias, **cfg)
        y, u, stats = relation.gated_norm_fwd(x, branch, second=second, save=True, **args)
        ctx.save_for_backward(x, branch, gate, post_weight, post_bias, pre_weight, pre_bias, stats)
        ctx.cfg = cfg
        ctx.set_materialize_grads(False)
        return (u if branch is None else y), (None if branch is None else u)

    @staticmethod
    @once("gated_norm")
    def backward(ctx, grad_y, grad_u):
        x, branch, gate, w1, c1, w2, c2, stats = ctx.saved_tensors
        if branch is None:                  # the one output is u
            grad_y, grad_u = None, grad_y
        if grad_y is None and grad_u is None:
            return (None,) * 9
        grads = relation.gated_norm_bwd(*(None if g is None else g.contiguous() for g in (grad_y, grad_u)),
                                        x, branch, stats, gate=gate, post_weight=w1, post_bias=c1,
                                        pre_weight=w2, pre_bias=c2, **ctx.cfg)
        return (*grads, None, None)


def box_attention(q, k, v, *, bias=None, q_boxes=None, k_boxes=None, q_len=None, k_len=None, k_mask=None,
                  **cfg):
    """relation.box_attn_fwd with gradients for q, k, v and bias.  Returns (out, lse); lse has
    no gradient.  `cfg`: scale, first_exp, octave_steps."""
    if not differentiated(q, k, v, bias):
        relation._rows4(q, "q")
        lse = torch.empty((q.shape[0], q.shape[2], q.shape[1]), dtype=torch.float32, device=q.device)
        return relation.box_attn_fwd(q, k, v, bias=bias, q_boxes=q_boxes, k_boxes=k_boxes, q_len=q_len,
                                     k_len=k_len, k_mask=k_mask, lse=lse, **cfg)[:2]     # nothing else is kept
    return BoxAttnFunction.apply(q, k, v, bias, q_boxes, k_boxes, q_len, k_len, k_mask, cfg)


def gated_norm(x, branch=None, *, gate=None, post_weight=None, post_bias=None, pre_weight=None,
               pre_bias=None, second: bool = True, alpha: float = 1.0, norm: str = "rms",
               eps: float = 1e-6):
    """relation.gated_norm_fwd with gradients for every tensor given.  Returns (y, u): y is x
    without a branch, u None without the second norm."""
    if branch is None and not second:
        raise ValueError("neither a branch nor the second norm: nothing to do")
    cfg = dict(alpha=alpha, norm=norm, eps=eps)
    given = (x, branch, gate, post_weight, post_bias, pre_weight, pre_bias)
    if not differentiated(*given):
        return relation.gated_norm_fwd(x, branch, gate=gate, post_weight=post_weight, post_bias=post_bias,
                                       pre_weight=pre_weight, pre_bias=pre_bias, second=second, **cfg)[:2]
    first, u = GatedNormFunction.apply(*given, cfg, second)
    return (x, first) if branch is None else (first, u)


class BoxMemory:
    """The 8-bit memories of a head's layers, which share one table of pages.

    Streams take pages of 32 boxes from one pool.  With evict "oldest" a stream with `max_pages`
    pages gives its oldest page back for a new one, so it remembers at least 32 * (max_pages - 1)
    boxes.  With evict "weight" a full stream loses the boxes that have received the least attention
    (`weight`: of all heads, rows and layers, of earlier frames `decay` times as much with every
    frame), as many as are needed for the new ones.  The
    order of places means nothing to the attention.  The table is kept on the host and copied to
    the device when it has changed."""

    def __init__(self, num_pages: int, streams: int, max_pages: int, kv_heads: int, dim: int,
                 layers: int = 1, device="cuda", evict: str = "oldest", decay: float = 0.9):
        if not 2 <= max_pages <= num_pages:
            raise ValueError("max_pages must be in [2, num_pages] (got %d of %d)" % (max_pages, num_pages))
        if streams < 1 or layers < 1:
            raise ValueError("a memory has at least one stream and one layer")
        if evict not in ("oldest", "weight"):
            raise ValueError("evict must be 'oldest' or 'weight' (got %r)" % (evict,))
        self.layers = [relation.box_memory(num_pages, kv_heads, dim, device) for _ in range(layers)]
        self.decay = decay
        self.weight = None                              # [streams, places] where it decides what leaves
        if evict == "weight":
            self.weight = torch.zeros((streams, max_pages * relation.MEMORY_PAGE), dtype=torch.float32, device=device)
        self.max_pages, self.device = max_pages, device
        self.free = list(range(num_pages - 1, -1, -1))
        self.table: List[List[int]] = [[] for _ in range(streams)]
        self.used = [0] * streams                       # boxes a stream remembers
        self._device_table = None

    def check(self, counts: Sequence[int]) -> None:
        """Raises where take(counts) would."""
        page = relation.MEMORY_PAGE
        most = page * (self.max_pages - 1)              # none of them meets a page of the same call
        if len(counts) != len(self.table) or any(c < 0 or c > most for c in counts):
            raise ValueError("counts must hold a number of boxes in [0, %d] for each of the %d streams"
                             % (most, len(self.table)))
        need = 0
        for pages, used, c in zip(self.table, self.used, counts):
            if self.weight is not None:                 # room is made for what does not fit
                used = min(used, page * self.max_pages - c)
            total = (used + c + page - 1) // page
            need += min(total, self.max_pages) - len(pages) if total > len(pages) else 0
        if need > len(self.free):
            raise RuntimeError("the memory has %d free pages, %d are needed" % (len(self.free), need))

    def take(self, counts: Sequence[int]):
        """Places for counts[s] new boxes of each stream: int64 slots of all of them, stream
        after stream.  Raises (and takes nothing) where the pool has too few pages."""
        self.check(counts)
        page, weight = relation.MEMORY_PAGE, self.weight
        free, table, used = list(self.free), [list(p) for p in self.table], list(self.used)
        if weight is not None:                          # the boxes of least weight leave, as many as have to
            used = [min(u, page * self.max_pages - c) for u, c in zip(used, counts)]
        keep = list(used)
        slots: List[int] = []
        for s, c in enumerate(counts):
            pages = table[s]
            while c > 0:
                if used[s] == page * len(pages):
                    if len(pages) == self.max_pages:
                        free.append(pages.pop(0))
                        used[s] -= page
                    pages.append(free.pop())
                at, into = used[s] % page, pages[used[s] // page]
                n = min(c, page - at)
                slots.extend(range(into * page + at, into * page + at + n))
                used[s] += n
                c -= n
        made = torch.tensor(slots, dtype=torch.int64, device=self.device)
        if weight is not None and keep != self.used:    # (the last that may fail: it moves boxes)
            held, lengths = self.pages_and_lengths()
            kept = torch.tensor(keep, dtype=torch.int32, device=self.device)
            _, weight, _ = evict.box_memory_evict(self.layers, held, lengths, weight, kept)
        self.free, self.table, self.used, self.weight, self._device_table = free, table, used, weight, None
        return made

    def forget(self, stream: int) -> None:
        """The stream's pages go back to the pool."""
        if self.weight is not None:
            self.weight = self.weight.clone()           # (made in inference mode it takes no writes outside)
            self.weight[stream] = 0
        self.free.extend(self.table[stream])
        self.table[stream], self.used[stream] = [], 0
        self._device_table = None

    def pages_and_lengths(self):
        """(pages int32 [streams, max_pages], lengths int32 [streams]) on the device."""
        if self._device_table is None:
            rows = [p + [-1] * (self.max_pages - len(p)) for p in self.table]
            self._device_table = (torch.tensor(rows, dtype=torch.int32, device=self.device),
                                  torch.tensor(self.used, dtype=torch.int32, device=self.device))
        return self._device_table


class RelationLayer(nn.Module):
    """One block: attention among the boxes (and over the memory), then two linear layers.  Each
    branch is normalised, gated for its image from the mean over its boxes, added to the features,
    and normalised for what follows, in one kernel."""

    def __init__(self, channels: int, heads: int, kv_heads: int, buckets: int, norm: str, fused: bool = False):
        super().__init__()
        self.fused = fused
        self.heads, self.kv_heads, self.dim = heads, kv_heads, channels // heads
        self.norm = norm
        linear = box_head().Dense if fused else nn.Linear
        self.qkv = linear(channels, (heads + 2 * kv_heads) * self.dim)
        self.proj = linear(channels, channels)
        self.fc1 = linear(channels, 2 * channels)
        self.fc2 = linear(2 * channels, channels)
        self.gate = linear(channels, channels)
        # parameters of the kernels stay binary32 when the module's type is changed
        self.bias = nn.Parameter(torch.zeros(heads, buckets, buckets))
        self.post = nn.ParameterList([nn.Parameter(torch.ones(channels)) for _ in range(2)])
        self.pre = nn.ParameterList([nn.Parameter(torch.ones(channels)) for _ in range(2)])

    def _apply(self, fn, recurse=True):
        own = lambda: (self.bias, *self.post, *self.pre)
        kept = [(p.data, None if p.grad is None else p.grad.data) for p in own()]
        super()._apply(fn, recurse)
        for p, (data, grad) in zip(own(), kept):        # as they were, not widened from another type
            if p.dtype != torch.float32:
                device = p.device
                p.grad = None                           # (a gradient has its parameter's type)
                p.data = data.to(device)
                p.grad = None if grad is None else grad.to(device)
        return self

    def _dense(self, layer, x, act: str = "none"):
        if self.fused:
            return box_head().dense(layer, x, act)
        return torch.relu(layer(x)) if act == "relu" else layer(x)

    def forward(self, x, u, gate, boxes, lengths, recall, last: bool, pre_next):
        """x [images, boxes, channels] and u, x normalised -> (x, u) for the next layer."""
        B, n, c = x.shape
        split = [self.heads, self.kv_heads, self.kv_heads]
        q, k, v = self._dense(self.qkv, u).view(B, n, sum(split), self.dim).split(split, 2)
        geo = dict(bias=self.bias, q_boxes=boxes, k_boxes=boxes, q_len=lengths, k_len=lengths)
        out = box_attention(q, k, v, **geo)[0] if recall is None else recall(q, k, v, geo)
        branch = self._dense(self.proj, out.reshape(B * n, c))
        gate = torch.sigmoid(self._dense(self.gate, gate)).float()
        x, u = gated_norm(x.reshape(B * n, c), branch, gate=gate, post_weight=self.post[0],
                          pre_weight=self.pre[1], norm=self.norm)
        branch = self._dense(self.fc2, self._dense(self.fc1, u, "relu"))
        x, u = gated_norm(x, branch, gate=gate, post_weight=self.post[1], pre_weight=pre_next,
                          norm=self.norm, second=not last)
        return x.view(B, n, c), None if u is None else u.view(B, n, c)


class RelationHead(nn.Module):
    """Layers of relations among the boxes of an image.  channels / heads channels a head, a
    multiple of 8; kv_heads heads share keys in equal groups; buckets a side of the bias table;
    fused: the dense layers run in linear_act's kernels, in torch's otherwise."""

    def __init__(self, channels: int, heads: int, kv_heads: Optional[int] = None, layers: int = 2,
                 buckets: int = 15, norm: str = "rms", fused: bool = False):
        super().__init__()
        kv_heads = kv_heads or heads
        if channels % heads or channels // heads % 8 or channels // heads > relation.MAX_DIM:
            raise ValueError("channels / heads must be a multiple of 8, at most %d" % relation.MAX_DIM)
        if heads % kv_heads:
            raise ValueError("kv_heads must divide heads")
        self.layers = nn.ModuleList(RelationLayer(channels, heads, kv_heads, buckets, norm, fused)
                                    for _ in range(layers))

    def memory(self, num_pages: int, streams: int, max_pages: int, evict: str = "oldest",
               decay: float = 0.9) -> BoxMemory:
        """A memory for `streams` videos, one image of each to a call."""
        first = self.layers[0]
        return BoxMemory(num_pages, streams, max_pages, first.kv_heads, first.dim, len(self.layers),
                         first.bias.device, evict, decay)

    def forward(self, x, boxes, counts: Optional[Sequence[int]] = None, memory: Optional[BoxMemory] = None):
        """x [images, boxes, channels] float32 or bfloat16, boxes float32 [images, boxes, 4] (x1, y1,
        x2, y2), counts: valid boxes of each image (a list, or a tensor, which is copied to
        the host where it is not there; None: all).  Rows past an image's count are
        0 in the result, and what they hold, NaN and infinities included, has no effect on it or
        on any gradient.  With a memory, image s
        is the next frame of stream s: its boxes attend to each other and to what the stream
        remembers, and are remembered (inference only: the memory has no gradient)."""
        B, n, c = x.shape
        if memory is not None and torch.is_grad_enabled():
            raise RuntimeError("a memory is for inference: call under torch.no_grad()")
        if memory is not None and len(memory.table) != B:
            raise ValueError("the memory has %d streams, x %d images" % (len(memory.table), B))
        if torch.is_tensor(counts):             # one copy, where the elements would be read one by one
            counts = counts.tolist()
        host = [n] * B if counts is None else [int(k) for k in counts]
        if len(host) != B or any(k < 0 or k > n for k in host):
            raise ValueError("counts must hold a number in [0, %d] for each of the %d images" % (n, B))
        lengths = None if counts is None else torch.tensor(host, dtype=torch.int32, device=x.device)
        if lengths is not None:                 # (chosen, not multiplied: 0 * NaN is NaN)
            valid = (torch.arange(n, device=x.device) < lengths[:, None])[..., None]
            x = torch.where(valid, x, torch.zeros_like(x))
            # (in binary32: bf16 has no 257, and the sum would be rounded before it is divided)
            gate = (x.sum(1, dtype=torch.float32) / lengths.clamp(min=1)[:, None]).to(x.dtype)
        else:
            gate = x.mean(1) if n else x.new_zeros(B, c)

        recalled = None
        fresh = []                              # what each layer is to remember
        weight = None if memory is None else memory.weight
        if memory is not None:
            memory.check(host)
            first = self.layers[0]
            if len(memory.layers) != len(self.layers) or any(
                    m[0].shape[1] != first.kv_heads or m[0].shape[3] != first.dim for m in memory.layers):
                raise ValueError("the memory is not one of this head's: %d layers of %d heads of %d channels"
                                 % (len(self.layers), first.kv_heads, first.dim))
            pages, remembered = memory.pages_and_lengths()
            rows = torch.cat([torch.arange(k, device=x.device) + i * n for i, k in enumerate(host)])
        _, u = gated_norm(x.reshape(B * n, c), pre_weight=self.layers[0].pre[0], norm=self.layers[0].norm)
        u = u.view(B, n, c)
        for i, layer in enumerate(self.layers):
            if memory is not None:
                def recalled(q, k, v, geo, held=memory.layers[i], first_layer=i == 0):
                    nonlocal weight
                    if differentiated(q, k, v):
                        raise RuntimeError("a memory is for inference: what it recalls has no forward-mode tangent")
                    # both parts in binary32 (the memory's by binary32 queries), rounded when joined
                    out, lse, full = relation.box_attn_fwd(q, k, v, save=True, **geo)
                    far, far_lse = relation.box_memory_attn_fwd(q.float(), held, pages, remembered, q_boxes=boxes,
                                                                bias=geo["bias"], q_len=lengths, save=True)
                    if weight is not None:      # their share of the softmax over both
                        weight = evict.box_memory_weigh(
                            q.float(), held, pages, remembered, torch.logaddexp(lse, far_lse), weight=weight,
                            decay=memory.decay if first_layer else 1.0, q_boxes=boxes, bias=geo["bias"], q_len=lengths)
                    fresh.append((held, *(t.reshape(B * n, *t.shape[2:])[rows] for t in (k, v))))
                    # one softmax over both: far's share is exp(far_lse) of the sum of both
                    share = torch.where(far_lse == -torch.inf, torch.zeros_like(lse),
                                        torch.sigmoid(far_lse - lse)).transpose(1, 2)[..., None]
                    return torch.lerp(out if full is None else full, far, share).to(out.dtype)
            last = i + 1 == len(self.layers)
            x, u = layer(x, u, gate, boxes, lengths, recalled, last,
                         None if last else self.layers[i + 1].pre[0])
        if lengths is not None:
            x = torch.where(valid, x, torch.zeros_like(x))
        if memory is not None:                  # nothing is taken or written before all of it is there
            kept = boxes.reshape(B * n, 4)[rows].contiguous()
            before, memory.weight = memory.weight, weight       # (the frame's own decide what leaves)
            try:
                slots = memory.take(host)
            except BaseException:
                memory.weight = before
                raise
            for held, k, v in fresh:
                relation.box_memory_append(held, slots, k, v, kept)
        return x
