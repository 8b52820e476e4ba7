"""Thin ctypes binding of include/box_evict.h (argument marshalling only): the attention that
the boxes of a memory have received, and the boxes of least weight making room.

As in `relation`, whose memory this is, every operation runs in the library's HIP kernels on
torch's current stream (or `stream`), and nothing falls back.

Paper anchors (MMDetection, arXiv 1906.07155): §2 attention modules.
"""
from __future__ import annotations

import ctypes
import os
import re
import struct
from typing import List, Optional, Sequence

from . import binding
from .binding import _dtype_code, _need_cuda, _torch, check
from .relation import (MEMORY_PAGE, _RECALL, _Call, _bias, _boxes, _dense, _lengths, _memory_descriptor, _ptr, _rows4,
                       _same_device, _size)

HEADER = os.path.join(os.path.dirname(binding.HERE), "include", "box_evict.h")

_VP, _SZ, _D = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_char_p
_SZP = ctypes.POINTER(_SZ)

SIGNATURES = {
    "box_memory_weigh": [_D, _D, _VP, _VP, ctypes.c_float, _VP, _VP],
    "box_memory_evict_workspace_size": [_D, _D, _SZP],
    "box_memory_evict": [_D, _D, _VP, _VP, _VP, _VP, _SZ, _VP],
}

_EVICT = struct.Struct("@2q4P")     # box_evict_t

_lib = None


def header_functions() -> List[str]:
    """Names of the functions include/box_evict.h declares."""
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return re.findall(r"^\s*re_status_t\s+(\w+)\s*\(", text, flags=re.M)


def lib():
    """libroi_extract.so with this header's signatures (raises if it has not been built)."""
    global _lib
    if _lib is None:
        L = binding.lib()
        for name, argtypes in SIGNATURES.items():
            fn = getattr(L, name)
            fn.argtypes = argtypes
            fn.restype = ctypes.c_int
        _lib = L
    return _lib


def _table(pages, lengths, batch=None):
    """(batch, max_pages) of a checked table of pages and its lengths."""
    torch = _torch()
    if pages.dim() != 2 or (batch is not None and pages.shape[0] != batch):
        raise ValueError("pages must be 2-D [batch, max_pages]%s" % ("" if batch is None else " with batch %d" % batch))
    b, p = pages.shape
    _dense(pages, (b, p), "pages", torch.int32)
    _dense(lengths, (b,), "lengths", torch.int32)
    return b, p


def box_memory_weigh(q, memory: Sequence, pages, lengths, lse, *, weight=None, decay: float = 1.0,
                     scale: Optional[float] = None, q_boxes=None, bias=None, first_exp: int = -4,
                     octave_steps: int = 1, q_len=None, out=None, stream=None):
    """The attention that each remembered box receives from q [B, Nq, H, D], summed over heads and
    rows and added to decay * weight (float32 [B, 32 * max_pages], None: zeros).  pages, lengths,
    scale, q_boxes, bias and q_len as for box_memory_attn_fwd; lse float32 [B, H, Nq], as it
    returned it or of a softmax over more keys than these.  Returns float32 [B, 32 * max_pages], 0
    where a stream remembers nothing; `out` may be `weight`."""
    torch = _torch()
    m, hkv, dim = _memory_descriptor(memory)
    qs = _rows4(q, "q")
    B, nq, H, D = q.shape
    if D != dim:
        raise ValueError("q has %d channels a head, the memory %d" % (D, dim))
    if H % hkv:
        raise ValueError("the memory's %d heads must divide q's %d" % (hkv, H))
    code = _dtype_code(q)
    shape = (B, _table(pages, lengths, B)[1] * MEMORY_PAGE)
    _dense(lse, (B, H, nq), "lse", torch.float32)
    if q_len is not None:
        _lengths(q_len, B, "q_len")
    n = _bias(bias, H)
    strides = (0, 0)
    if n:
        strides = _boxes(q_boxes, B, nq, "q_boxes")
    else:
        q_boxes = None
    for t, name in ((weight, "weight"), (out, "out")):
        if t is not None:
            _dense(t, shape, name, torch.float32)
    _need_cuda(q, "q", memory[0])
    _same_device(q, "pages lengths lse q_len bias q_boxes weight out",
                 (pages, lengths, lse, q_len, bias, q_boxes, weight, out))
    d = _RECALL.pack(q.data_ptr(), code, H, B, nq, pages.shape[1], *qs[:3],
                     D ** -0.5 if scale is None else scale, n, first_exp, octave_steps,
                     _ptr(bias), _ptr(q_boxes), *strides, _ptr(q_len), pages.data_ptr(),
                     lengths.data_ptr())
    with _Call(q, stream) as c:
        if out is None:
            out = c.empty(shape, torch.float32)
        check(lib().box_memory_weigh(m, d, lse.data_ptr(), _ptr(weight), decay, out.data_ptr(), c.stream),
              "box_memory_weigh")
    return out


def box_memory_evict(memory: Sequence, pages, lengths, weight, keep, *, workspace=None, stream=None):
    """Each stream keeps its keep[b] (int32 [B]) boxes of the largest weight (float32
    [B, 32 * max_pages]), of equal ones those in lower places, in its first places; only kept boxes
    further on are moved.  pages (each named once) and lengths as for box_memory_attn_fwd.  memory may
    also be a list of memories with these pages (a head's layers), whose boxes are moved alike: where
    the call raises for want of memory or for an argument, none of them has changed.  Returns
    (lengths, weight, origin): int32 [B], float32 [B, 32 * max_pages] of the boxes where they now are (0
    behind them), and int32 [B, 32 * max_pages], the place that each was in (-1 behind them)."""
    torch = _torch()
    several = [memory] if len(memory) == 0 or torch.is_tensor(memory[0]) else list(memory)
    held_by = [_memory_descriptor(m)[0] for m in several]
    B, p = _table(pages, lengths)
    shape = (B, p * MEMORY_PAGE)
    _dense(weight, shape, "weight", torch.float32)
    _dense(keep, (B,), "keep", torch.int32)
    like = several[0][0]
    for m in several[1:]:
        if m[0].shape[0] != like.shape[0]:
            raise ValueError("memories with one table must have as many pages (got %d and %d)"
                             % (like.shape[0], m[0].shape[0]))
    _same_device(like, "pages lengths weight keep", (pages, lengths, weight, keep))
    _same_device(like, " ".join(["memory"] * len(several)), [m[0] for m in several])
    if workspace is not None:
        binding._workspace(workspace, like)
        _same_device(like, "workspace", (workspace,))
    d = _EVICT.pack(B, p, pages.data_ptr(), lengths.data_ptr(), keep.data_ptr(), weight.data_ptr())
    L = lib()
    with _Call(like, stream) as c:
        left, held, origin = c.empty((B,), torch.int32), c.empty(shape, torch.float32), c.empty(shape, torch.int32)
        need = 0
        if workspace is None or len(several) > 1:       # (which looks at all that the call looks at)
            need = max(_size(L.box_memory_evict_workspace_size, "box_memory_evict_workspace_size", m, d) for m in held_by)
        ws, wsb, _keep = c.workspace(workspace, need)
        for m in held_by:
            check(L.box_memory_evict(m, d, left.data_ptr(), held.data_ptr(), origin.data_ptr(), ws, wsb, c.stream),
                  "box_memory_evict")
    return left, held, origin
