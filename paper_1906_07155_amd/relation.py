"""Thin ctypes binding of include/box_relation.h (argument marshalling only): attention
among the boxes of an image with a learned bias by bucket, its 8-bit memory of earlier
frames, and the gated norms around it.

As in `binding`, every operation runs in the library's HIP kernels on torch's current
stream (or `stream`), and nothing falls back.  The descriptors are packed in one go into
bytes, field by field in the order of the C structs: these calls are short, and setting
ctypes fields one by one would cost more than some of them take on the GPU.

Paper anchors (MMDetection, arXiv 1906.07155): §2 attention modules (Generalized
Attention, GCNet), §3.1 RoIHead.
"""
from __future__ import annotations

import ctypes
import os
import re
import struct
from typing import List, Optional, Sequence, Tuple

from . import binding
from .binding import RE_DTYPE_BF16, _dtype_code, _need_cuda, _torch, check

HEADER = os.path.join(os.path.dirname(binding.HERE), "include", "box_relation.h")

MAX_DIM, MAX_HEADS, MAX_BUCKETS, MEMORY_PAGE = 128, 256, 31, 32
FEW_KEYS = 64                       # RE_ATTN_FEW_KEYS
NORMS = {"rms": 0, "layer": 1}      # RE_NORM_RMS, RE_NORM_LAYER

_VP, _I32, _I64, _SZ, _D = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t,
                            ctypes.c_char_p)
_SZP = ctypes.POINTER(_SZ)

SIGNATURES = {
    "box_attn_workspace_size": [_D, _I32, _SZP],
    "box_attn_fwd": [_D, _VP, _VP, _VP, _VP, _SZ, _VP],
    "box_attn_bwd": [_D, _VP, _VP, _VP, _VP, _VP, _VP, _VP, _VP, _VP, _SZ, _VP],
    "box_memory_append": [_D, _VP, _I64, _VP, _VP, _I32, _D, _D, _VP, _VP],
    "box_memory_read": [_D, _VP, _I64, _VP, _VP, _I32, _VP, _VP],
    "box_memory_attn_workspace_size": [_D, _D, _SZP],
    "box_memory_attn_fwd": [_D, _D, _VP, _VP, _VP, _SZ, _VP],
    "gated_norm_workspace_size": [_D, _SZP],
    "gated_norm_fwd": [_D, _VP, _VP, _VP, _VP],
    "gated_norm_bwd": [_D, _VP, _VP, _VP, _D, _VP, _SZ, _VP],
}

# box_attn_t, box_memory_t, box_recall_t, gated_norm_t, gated_norm_grads_t
_ATTN = struct.Struct("@3P4i12qf3i3P4q3P")
_MEMORY = struct.Struct("@5Pq2i")
_RECALL = struct.Struct("@P2i6qf3i2P2q3P")
_NORM = struct.Struct("@2P2q2iqi2f4xq5P")
_GRADS = struct.Struct("@7P")
_PAIR = struct.Struct("@2q")

_lib = None


def header_functions() -> List[str]:
    """Names of the functions include/box_relation.h declares."""
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


# ---------------------------------------------------------------------------
# Marshalling
# ---------------------------------------------------------------------------

class _Call:
    """One call's stream, and a `with` block's worth of its device where that is not the
    current one.  Tensors that a call on a given stream allocates itself come from that stream's
    memory (what the current stream has given back may still be in use by what is enqueued there),
    and the current stream, on which their user is, is recorded with them."""

    __slots__ = ("device", "other", "stream", "guard")

    def __init__(self, like, stream):
        torch = _torch()
        self.device, self.other, self.guard = like.device, stream, None
        index = like.get_device()
        # (torch.cuda.current_device looks whether CUDA is there first: 0.25 us, 0.05 without; it is,
        # with a tensor on it.  torch.cuda.current_stream makes a Stream object: 1.9 us, the handle
        # alone 0.1 us)
        if index != torch._C._cuda_getDevice():
            self.guard = torch.cuda.device(self.device)
        self.stream = torch._C._cuda_getCurrentRawStream(index) if stream is None else stream.cuda_stream

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()
        return self

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)

    def empty(self, shape, dtype):
        torch = _torch()
        if self.other is None:
            return torch.empty(*shape, dtype=dtype, device=self.device)   # (0.4 us less than a tuple)
        with torch.cuda.stream(self.other):
            t = torch.empty(*shape, dtype=dtype, device=self.device)
        t.record_stream(torch.cuda.current_stream(self.device))
        return t

    def workspace(self, given, need):
        """(pointer, bytes, tensor to keep) of the given workspace or of one of `need` bytes."""
        if given is not None:
            return given.data_ptr(), given.numel(), given
        if need == 0:
            return None, 0, None
        t = self.empty((need,), _torch().uint8)
        return t.data_ptr(), need, t


def _rows4(t, name: str, shape=None):
    """The strides of a [batch, rows, heads, dim] tensor with adjacent channels."""
    if t.dim() != 4 or (shape is not None and t.shape != shape):
        raise ValueError("%s must be a 4-D [batch, rows, heads, dim] tensor%s (got %s)"
                         % (name, "" if shape is None else " of shape %s" % (tuple(shape),),
                            tuple(t.shape)))
    strides = t.stride()
    if strides[3] != 1 and t.shape[3] > 1 and t.numel() > 0:
        raise ValueError("the channels of %s must be adjacent" % name)
    return strides


def _dense(t, shape, name: str, dtype):
    if t.shape != shape or t.dtype != dtype or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor of shape %s (got %s %s)"
                         % (name, dtype, tuple(shape), t.dtype, tuple(t.shape)))
    return t


def _boxes(t, batch: int, num: int, name: str):
    torch = _torch()
    if t is None:
        raise ValueError("%s is required with a bias" % name)
    if t.dtype != torch.float32 or t.shape != (batch, num, 4):
        raise ValueError("%s must be a float32 tensor of shape %s (got %s %s)"
                         % (name, (batch, num, 4), t.dtype, tuple(t.shape)))
    strides = t.stride()
    if strides[2] != 1 and t.numel() > 0:
        raise ValueError("the coordinates of %s must be adjacent" % name)
    return strides[:2]


def _bias(bias, heads: int):
    torch = _torch()
    if bias is None:
        return 0
    n = bias.shape[-1] if bias.dim() else 0
    if n < 1 or n > MAX_BUCKETS or n % 2 == 0:
        raise ValueError("bias must have an odd number of buckets per axis, at most %d" % MAX_BUCKETS)
    _dense(bias, (heads, n, n), "bias", torch.float32)
    return n


def _lengths(t, batch: int, name: str):
    _dense(t, (batch,), name, _torch().int32)


def _same_device(like, names, tensors):
    """Every given tensor (None skipped) is on the device of `like`."""
    index = like.get_device()               # (an int is compared faster than a device)
    for t in tensors:
        if t is not None and t.get_device() != index:
            for name, u in zip(names.split(), tensors):
                if u is not None:
                    _need_cuda(u, name, like)


def _ptr(t):
    return 0 if t is None else t.data_ptr()


def _attn_descriptor(q, k, v, scale, q_boxes, k_boxes, bias, first_exp, octave_steps, q_len,
                     k_len, k_mask):
    """box_attn_t of checked tensors, as bytes."""
    torch = _torch()
    qs, ks = _rows4(q, "q"), _rows4(k, "k")
    B, nq, H, D = q.shape
    _, nk, hkv, _ = k.shape
    if k.shape != (B, nk, hkv, D):
        _rows4(k, "k", (B, nk, hkv, D))
    vs = _rows4(v, "v", k.shape)
    code = _dtype_code(q)
    if k.dtype != q.dtype or v.dtype != q.dtype:
        raise TypeError("q, k and v must have one dtype (got %s, %s, %s)"
                        % (q.dtype, k.dtype, v.dtype))
    n = _bias(bias, H)
    boxes = (0,) * 4
    if n:
        boxes = _boxes(q_boxes, B, nq, "q_boxes") + _boxes(k_boxes, B, nk, "k_boxes")
    else:
        q_boxes = k_boxes = None
    if q_len is not None:
        _lengths(q_len, B, "q_len")
    if k_len is not None:
        _lengths(k_len, B, "k_len")
    if k_mask is not None:
        if k_mask.dtype not in (torch.bool, torch.uint8):
            raise ValueError("k_mask must be bool or uint8 (got %s)" % k_mask.dtype)
        _dense(k_mask, (B, nk), "k_mask", k_mask.dtype)
    _need_cuda(q, "q")
    _same_device(q, "k v bias q_boxes k_boxes q_len k_len k_mask",
                 (k, v, bias, q_boxes, k_boxes, q_len, k_len, k_mask))
    if scale is None:
        scale = D ** -0.5
    return _ATTN.pack(q.data_ptr(), k.data_ptr(), v.data_ptr(), code, H, hkv, D, B, nq, nk,
                      *qs[:3], *ks[:3], *vs[:3], scale, n, first_exp,
                      octave_steps, _ptr(bias), _ptr(q_boxes), _ptr(k_boxes), *boxes,
                      _ptr(q_len), _ptr(k_len), _ptr(k_mask))


def _size(fn, where, *args) -> int:
    n = ctypes.c_size_t(0)
    check(fn(*args, ctypes.byref(n)), where)
    return n.value


# ---------------------------------------------------------------------------
# Attention among boxes
# ---------------------------------------------------------------------------

def box_attn_workspace_size(q, k, v, backward: bool = False, *, q_boxes=None, k_boxes=None,
                            bias=None) -> int:
    """Workspace bytes of box_attn_fwd (and box_attn_bwd where `backward`) at these shapes."""
    d = _attn_descriptor(q, k, v, None, q_boxes, k_boxes, bias, -4, 1, None, None, None)
    return _size(lib().box_attn_workspace_size, "box_attn_workspace_size", d, int(backward))


def box_attn_fwd(q, k, v, *, scale: Optional[float] = None, q_boxes=None, k_boxes=None, bias=None,
                 first_exp: int = -4, octave_steps: int = 1, q_len=None, k_len=None, k_mask=None,
                 save: bool = False, out=None, lse=None, out_f32=None, workspace=None, stream=None):
    """Attention of q [B, Nq, H, D] over k, v [B, Nk, Hkv, D] (heads share keys where Hkv < H).
    bias: float32 [H, n, n] by bucket of (q_boxes [B, Nq, 4], k_boxes [B, Nk, 4]); q_len,
    k_len: int32 [B] valid rows; k_mask: bool [B, Nk], False leaves a key out; scale: D^-1/2
    by default.  Returns (out, lse, out_f32): lse float32 [B, H, Nq] and (for bf16 data) out_f32,
    `out` in float32, are what the backward takes, made where `save` is true or they are given,
    else None."""
    torch = _torch()
    d = _attn_descriptor(q, k, v, scale, q_boxes, k_boxes, bias, first_exp, octave_steps, q_len,
                         k_len, k_mask)
    B, nq, H, D = q.shape
    if out is not None:
        _dense(out, (B, nq, H, D), "out", q.dtype)
    if out_f32 is not None:
        _dense(out_f32, (B, nq, H, D), "out_f32", torch.float32)
    if lse is not None:
        _dense(lse, (B, H, nq), "lse", torch.float32)
    _same_device(q, "out lse out_f32", (out, lse, out_f32))
    if workspace is not None:
        binding._workspace(workspace, q)
        _same_device(q, "workspace", (workspace,))
    L = lib()
    with _Call(q, stream) as c:
        if out is None:
            out = c.empty((B, nq, H, D), q.dtype)
        if save and lse is None:
            lse = c.empty((B, H, nq), torch.float32)
        if save and out_f32 is None and q.dtype == torch.bfloat16:
            out_f32 = c.empty((B, nq, H, D), torch.float32)
        need = 0
        if workspace is None:
            need = _size(L.box_attn_workspace_size, "box_attn_workspace_size", d, 0)
        ws, wsb, _keep = c.workspace(workspace, need)
        check(L.box_attn_fwd(d, out.data_ptr(), _ptr(lse), _ptr(out_f32), ws, wsb, c.stream),
              "box_attn_fwd")
    return out, lse, out_f32


def box_attn_bwd(grad_out, q, k, v, out, lse, out_f32=None, *, scale: Optional[float] = None,
                 q_boxes=None, k_boxes=None, bias=None, first_exp: int = -4, octave_steps: int = 1,
                 q_len=None, k_len=None, k_mask=None, grad_q=None, grad_k=None, grad_v=None,
                 grad_bias=None, workspace=None, stream=None):
    """Gradients of box_attn_fwd for upstream grad_out (contiguous, as out); out, lse and
    out_f32 as it returned them.  Returns (grad_q, grad_k, grad_v, grad_bias): dense, of
    the inputs' dtype, and float32 [H, n, n] (None without bias)."""
    torch = _torch()
    d = _attn_descriptor(q, k, v, scale, q_boxes, k_boxes, bias, first_exp, octave_steps, q_len,
                         k_len, k_mask)
    B, nq, H, D = q.shape
    for t, name in ((grad_out, "grad_out"), (out, "out"), (grad_q, "grad_q")):
        if t is not None:
            _dense(t, q.shape, name, q.dtype)
    for t, name in ((grad_k, "grad_k"), (grad_v, "grad_v")):
        if t is not None:
            _dense(t, k.shape, name, q.dtype)
    if out_f32 is not None:
        _dense(out_f32, q.shape, "out_f32", torch.float32)
    _dense(lse, (B, H, nq), "lse", torch.float32)
    if grad_bias is not None:
        if bias is None:
            raise ValueError("grad_bias without a bias")
        _dense(grad_bias, bias.shape, "grad_bias", torch.float32)
    _same_device(q, "grad_out out lse out_f32 grad_q grad_k grad_v grad_bias",
                 (grad_out, out, lse, out_f32, grad_q, grad_k, grad_v, grad_bias))
    if workspace is not None:
        binding._workspace(workspace, q)
        _same_device(q, "workspace", (workspace,))
    L = lib()
    with _Call(q, stream) as c:
        if grad_q is None:
            grad_q = c.empty(q.shape, q.dtype)
        if grad_k is None:
            grad_k = c.empty(k.shape, q.dtype)
        if grad_v is None:
            grad_v = c.empty(k.shape, q.dtype)
        if grad_bias is None and bias is not None:
            grad_bias = c.empty(bias.shape, torch.float32)
        need = 0
        if workspace is None:
            need = _size(L.box_attn_workspace_size, "box_attn_workspace_size", d, 1)
        ws, wsb, _keep = c.workspace(workspace, need)
        check(L.box_attn_bwd(d, grad_out.data_ptr(), out.data_ptr(), lse.data_ptr(), _ptr(out_f32),
                             grad_q.data_ptr(), grad_k.data_ptr(), grad_v.data_ptr(),
                             _ptr(grad_bias), ws, wsb, c.stream), "box_attn_bwd")
    return grad_q, grad_k, grad_v, grad_bias


# ---------------------------------------------------------------------------
# The memory
# ---------------------------------------------------------------------------

def box_memory(num_pages: int, kv_heads: int, dim: int, device="cuda"):
    """A zeroed memory of `num_pages` pages of 32 boxes: (k, v, k_scale, v_scale, boxes)."""
    torch = _torch()
    p = MEMORY_PAGE
    return (torch.zeros((num_pages, kv_heads, p, dim), dtype=torch.int8, device=device),
            torch.zeros((num_pages, kv_heads, dim, p), dtype=torch.int8, device=device),
            torch.zeros((num_pages, kv_heads, p), dtype=torch.float32, device=device),
            torch.zeros((num_pages, kv_heads, p), dtype=torch.float32, device=device),
            torch.zeros((num_pages, p, 4), dtype=torch.float32, device=device))


def _memory_descriptor(memory):
    torch = _torch()
    if len(memory) != 5:
        raise ValueError("a memory is (k, v, k_scale, v_scale, boxes)")
    k, v, ks, vs, boxes = memory
    if k.dim() != 4 or k.shape[2] != MEMORY_PAGE:
        raise ValueError("the memory's k must be [pages, kv_heads, %d, dim] (got %s)"
                         % (MEMORY_PAGE, tuple(k.shape)))
    pages, hkv, p, dim = k.shape
    _dense(k, (pages, hkv, p, dim), "the memory's k", torch.int8)
    _dense(v, (pages, hkv, dim, p), "the memory's v", torch.int8)
    _dense(ks, (pages, hkv, p), "the memory's k_scale", torch.float32)
    _dense(vs, (pages, hkv, p), "the memory's v_scale", torch.float32)
    _dense(boxes, (pages, p, 4), "the memory's boxes", torch.float32)
    _need_cuda(k, "the memory")
    _same_device(k, "v k_scale v_scale boxes", (v, ks, vs, boxes))
    return _MEMORY.pack(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(),
                        boxes.data_ptr(), pages, hkv, dim), hkv, dim


def _slots(slots, like):
    torch = _torch()
    if slots.dim() != 1:
        raise ValueError("slots must be 1-D")
    _dense(slots, (slots.shape[0],), "slots", torch.int64)
    _same_device(like, "slots", (slots,))
    return slots.shape[0]


def box_memory_append(memory: Sequence, slots, k, v, boxes, stream=None) -> None:
    """Quantise k, v [N, Hkv, D] and write them with their boxes [N, 4] to slots (int64 [N];
    slot s is place s % 32 of page s // 32; one outside the memory is skipped)."""
    torch = _torch()
    d, hkv, dim = _memory_descriptor(memory)
    like = memory[0]
    n = _slots(slots, like)
    for t, name in ((k, "k"), (v, "v")):
        if tuple(t.shape) != (n, hkv, dim):
            raise ValueError("%s must have shape %s (got %s)" % (name, (n, hkv, dim), tuple(t.shape)))
        if n > 0 and t.stride(2) != 1:
            raise ValueError("the channels of %s must be adjacent" % name)
    if k.dtype != v.dtype:
        raise TypeError("k and v must have one dtype (got %s, %s)" % (k.dtype, v.dtype))
    code = _dtype_code(k)
    _dense(boxes, (n, 4), "boxes", torch.float32)
    _same_device(like, "k v boxes", (k, v, boxes))
    with _Call(like, stream) as c:
        check(lib().box_memory_append(d, slots.data_ptr(), n, k.data_ptr(), v.data_ptr(), code,
                                      _PAIR.pack(*k.stride()[:2]), _PAIR.pack(*v.stride()[:2]),
                                      boxes.data_ptr(), c.stream), "box_memory_append")


def box_memory_read(memory: Sequence, slots, dtype=None, stream=None):
    """What the slots (int64 [N]) hold: (k [N, Hkv, D], v, boxes [N, 4]); dtype float32 or
    bfloat16.  A slot outside the memory reads as 0."""
    torch = _torch()
    d, hkv, dim = _memory_descriptor(memory)
    like = memory[0]
    n = _slots(slots, like)
    dtype = dtype or torch.float32
    if dtype not in (torch.float32, torch.bfloat16):
        raise TypeError("only float32 and bfloat16 tensors are supported, got %s" % dtype)
    with _Call(like, stream) as c:
        k, v = c.empty((n, hkv, dim), dtype), c.empty((n, hkv, dim), dtype)
        boxes = c.empty((n, 4), torch.float32)
        check(lib().box_memory_read(d, slots.data_ptr(), n, k.data_ptr(), v.data_ptr(),
                                    int(dtype == torch.bfloat16) * RE_DTYPE_BF16,
                                    boxes.data_ptr(), c.stream), "box_memory_read")
    return k, v, boxes


def box_memory_attn_fwd(q, memory: Sequence, pages, lengths, *, scale: Optional[float] = None,
                        q_boxes=None, bias=None, first_exp: int = -4, octave_steps: int = 1,
                        q_len=None, save: bool = False, out=None, lse=None, workspace=None,
                        stream=None):
    """Attention of q [B, Nq, H, D] over what each stream remembers: the first lengths[b]
    places of the memory's pages[b] (int32 [B, max_pages]).  Returns (out, lse); lse is made
    where `save` is true or it is given, else None."""
    torch = _torch()
    m, hkv, dim = _memory_descriptor(memory)
    qs = _rows4(q, "q")
    B, nq, H, D = q.shape
    if D != dim:
        raise ValueError("q has %d channels a head, the memory %d" % (D, dim))
    if H % hkv:
        raise ValueError("the memory's %d heads must divide q's %d" % (hkv, H))
    code = _dtype_code(q)
    if pages.dim() != 2:
        raise ValueError("pages must be 2-D [batch, max_pages]")
    _dense(pages, (B, pages.shape[1]), "pages", torch.int32)
    _dense(lengths, (B,), "lengths", torch.int32)
    if q_len is not None:
        _lengths(q_len, B, "q_len")
    n = _bias(bias, H)
    strides = (0, 0)
    if n:
        strides = _boxes(q_boxes, B, nq, "q_boxes")
    else:
        q_boxes = None
    if out is not None:
        _dense(out, q.shape, "out", q.dtype)
    if lse is not None:
        _dense(lse, (B, H, nq), "lse", torch.float32)
    _need_cuda(q, "q", memory[0])
    _same_device(q, "pages lengths q_len bias q_boxes out lse",
                 (pages, lengths, q_len, bias, q_boxes, out, lse))
    if workspace is not None:
        binding._workspace(workspace, q)
        _same_device(q, "workspace", (workspace,))
    d = _RECALL.pack(q.data_ptr(), code, H, B, nq, pages.shape[1], *qs[:3],
                     D ** -0.5 if scale is None else scale, n, first_exp, octave_steps,
                     _ptr(bias), _ptr(q_boxes), *strides, _ptr(q_len), pages.data_ptr(),
                     lengths.data_ptr())
    L = lib()
    with _Call(q, stream) as c:
        if out is None:
            out = c.empty((B, nq, H, D), q.dtype)
        if save and lse is None:
            lse = c.empty((B, H, nq), torch.float32)
        need = 0
        if workspace is None:
            need = _size(L.box_memory_attn_workspace_size, "box_memory_attn_workspace_size", m, d)
        ws, wsb, _keep = c.workspace(workspace, need)
        check(L.box_memory_attn_fwd(m, d, out.data_ptr(), _ptr(lse), ws, wsb, c.stream),
              "box_memory_attn_fwd")
    return out, lse


# ---------------------------------------------------------------------------
# Gated norms
# ---------------------------------------------------------------------------

def _norm_descriptor(x, branch, gate, alpha, post_weight, post_bias, pre_weight, pre_bias, norm,
                     eps):
    torch = _torch()
    if norm not in NORMS:
        raise ValueError("norm must be one of %s" % sorted(NORMS))
    if x.dim() != 2:
        raise ValueError("x must be 2-D [rows, channels] (got %s)" % (tuple(x.shape),))
    m, c = shape = x.shape
    code = _dtype_code(x)
    strides, bstrides = x.stride(), (0, 1)
    if branch is not None:
        if branch.shape != shape or branch.dtype != x.dtype:
            raise ValueError("branch must be a %s tensor of shape %s (got %s %s)"
                             % (x.dtype, (m, c), branch.dtype, tuple(branch.shape)))
        bstrides = branch.stride()
    if (strides[1] != 1 or bstrides[1] != 1) and c > 1 and m > 0:
        raise ValueError("the channels of x and branch must be adjacent")
    gates = 0
    if gate is not None:
        if branch is None:
            raise ValueError("a gate needs a branch")
        gates = gate.shape[0] if gate.dim() == 2 else -1
        if gates < 0 or (gates == 0 and m > 0) or (gates > 0 and m % gates):
            raise ValueError("gate must be [gates, channels] with gates dividing the %d rows" % m)
        _dense(gate, (gates, c), "gate", torch.float32)
    params = (post_weight, post_bias, pre_weight, pre_bias)
    for t, name in zip(params, ("post_weight", "post_bias", "pre_weight", "pre_bias")):
        if t is not None:
            _dense(t, (c,), name, torch.float32)
    _need_cuda(x, "x")
    _same_device(x, "branch gate post_weight post_bias pre_weight pre_bias",
                 (branch, gate, post_weight, post_bias, pre_weight, pre_bias))
    return _NORM.pack(x.data_ptr(), _ptr(branch), strides[0], bstrides[0], code, NORMS[norm], m, c,
                      alpha, eps, gates, _ptr(gate), *map(_ptr, params))


def gated_norm_fwd(x, branch=None, *, gate=None, alpha: float = 1.0, post_weight=None,
                   post_bias=None, pre_weight=None, pre_bias=None, norm: str = "rms",
                   eps: float = 1e-6, second: bool = True, save: bool = False, y=None, u=None,
                   stats=None, stream=None):
    """y = x + alpha * gate * N1(branch), u = N2(y) over the rows of x [rows, channels].
    gate: float32 [gates, channels], one row for each of `gates` equal runs of rows; weights
    and biases float32 [channels] or None (1 and 0); norm "rms" or "layer"; second=False leaves
    N2 out.  Returns (y, u, stats); without a branch y is x; stats float32 [rows, 4] is made
    where `save` is true or it is given, else None."""
    torch = _torch()
    d = _norm_descriptor(x, branch, gate, alpha, post_weight, post_bias, pre_weight, pre_bias, norm,
                         eps)
    m, ch = x.shape
    if branch is None and not second and y is None:
        raise ValueError("neither a branch nor the second norm: nothing to do")
    for t, name in ((y, "y"), (u, "u")):
        if t is not None:
            _dense(t, (m, ch), name, x.dtype)
    if u is not None and not second:
        raise ValueError("u without the second norm")
    if stats is not None:
        _dense(stats, (m, 4), "stats", torch.float32)
    _same_device(x, "y u stats", (y, u, stats))
    with _Call(x, stream) as c:
        if y is None and branch is not None:
            y = c.empty((m, ch), x.dtype)
        if u is None and second:
            u = c.empty((m, ch), x.dtype)
        if stats is None and save:
            stats = c.empty((m, 4), torch.float32)
        check(lib().gated_norm_fwd(d, _ptr(y), _ptr(u), _ptr(stats), c.stream), "gated_norm_fwd")
    return x if y is None else y, u, stats


def gated_norm_bwd(grad_y, grad_u, x, branch, stats, *, gate=None, alpha: float = 1.0,
                   post_weight=None, post_bias=None, pre_weight=None, pre_bias=None,
                   norm: str = "rms", eps: float = 1e-6, workspace=None, stream=None):
    """Gradients of gated_norm_fwd for upstream grad_y and grad_u (contiguous, either may be
    None); stats as it returned them.  Returns (grad_x, grad_branch, grad_gate,
    grad_post_weight, grad_post_bias, grad_pre_weight, grad_pre_bias), None for what was not
    given to the forward."""
    torch = _torch()
    d = _norm_descriptor(x, branch, gate, alpha, post_weight, post_bias, pre_weight, pre_bias, norm,
                         eps)
    m, ch = x.shape
    for t, name in ((grad_y, "grad_y"), (grad_u, "grad_u")):
        if t is not None:
            _dense(t, (m, ch), name, x.dtype)
    _dense(stats, (m, 4), "stats", torch.float32)
    _same_device(x, "grad_y grad_u stats", (grad_y, grad_u, stats))
    if workspace is not None:
        binding._workspace(workspace, x)
        _same_device(x, "workspace", (workspace,))
    L = lib()
    with _Call(x, stream) as c:
        gx = c.empty((m, ch), x.dtype)
        gb = None if branch is None else c.empty((m, ch), x.dtype)
        params = (gate, post_weight, post_bias, pre_weight, pre_bias)
        if branch is None:
            params = (None, None, None, pre_weight, pre_bias)
        sizes = [0 if p is None else p.numel() for p in params]
        # parts of one buffer (all of them begin at 16 bytes where ch is a multiple of 4, and where
        # it is not the kernels ask for no alignment)
        small = [None] * 5
        if any(sizes):
            parts = c.empty((sum(sizes),), torch.float32).split_with_sizes(sizes)
            small = [None if p is None else t if p.dim() == 1 else t.view(p.shape)
                     for p, t in zip(params, parts)]
        need = 0
        if workspace is None:
            need = _size(L.gated_norm_workspace_size, "gated_norm_workspace_size", d)
        ws, wsb, _keep = c.workspace(workspace, need)
        check(L.gated_norm_bwd(d, _ptr(grad_y), _ptr(grad_u), stats.data_ptr(),
                               _GRADS.pack(gx.data_ptr(), _ptr(gb), *map(_ptr, small)), ws, wsb,
                               c.stream), "gated_norm_bwd")
    return (gx, gb, *small)
