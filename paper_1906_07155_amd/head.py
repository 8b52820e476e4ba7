"""Thin ctypes binding of include/box_head.h (argument marshalling only): dense layers with
their epilogue, and the log probabilities of classes.

As in `relation`, every operation runs in the library's HIP kernels on torch's current stream
(or `stream`), and nothing falls back; descriptors are packed in one go into bytes.

Paper anchors (MMDetection, arXiv 1906.07155): §3.1 RoIHead, §3.2 losses.
"""
from __future__ import annotations

import ctypes
import os
import re
import struct
from typing import List

from . import binding
from .binding import RE_ERR_WORKSPACE, _dtype_code, _need_cuda, _torch, check
from .relation import _Call, _dense, _ptr, _same_device, _size

HEADER = os.path.join(os.path.dirname(binding.HERE), "include", "box_head.h")

ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}      # RE_ACT_*

_VP, _I32, _SZ, _D = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t, ctypes.c_char_p
_SZP = ctypes.POINTER(_SZ)

SIGNATURES = {
    "linear_act_workspace_size": [_D, _I32, _SZP],
    "linear_act_fwd": [_D, _VP, _VP, _VP, _SZ, _VP],
    "linear_act_bwd": [_D, _VP, _VP, _VP, _VP, _VP, _VP, _VP, _SZ, _VP],
    "class_logprob_workspace_size": [_D, _SZP],
    "class_logprob_fwd": [_D, _VP, _VP, _VP, _VP, _VP, _VP, _SZ, _VP],
    "class_logprob_bwd": [_D, _VP, _VP, _VP, _VP, _VP, _VP],
}

# linear_act_t, class_logprob_t
_LINEAR = struct.Struct("@4P6q3i4x")
_LOGPROB = struct.Struct("@2P3q2if4x")
MAX_TOP = 16                        # RE_LOGPROB_MAX_TOP
LOGPROB_SPAN = 4088                 # rows of more classes come in parts, which need a workspace

_lib = None


def header_functions() -> List[str]:
    """Names of the functions include/box_head.h declares."""
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
# Dense layers
# ---------------------------------------------------------------------------

def _matrix(t, shape, name: str, dtype):
    """The row stride of a 2-D tensor with adjacent columns."""
    if t.shape != shape or t.dtype != dtype:
        raise ValueError("%s must be a %s tensor of shape %s (got %s %s)"
                         % (name, dtype, tuple(shape), t.dtype, tuple(t.shape)))
    row, column = t.stride()
    if column != 1 and shape[1] > 1 and shape[0] > 0:
        raise ValueError("the columns of %s must be adjacent" % name)
    return row


def _linear_descriptor(x, weight, bias, act, residual):
    torch = _torch()
    if act not in ACTS:
        raise ValueError("act must be one of %s (got %r)" % (sorted(ACTS), act))
    if x.dim() != 2 or weight.dim() != 2:
        raise ValueError("x must be 2-D [rows, ins] and weight 2-D [outs, ins] (got %s, %s)"
                         % (tuple(x.shape), tuple(weight.shape)))
    m, k = x.shape
    n = weight.shape[0]
    dtype = x.dtype
    code = _dtype_code(x)
    xs, ws, rs = _matrix(x, (m, k), "x", dtype), _matrix(weight, (n, k), "weight", dtype), 0
    bias_code = 0
    if bias is not None:
        if bias.dtype != dtype:
            _dense(bias, (n,), "bias", torch.float32)
        else:
            _dense(bias, (n,), "bias", dtype)
            bias_code = code
    if residual is not None:
        rs = _matrix(residual, (m, n), "residual", dtype)
    _need_cuda(x, "x")
    _same_device(x, "weight bias residual", (weight, bias, residual))
    return _LINEAR.pack(x.data_ptr(), weight.data_ptr(), _ptr(bias), _ptr(residual), xs, ws, rs, m, k, n,
                        code, bias_code, ACTS[act])


def linear_act_workspace_size(x, weight, bias=None, backward: bool = False, *, act: str = "none") -> int:
    """Workspace bytes of linear_act_fwd (or of linear_act_bwd where `backward`) for these tensors."""
    d = _linear_descriptor(x, weight, bias, act, None)
    return _size(lib().linear_act_workspace_size, "linear_act_workspace_size", d, int(backward))


def _slope(x, shape):
    """Shape and type of a layer's slopes: 24 bits each beside bf16 data."""
    torch = _torch()
    if x.dtype == torch.bfloat16:
        return (3 * shape[0] * shape[1],), torch.uint8
    return shape, torch.float32


def linear_act_fwd(x, weight, bias=None, *, act: str = "none", residual=None, save: bool = False, out=None,
                   workspace=None, stream=None):
    """y = act(x weight^T + bias) + residual of x [rows, ins] and weight [outs, ins] (one dtype, rows
    may be strided), bias [outs] of that dtype or float32, act "none", "relu", "gelu" or "silu",
    residual [rows, outs].  `out` may be the residual's memory and none of the others'.  Returns
    (y, saved): saved, made where `save` is true, is what the backward takes: None without an
    activation, y itself for relu without a residual, else the activation's slopes."""
    d = _linear_descriptor(x, weight, bias, act, residual)
    shape = (x.shape[0], weight.shape[0])
    if out is not None:
        _dense(out, shape, "out", x.dtype)
        _same_device(x, "out", (out,))
    if workspace is not None:
        binding._workspace(workspace, x)
        _same_device(x, "workspace", (workspace,))
    L = lib()
    with _Call(x, stream) as c:
        if out is None:
            out = c.empty(shape, x.dtype)
        saved = slope = None
        if save and act != "none":
            if act == "relu" and residual is None:
                saved = out
            else:
                saved = slope = c.empty(*_slope(x, shape))
        ws, wsb, _keep = c.workspace(workspace, 0)
        status = L.linear_act_fwd(d, out.data_ptr(), _ptr(slope), ws, wsb, c.stream)
        if status == RE_ERR_WORKSPACE and workspace is None:       # (most calls need none: not asked first)
            need = _size(L.linear_act_workspace_size, "linear_act_workspace_size", d, 0)
            ws, wsb, _keep = c.workspace(None, need)
            status = L.linear_act_fwd(d, out.data_ptr(), _ptr(slope), ws, wsb, c.stream)
        check(status, "linear_act_fwd")
    return out, saved


def linear_act_bwd(grad_y, x, weight, saved=None, *, bias=None, act: str = "none", want_x: bool = True,
                   want_weight: bool = True, want_bias: bool = True, workspace=None, stream=None):
    """Gradients of linear_act_fwd for upstream grad_y (contiguous [rows, outs]); saved as it
    returned it.  Returns (grad_x, grad_weight, grad_bias), None for what is not wanted or (bias)
    was not given; the residual's gradient is grad_y."""
    torch = _torch()
    d = _linear_descriptor(x, weight, bias, act, None)
    shape = (x.shape[0], weight.shape[0])
    _dense(grad_y, shape, "grad_y", x.dtype)
    slope = y = None
    if act == "none":
        if saved is not None:
            raise ValueError("saved without an activation")
    else:
        if saved is None:
            raise ValueError("%s needs what the forward saved" % act)
        if act == "relu" and saved.dtype == x.dtype:
            y = _dense(saved, shape, "saved", x.dtype)
        else:
            like, dtype = _slope(x, shape)
            slope = _dense(saved, like, "saved", dtype)
    _same_device(x, "grad_y saved", (grad_y, saved))
    if workspace is not None:
        binding._workspace(workspace, x)
        _same_device(x, "workspace", (workspace,))
    L = lib()
    with _Call(x, stream) as c:
        gx = c.empty(x.shape, x.dtype) if want_x else None
        gw = c.empty(weight.shape, x.dtype) if want_weight else None
        gb = c.empty(bias.shape, bias.dtype) if want_bias and bias is not None else None
        need = 0
        if workspace is None:
            need = _size(L.linear_act_workspace_size, "linear_act_workspace_size", d, 1)
        ws, wsb, _keep = c.workspace(workspace, need)
        check(L.linear_act_bwd(d, grad_y.data_ptr(), _ptr(slope), _ptr(y), _ptr(gx), _ptr(gw), _ptr(gb), ws, wsb,
                               c.stream), "linear_act_bwd")
    return gx, gw, gb


# ---------------------------------------------------------------------------
# Log probabilities of classes
# ---------------------------------------------------------------------------

def _logprob_descriptor(logits, labels, scale, top):
    torch = _torch()
    if logits.dim() != 2 or logits.shape[1] < 1:
        raise ValueError("logits must be 2-D [rows, classes] (got %s)" % (tuple(logits.shape),))
    m, c = logits.shape
    code = _dtype_code(logits)
    stride, column = logits.stride()
    if column != 1 and c > 1 and m > 0:
        raise ValueError("the classes of logits must be adjacent")
    if not 0 <= top <= min(c, MAX_TOP):
        raise ValueError("top must be in [0, %d] (got %d)" % (min(c, MAX_TOP), top))
    _dense(labels, (m,), "labels", torch.int64)
    _need_cuda(logits, "logits")
    _same_device(logits, "labels", (labels,))
    return _LOGPROB.pack(logits.data_ptr(), labels.data_ptr(), stride, m, c, code, top, scale)


def class_logprob_fwd(logits, labels, *, scale: float = 1.0, top: int = 0, out=None, workspace=None, stream=None):
    """Log probabilities over logits [rows, classes] times `scale`: returns (logp, entropy,
    stats, top_logp, top_index): float32 [rows] of the labels (int64 [rows]; one outside the classes is
    not counted: 0) and of the entropy; stats float32 [rows, 2], which the backward takes, the
    largest of a row and the log sum relative to it; float32 and int64 [rows, top] of the `top` classes
    with the largest logits, the lower class first among equals (None where top is 0).  out: (logp,
    entropy, stats) to write."""
    torch = _torch()
    d = _logprob_descriptor(logits, labels, scale, top)
    if workspace is not None:
        binding._workspace(workspace, logits)
        _same_device(logits, "workspace", (workspace,))
    m, c = logits.shape
    if out is not None:
        for t, shape, name in zip(out, ((m,), (m,), (m, 2)), ("logp", "entropy", "stats")):
            _dense(t, shape, name, torch.float32)
        _same_device(logits, "logp entropy stats", out)
    L = lib()
    with _Call(logits, stream) as call:
        if out is None:
            # (parts of one buffer, an allocation costs more than a part, and to autograd tensors of their
            # own, which may be written to)
            logp, entropy, stats = torch.unsafe_split_with_sizes(call.empty((4 * m,), torch.float32), (m, m, 2 * m))
            stats = stats.view(m, 2)
        else:
            logp, entropy, stats = out
        top_logp = top_index = None
        if top:
            top_logp, top_index = call.empty((m, top), torch.float32), call.empty((m, top), torch.int64)
        need = 0
        if workspace is None and c > LOGPROB_SPAN:
            need = _size(L.class_logprob_workspace_size, "class_logprob_workspace_size", d)
        ws, wsb, _keep = call.workspace(workspace, need)
        check(L.class_logprob_fwd(d, logp.data_ptr(), entropy.data_ptr(), stats.data_ptr(), _ptr(top_logp),
                                  _ptr(top_index), ws, wsb, call.stream), "class_logprob_fwd")
    return logp, entropy, stats, top_logp, top_index


def class_logprob_bwd(grad_logp, grad_entropy, logits, labels, stats, entropy, *, scale: float = 1.0, stream=None):
    """Gradient of the logits ([rows, classes] of their dtype) for upstream grad_logp and grad_entropy
    (float32 [rows], either may be None); stats and entropy as class_logprob_fwd returned them."""
    torch = _torch()
    d = _logprob_descriptor(logits, labels, scale, 0)
    m, c = logits.shape
    _dense(stats, (m, 2), "stats", torch.float32)
    for t, name in ((grad_logp, "grad_logp"), (grad_entropy, "grad_entropy"), (entropy, "entropy")):
        if t is not None:
            _dense(t, (m,), name, torch.float32)
    _same_device(logits, "grad_logp grad_entropy stats entropy", (grad_logp, grad_entropy, stats, entropy))
    with _Call(logits, stream) as call:
        grad = call.empty((m, c), logits.dtype)
        check(lib().class_logprob_bwd(d, _ptr(grad_logp), _ptr(grad_entropy), stats.data_ptr(), entropy.data_ptr(),
                                      grad.data_ptr(), call.stream), "class_logprob_bwd")
    return grad
