"""Layer operators and gradient clipping: the entry points of include/ssd_layers.h for torch tensors.

Argument marshalling only, as in `binding`: the arithmetic runs in the CUDA library, and there is no fallback.
Outputs that are not given are allocated by torch and returned; the workspace of a call, unless one is given,
comes from torch's caching allocator on the stream that the call runs on.

    y, z = ssd_linear_forward(x, weight, bias=b, act=SSD_ACT_GELU, keep=True)
    dx, dw, db = ssd_linear_backward(dy, x, weight, z, act=SSD_ACT_GELU, dweight=arena_view, dbias=arena_view2)
    clip = GradList(arenas, groups=range(K)); norms = ssd_clip_grad_norm(clip, 1.0)

Activations x, y, z, ... may have leading dimensions that flatten to rows; weights are [out, in] as
torch.nn.Linear has them.  The last dimension is contiguous, rows may be strided.

Autograd does not see these calls: inputs that require gradients are taken as they are, and outputs have no history.  Gradients come from the
backward calls.
"""
from __future__ import annotations

import contextlib
import ctypes as C
from typing import Optional, Sequence

import torch

from . import binding as B
from .binding import SSD_BF16, SSD_F32, SsdError

SSD_ACT_NONE, SSD_ACT_RELU, SSD_ACT_GELU, SSD_ACT_SILU = range(4)
ACTS = {"none": SSD_ACT_NONE, "relu": SSD_ACT_RELU, "gelu": SSD_ACT_GELU, "silu": SSD_ACT_SILU}
SSD_NONFINITE_KEEP, SSD_NONFINITE_ZERO = 0, 1

_DTYPES = {torch.float32: SSD_F32, torch.bfloat16: SSD_BF16}

EXPORTS = (
    "ssd_linear_forward_workspace", "ssd_linear_backward_workspace", "ssd_gated_forward_workspace", "ssd_gated_backward_workspace",
    "ssd_linear_forward", "ssd_linear_backward", "ssd_gated_forward", "ssd_gated_backward",
    "ssd_grad_list_bytes", "ssd_grad_list_create", "ssd_grad_list_destroy", "ssd_clip_grad_norm", "ssd_grad_norm",
    "ssd_layer_error", "ssd_layer_cuda_error", "ssd_layer_launches",
)


def _struct(name: str, ints: str, mats: str):
    """`mats`: members in order; a leading '*' marks one without a row pitch."""
    fields = [(n, C.c_int64) for n in ("rows", "in_features", "out_features")] + [(n, C.c_int32) for n in ints.split()]
    for m in mats.split():
        fields.append((m.lstrip("*").split(":")[0], C.c_void_p))
        if not m.startswith("*"):
            fields.append((m.split(":")[1], C.c_int64))
    return type(name, (C.Structure,), {"_fields_": fields})


ssd_linear_fwd = _struct("ssd_linear_fwd", "dtype act", "x:ldx weight:ldw *bias residual:ldr y:ldy z:ldz")
ssd_linear_bwd = _struct("ssd_linear_bwd", "dtype act grad_dtype reserved", "dy:lddy x:ldx weight:ldw z:ldz dx:lddx dweight:lddw *dbias")
ssd_gated_fwd = _struct("ssd_gated_fwd", "dtype act", "x:ldx w_gate:ldwg w_up:ldwu *b_gate *b_up h:ldh gate:ldgate up:ldup")
ssd_gated_bwd = _struct("ssd_gated_bwd", "dtype act grad_dtype reserved",
                        "dh:lddh x:ldx w_gate:ldwg w_up:ldwu gate:ldgate up:ldup dx:lddx dw_gate:lddwg dw_up:lddwu *db_gate *db_up")

_lib = None


def lib() -> C.CDLL:
    """The library with the signatures of include/ssd_layers.h set; raises if it has not been built."""
    global _lib
    if _lib is None:
        L = B.lib()
        P, vp, i32, i64 = C.POINTER, C.c_void_p, C.c_int32, C.c_int64
        for op, args in (("linear_forward", ssd_linear_fwd), ("linear_backward", ssd_linear_bwd),
                         ("gated_forward", ssd_gated_fwd), ("gated_backward", ssd_gated_bwd)):
            fn = getattr(L, f"ssd_{op}_workspace")
            fn.restype, fn.argtypes = i32, [P(args), vp]
            fn = getattr(L, f"ssd_{op}")
            fn.restype, fn.argtypes = i32, [P(args), vp, i64, vp]
        sigs = {
            "ssd_grad_list_bytes": (i32, [i32, P(i64), i32, P(i64)]),
            "ssd_grad_list_create": (i32, [P(vp), i32, P(i64), P(i32), i32, P(vp), i32, P(vp), i32, vp, i64, vp]),
            "ssd_grad_list_destroy": (None, [vp]),
            "ssd_clip_grad_norm": (i32, [vp, C.c_float, i32, vp, vp]),
            "ssd_grad_norm": (i32, [vp, vp, vp]),
            "ssd_layer_error": (i32, [P(i32)]),
            "ssd_layer_cuda_error": (C.c_char_p, []),
            "ssd_layer_launches": (i64, []),
        }
        for name, (res, args) in sigs.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _lib = L
    return _lib


def _check(st: int, where: str):
    if st != B.SSD_OK:
        raise SsdError(st, where, lib().ssd_layer_cuda_error().decode() if st == B.SSD_ERR_CUDA else "")


def _fail(where: str, what: str):
    raise SsdError(B.SSD_ERR_ARG, where, what)


_torch = None


def _marshal():
    """The compiled marshalling module (csrc/ssd_torch.cpp), told where the entry points are."""
    global _torch
    if _torch is None:
        L = lib()
        from . import _ssd_torch
        _ssd_torch.setup(SsdError, {name: C.cast(getattr(L, name), C.c_void_p).value for name in EXPORTS}, torch.OutOfMemoryError)
        _torch = _ssd_torch
    return _torch


def _on(stream):
    """Calls run, and take outputs and workspace, on the current stream; another one is made current for the call."""
    return torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(stream)))


def _grad_code(where: str, dtype) -> int:
    if dtype is None:
        return SSD_F32
    if dtype not in _DTYPES:
        _fail(where, "weight gradients are float32 or bfloat16")
    return _DTYPES[dtype]


def ssd_linear_forward(x, weight, y=None, bias=None, residual=None, z=None, act: int = SSD_ACT_NONE, keep: bool = False,
                       workspace=None, stream=None):
    """y = act(x weight^T + bias) + residual.  Returns (y, z); z, the pre-activation, is given or kept on request, else None."""
    if stream is not None:
        with _on(stream):
            return ssd_linear_forward(x, weight, y, bias, residual, z, act, keep, workspace)
    return (_torch or _marshal()).linear_forward(x, weight, y, bias, residual, z, act, True if keep else False, workspace)


def ssd_linear_backward(dy, x, weight, z=None, act: int = SSD_ACT_NONE, dx=None, dweight=None, dbias=None, grad_dtype=None,
                        want_dx: bool = True, want_dweight: bool = True, bias: bool = True, workspace=None, stream=None):
    """Gradients of ssd_linear_forward: (dx, dweight, dbias).  dweight and dbias have the type of the tensors given for them (views of a
    gradient arena), else `grad_dtype` (float32).  want_dx, want_dweight, bias: which of them to compute where none is given."""
    if stream is not None:
        with _on(stream):
            return ssd_linear_backward(dy, x, weight, z, act, dx, dweight, dbias, grad_dtype, want_dx, want_dweight, bias, workspace)
    return (_torch or _marshal()).linear_backward(dy, x, weight, z, act, dx, dweight, dbias, _grad_code("ssd_linear_backward", grad_dtype),
                                                  True if want_dx else False, True if want_dweight else False, True if bias else False, workspace)


def ssd_gated_forward(x, w_gate, w_up, b_gate=None, b_up=None, h=None, gate=None, up=None, act: int = SSD_ACT_SILU,
                      keep: bool = False, workspace=None, stream=None):
    """h = act(x w_gate^T + b_gate) * (x w_up^T + b_up).  Returns (h, gate, up); gate and up, which the backward pass needs, are
    given or kept on request, else None."""
    if stream is not None:
        with _on(stream):
            return ssd_gated_forward(x, w_gate, w_up, b_gate, b_up, h, gate, up, act, keep, workspace)
    return (_torch or _marshal()).gated_forward(x, w_gate, w_up, b_gate, b_up, h, gate, up, act, True if keep else False, workspace)


def ssd_gated_backward(dh, x, w_gate, w_up, gate, up, act: int = SSD_ACT_SILU, dx=None, dw_gate=None, dw_up=None, db_gate=None,
                       db_up=None, grad_dtype=None, want_dx: bool = True, want_dweight: bool = True, bias: bool = True,
                       workspace=None, stream=None):
    """Gradients of ssd_gated_forward: (dx, dw_gate, dw_up, db_gate, db_up); types and choices as for ssd_linear_backward."""
    if stream is not None:
        with _on(stream):
            return ssd_gated_backward(dh, x, w_gate, w_up, gate, up, act, dx, dw_gate, dw_up, db_gate, db_up, grad_dtype, want_dx,
                                      want_dweight, bias, workspace)
    return (_torch or _marshal()).gated_backward(dh, x, w_gate, w_up, gate, up, act, dx, dw_gate, dw_up, db_gate, db_up,
                                                 _grad_code("ssd_gated_backward", grad_dtype), True if want_dx else False,
                                                 True if want_dweight else False, True if bias else False, workspace)


class GradList:
    """The tensors that are clipped together, made once for buffers that are used again and again.

    grads: contiguous tensors of one type; out: where the clipped gradients go (None = in place); groups: the
    group of every tensor, ascending (None = one group); e.g. a worker's arena each, with groups=range(K).

    Making one costs about a microsecond of host time a tensor and waits for the copy of its table: worth it for arenas that live as long as
    the training, not for gradients that are allocated anew each step.  A list outlives the CUDA graphs that its calls were captured into.
    Calls on one list must not overlap on the GPU; they may run on any stream."""

    def __init__(self, grads: Sequence[torch.Tensor], out: Optional[Sequence[torch.Tensor]] = None,
                 groups: Optional[Sequence[int]] = None, num_groups: Optional[int] = None, stream=None):
        where = "ssd_grad_list_create"
        self._h, self.address = C.c_void_p(), 0
        grads = list(grads)
        out = grads if out is None else list(out)
        groups = None if groups is None else [int(g) for g in groups]
        if not grads or len(out) != len(grads) or (groups is not None and len(groups) != len(grads)):
            _fail(where, "needs at least one tensor, and as many destinations and group numbers")
        self.device, self.num_groups = grads[0].device, int(num_groups or (1 if groups is None else max(groups) + 1))
        for ts in (grads, out):
            if any(t.dtype != ts[0].dtype or t.device != self.device or not t.is_contiguous() for t in ts):
                _fail(where, "tensors are contiguous, on one device and of one type")
        if not -1 << 31 <= self.num_groups < 1 << 31 or (groups is not None and not all(-1 << 31 <= g < 1 << 31 for g in groups)):
            _fail(where, "group numbers are integers of 32 bits")
        if any(a.numel() != b.numel() for a, b in zip(grads, out)):
            _fail(where, "a destination has another size")
        if not grads[0].is_cuda or grads[0].dtype not in _DTYPES or out[0].dtype not in _DTYPES:
            _fail(where, "needs float32 or bfloat16 CUDA tensors")
        T = len(grads)
        numel = (C.c_int64 * T)(*[t.numel() for t in grads])
        need = C.c_int64()
        _check(lib().ssd_grad_list_bytes(T, numel, self.num_groups, C.byref(need)), "ssd_grad_list_bytes")
        # the table's memory comes from the stream that fills it, so that nothing still under way elsewhere has it
        with torch.cuda.device(self.device), contextlib.nullcontext() if stream is None else _on(stream):
            if torch.cuda.current_device() != self.device.index:
                _fail(where, "the stream belongs to another device")
            self._keep = (grads, out)
            self.table, self.home = torch.empty(need.value, dtype=torch.uint8, device=self.device), torch.cuda.current_stream().cuda_stream
            _check(lib().ssd_grad_list_create(
                C.byref(self._h), T, numel, None if groups is None else (C.c_int32 * T)(*groups), self.num_groups,
                (C.c_void_p * T)(*[t.data_ptr() for t in grads]), _DTYPES[grads[0].dtype],
                (C.c_void_p * T)(*[t.data_ptr() for t in out]), _DTYPES[out[0].dtype],
                self.table.data_ptr(), need.value, self.home), where)
        self.address = self._h.value

    def ssd_grad_list_destroy(self):
        if self._h:
            lib().ssd_grad_list_destroy(self._h)
            self._h, self.address = C.c_void_p(), 0          # calls with the list are refused from here on

    def __del__(self):
        try:
            self.ssd_grad_list_destroy()
        except Exception:
            pass


def ssd_clip_grad_norm(grads: GradList, max_norm: float, nonfinite: int = SSD_NONFINITE_KEEP, norms=None, stream=None):
    """Scales every group by min(1, max_norm / (norm + 1e-6)) and returns the norms before the scaling (one float32 per group, on the device)."""
    if stream is not None:
        with _on(stream):
            return ssd_clip_grad_norm(grads, max_norm, nonfinite, norms)
    return (_torch or _marshal()).clip(grads.address, grads.device.index, grads.num_groups, max_norm, nonfinite, norms, grads.table, grads.home)


def ssd_grad_norm(grads: GradList, norms=None, stream=None):
    """The norms alone; no gradient is written."""
    if stream is not None:
        with _on(stream):
            return ssd_grad_norm(grads, norms)
    return (_torch or _marshal()).clip(grads.address, grads.device.index, grads.num_groups, None, 0, norms, grads.table, grads.home)


def ssd_layer_error() -> int:
    out = C.c_int32()
    _check(lib().ssd_layer_error(C.byref(out)), "ssd_layer_error")
    return out.value


def ssd_layer_launches() -> int:
    return lib().ssd_layer_launches()
