"""Operators of the temporal head behind a rollout (the sr_microscale_*, sr_rms_norm and sr_linear_attention_* calls of include/sr_rollout.h).

Argument marshalling only, like `Graph`, and a call's common case in compiled code (csrc/sr_python.cpp; what that does not take comes back
here to be done or refused): tensors live on a CUDA device, work goes to the current stream of that device, outputs and
workspaces come from PyTorch's allocator, and every refusal is an `SrError`.  There are no derivatives: a tensor that
requires a gradient is refused while gradients are recorded, one with a tangent always.

  quantize, Microscaled, product   matrices in groups of 32 with a scale each, 4 ("mx4") or 8 ("mx8") bits per element; a dense node's update
  rms_norm                         root-mean-square norm with the residual's addition, output in full or microscaled
  linear_attention_run, _step      linear attention with a decay for each head: whole clips, single frames
  TemporalHead                     norm, product, attention and product as one head on the features of a rollout (`Graph.rollout(frames, head=...)`)
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional

import torch

from torch.autograd import forward_ad as _forward_ad

from . import binding
from .binding import SrError

binding.load_library()
try:
    from . import _operators as _compiled
except ImportError as _first:                          # not built yet, or for another PyTorch or Python
    from . import build as _build
    try:
        _build.build_extension()
        from . import _operators as _compiled
    except Exception as _second:
        raise ImportError("the operators' extension cannot be loaded (%s) and building it failed (%s)" % (_first, _second)) from _second

FORMATS = {"mx8": 2, "mx4": 3}
_DTYPES = {torch.float32: 0, torch.bfloat16: 1}


class _Strides(ctypes.Structure):
    _fields_ = [("frame", ctypes.c_int64), ("sequence", ctypes.c_int64), ("head", ctypes.c_int64)]


class _AttentionDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "batch", "heads", "groups", "dk", "dv")] + [("frames", ctypes.c_int64), ("scale", ctypes.c_float)] + \
        [(n, _Strides) for n in ("q", "k", "v", "out", "log_decay")]


class _ProductPlan(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("rows", "outs", "parts", "pair")]


class _AttentionPlan(ctypes.Structure):
    _fields_ = [("chunk", ctypes.c_int32), ("segment", ctypes.c_int64), ("segments", ctypes.c_int64)]


_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = binding.load_library()
        vp, i32, i64, size = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.POINTER(ctypes.c_size_t)
        desc = ctypes.POINTER(_AttentionDesc)
        for name, args in {
            "sr_microscale_bytes": [i64, i64, i32, size, size],
            "sr_microscale_quantize": [vp, i32, i64, i64, i64, i32, vp, vp, vp],
            "sr_microscale_values": [vp, vp, i32, i64, i64, vp, vp],
            "sr_microscale_product": [vp, vp, vp, vp, i32, i64, i64, i64, vp, i32, vp, i32, i64, vp],
            "sr_microscale_product_plan": [i32, i64, i64, i64, i32, ctypes.POINTER(_ProductPlan)],
            "sr_linear_attention_plan": [desc, i32, i32, ctypes.POINTER(_AttentionPlan)],
            "sr_rms_norm": [vp, vp, vp, ctypes.c_float, i32, i64, i64, i64, i64, vp, vp, i32, vp, vp],
            "sr_linear_attention_workspace_bytes": [desc, i32, size],
            "sr_linear_attention_run": [desc, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp],
            "sr_linear_attention_step": [desc, vp, vp, vp, vp, vp, vp, vp],
            "sr_operator_status": [vp],
            "sr_operator_reset": [vp],
        }.items():
            f = getattr(lib, name)
            f.argtypes, f.restype = args, i32
        _lib = lib
    return _lib


def _refuse(call: str, why: str):
    raise SrError(1, "%s: %s" % (call, why))


# The current device and a device's current stream without the objects around them (a call's host time is a few microseconds).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", None)
_grad = torch.is_grad_enabled
_wrapped = torch._C._functorch.is_functorch_wrapped_tensor


def _call(call: str, device: int, function, *args):
    """function(*args, stream) with `device` as the current one, on its current stream."""
    if _current_device() == device:
        code = function(*args, _raw_stream(device))
    else:
        with torch.cuda.device(device):
            code = function(*args, _raw_stream(device))
    if code:
        raise SrError(code, call)


def _tensors(call: str, first, *others) -> int:
    """All on one CUDA device (its index is returned), none that a gradient is recorded for, in either direction."""
    if not isinstance(first, torch.Tensor) or any(t is not None and not isinstance(t, torch.Tensor) for t in others):
        _refuse(call, "tensors are required")
    if _grad() and (first.requires_grad or any(t is not None and t.requires_grad for t in others)):
        _refuse(call, "there is no backward pass (use torch.no_grad() or detach)")
    if any(t is not None and (_wrapped(t) or _forward_ad.unpack_dual(t).tangent is not None) for t in (first,) + others):
        _refuse(call, "there is no forward derivative (use the primal, or detach)")
    device = first.get_device()
    if device < 0 or not first.is_cuda:
        _refuse(call, "tensors on a CUDA device are required")
    for t in others:
        if t is not None and t.get_device() != device:
            _refuse(call, "tensors lie on different devices")
    return device


def _written(*tensors):
    """Written in place: whoever has kept one for a gradient learns of it.  (Tensors of inference mode have no versions.)"""
    for t in tensors:
        if t is not None and not t.is_inference():
            torch.autograd.graph.increment_version(t)


def _counts(call: str, *sizes):
    """Sizes that the calls in C take in 32 bits (ctypes would cut them off)."""
    if max(sizes) > 0x7FFFFFFF:
        _refuse(call, "a size is out of range")


def _float_vector(call: str, name: str, t, n: int):
    if t is None:
        return None
    if t.dtype is not torch.float32 or t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        _refuse(call, "%s has to be float32 [%d] without gaps" % (name, n))
    return t.data_ptr()


def _rows(call: str, name: str, t):
    """A matrix whose rows have no gaps inside; its row stride."""
    if t.dim() != 2 or t.dtype not in _DTYPES:
        _refuse(call, "%s has to be a float32 or bfloat16 matrix" % name)
    rows, cols = t.shape
    if cols < 1:
        _refuse(call, "%s has no columns" % name)
    a, b = t.stride()
    if b != 1 and cols > 1:
        _refuse(call, "the columns of %s have to lie side by side" % name)
    return a if rows > 1 else cols


class Microscaled:
    """A matrix [rows][cols] in a microscaled format ("mx4" or "mx8"; layout in include/sr_rollout.h): `data` and `scales` are uint8 tensors."""
    __slots__ = ("data", "scales", "rows", "cols", "format")

    def __init__(self, data, scales, rows: int, cols: int, format: str):
        self.data, self.scales, self.rows, self.cols, self.format = data, scales, rows, cols, format
        self._check("Microscaled")

    def _check(self, call: str):
        """Whether data and scales have the sizes that rows, cols and format make (all of them can be assigned)."""
        data, scales, rows, cols, format = self.data, self.scales, self.rows, self.cols, self.format
        if not isinstance(data, torch.Tensor) or not isinstance(scales, torch.Tensor):
            _refuse(call, "tensors are required")
        if format not in FORMATS:
            _refuse(call, "format is one of %s" % ", ".join(FORMATS))
        if rows < 0 or cols < 1:
            _refuse(call, "a size is out of range")
        groups = -(-cols // 32)
        if data.dtype is not torch.uint8 or scales.dtype is not torch.uint8 or not data.is_contiguous() or not scales.is_contiguous() or \
                data.numel() != rows * groups * (16 if format == "mx4" else 32) or scales.numel() != -(-rows // 128) * -(-groups // 4) * 512:
            _refuse(call, "data and scales have to be uint8, without gaps, of the sizes that rows, cols and format make")

    @classmethod
    def empty(cls, rows: int, cols: int, format: str, device):
        return cls._like(torch.empty(0, device=device), rows, cols, format)

    @classmethod
    def _like(cls, x, rows: int, cols: int, format: str):
        """One without values on x's device."""
        m = cls.__new__(cls)
        if format not in FORMATS:
            _refuse("Microscaled", "format is one of %s" % ", ".join(FORMATS))
        groups = (cols + 31) // 32
        m.data = x.new_empty((rows, groups * (16 if format == "mx4" else 32)), dtype=torch.uint8)
        m.scales = x.new_empty((rows + 127) // 128 * ((groups + 3) // 4) * 512, dtype=torch.uint8)
        m.rows, m.cols, m.format = rows, cols, format
        return m

    def values(self):
        """The values it stands for, float32 [rows][cols]."""
        self._check("values")
        device = _tensors("values", self.data, self.scales)
        out = self.data.new_empty((self.rows, self.cols), dtype=torch.float32)
        _call("sr_microscale_values", device, _library().sr_microscale_values, self.data.data_ptr(), self.scales.data_ptr(), FORMATS[self.format], self.rows,
              self.cols, out.data_ptr())
        return out


def quantize(x, format: str = "mx4") -> Microscaled:
    """x [rows][cols] (float32 or bfloat16; rows may have gaps between them) in a microscaled format."""
    fast = _compiled.quantize(x, FORMATS.get(format, 0))
    if fast is not None:
        m = Microscaled.__new__(Microscaled)
        m.data, m.scales = fast
        m.rows, m.cols = x.shape
        m.format = format
        return m
    device = _tensors("quantize", x)
    stride = _rows("quantize", "x", x)
    m = Microscaled._like(x, x.shape[0], x.shape[1], format)
    _call("sr_microscale_quantize", device, _library().sr_microscale_quantize, x.data_ptr(), _DTYPES[x.dtype], m.rows, m.cols, stride, FORMATS[format],
          m.data.data_ptr(), m.scales.data_ptr())
    return m


def product(a: Microscaled, w: Microscaled, bias=None, relu: bool = False, dtype=torch.bfloat16, out=None):
    """act(bias + a w^T), [a.rows][w.rows]: a dense node's update on microscaled operands of the same format.  `out` (rows may have
    gaps between them) is written in place of a new tensor of `dtype`."""
    if not isinstance(a, Microscaled) or not isinstance(w, Microscaled):
        _refuse("product", "microscaled matrices are required")
    if a.format != w.format or a.cols != w.cols:
        _refuse("product", "both matrices have the same format and number of columns")
    fast = _compiled.product(a.data, a.scales, a.rows, w.data, w.scales, w.rows, a.cols, FORMATS.get(a.format, 0), bias, relu, _DTYPES.get(dtype, -1), out) \
        if out is not None or dtype in _DTYPES else None
    if fast is not None:
        return fast
    a._check("product")
    w._check("product")
    device = _tensors("product", a.data, a.scales, w.data, w.scales, bias, out)
    b = _float_vector("product", "bias", bias, w.rows)
    given = out
    if out is None:
        if dtype not in _DTYPES:
            _refuse("product", "the output is float32 or bfloat16")
        out = a.data.new_empty((a.rows, w.rows), dtype=dtype)
        stride = w.rows
    else:
        if tuple(out.shape) != (a.rows, w.rows):
            _refuse("product", "out has to be [%d][%d]" % (a.rows, w.rows))
        stride = _rows("product", "out", out) if w.rows else 0
    _call("sr_microscale_product", device, _library().sr_microscale_product, a.data.data_ptr(), a.scales.data_ptr(), w.data.data_ptr(), w.scales.data_ptr(),
          FORMATS[a.format], a.rows, a.cols, w.rows, b, 1 if relu else 0, out.data_ptr(), _DTYPES[out.dtype], stride)
    _written(given)
    return out


def product_plan(rows: int, cols: int, outs: int, format: str = "mx4", sms: int = 0) -> dict:
    """How a product of these sizes is cut (sr_microscale_product_plan) on the current device or one of `sms` SMs."""
    p = _ProductPlan()
    code = _library().sr_microscale_product_plan(FORMATS.get(format, 0), rows, cols, outs, sms, ctypes.byref(p))
    if code:
        raise SrError(code, "sr_microscale_product_plan")
    return {n: getattr(p, n) for n, _ in _ProductPlan._fields_}


def rms_norm(x, weight=None, residual=None, eps: float = 1e-6, format: Optional[str] = None):
    """s = x + residual, s / sqrt(mean(s^2) + eps) * weight for every row of x [rows][cols].  The output has x's type, or is `Microscaled` where
    a format is given; with a residual the result is (output, s rounded to x's type)."""
    fast = _compiled.rms_norm(x, weight, residual, eps, 0 if format is None else FORMATS[format]) if format is None or format in FORMATS else None
    if fast is not None:
        out, total = fast
        if format is not None:
            m = Microscaled.__new__(Microscaled)
            m.data, m.scales = out
            m.rows, m.cols = x.shape
            m.format = format
            out = m
        return out if residual is None else (out, total)
    device = _tensors("rms_norm", x, weight, residual)
    xs = _rows("rms_norm", "x", x)
    rows, cols = x.shape
    rs, rp, total, tp = 0, None, None, None
    if residual is not None:
        if residual.shape != x.shape or residual.dtype is not x.dtype:
            _refuse("rms_norm", "the residual has x's shape and type")
        rs, rp = _rows("rms_norm", "residual", residual), residual.data_ptr()
        total = x.new_empty((rows, cols))
        tp = total.data_ptr()
    w = _float_vector("rms_norm", "weight", weight, cols)
    if format is None:
        out = x.new_empty((rows, cols))
        op, code, sp = out.data_ptr(), _DTYPES[x.dtype], None
    else:
        out = Microscaled._like(x, rows, cols, format)
        op, code, sp = out.data.data_ptr(), FORMATS[format], out.scales.data_ptr()
    _call("sr_rms_norm", device, _library().sr_rms_norm, x.data_ptr(), rp, w, eps, _DTYPES[x.dtype], rows, cols, xs, rs, tp, op, code, sp)
    return out if residual is None else (out, total)


# Descriptions made so far, by everything that they hold (sizes, strides, type, scale), with the workspace they need.
_descs: dict = {}


def _desc(call: str, device: int, q, k, v, log_decay, packed: bool, step: bool, batch: int, scale: float):
    key = (q.dtype, k.dtype, v.dtype, log_decay.dtype, q.shape, k.shape, v.shape, log_decay.shape, q.stride(), k.stride(), v.stride(), log_decay.stride(),
           packed, step, batch, scale, device)
    hit = _descs.get(key)
    if hit is not None:
        return hit
    lead = q.dim() - 2
    if q.dtype not in _DTYPES or k.dtype is not q.dtype or v.dtype is not q.dtype or log_decay.dtype is not torch.float32:
        _refuse(call, "q, k and v have one type, float32 or bfloat16; log_decay is float32")
    want = 1 if packed or step else 2
    if lead != want or k.dim() != q.dim() or v.dim() != q.dim() or k.shape[:-2] != q.shape[:-2] or v.shape[:-2] != q.shape[:-2]:
        _refuse(call, "q, k and v have to be %s[heads][size] with the same leading sizes" % ("[sequences]" if step else "[frames]" if packed else "[frames][sequences]"))
    heads, dk = q.shape[-2:]
    groups, dv = k.shape[-2], v.shape[-1]
    if k.shape[-1] != dk or v.shape[-2] != groups or groups < 1 or heads % groups or heads < 1:
        _refuse(call, "k has q's size, v has k's heads, and q's heads are a multiple of them")
    if tuple(log_decay.shape) not in ((groups,), tuple(q.shape[:-2]) + (groups,)):
        _refuse(call, "log_decay has to be [groups] or %s[groups]" % ("[sequences]" if step else "[frames]" if packed else "[frames][sequences]"))
    for name, t in (("q", q), ("k", k), ("v", v)):
        if t.stride(-1) != 1 and t.shape[-1] > 1:
            _refuse(call, "the elements of a head of %s have to lie side by side" % name)

    def strides(st):
        s = _Strides()
        if step:
            s.sequence, s.head = st[0], st[1]
        elif packed:
            s.frame, s.head = st[0], st[1]
        else:
            s.frame, s.sequence, s.head = st[0], st[1], st[2]
        return s

    _counts(call, batch, heads, groups, dk, dv)
    out = tuple(q.shape[:-1]) + (dv,)                # without gaps
    d = _AttentionDesc(_DTYPES[q.dtype], batch, heads, groups, dk, dv, 1 if step else q.shape[0], scale, strides(q.stride()), strides(k.stride()),
                       strides(v.stride()), strides(tuple(math.prod(out[i + 1:]) for i in range(len(out)))))
    ld = log_decay.stride()
    d.log_decay = _Strides(0, 0, ld[0]) if log_decay.dim() == 1 else strides(ld)
    size = ctypes.c_size_t()
    with torch.cuda.device(device):                  # (the workspace goes by the device's SMs)
        code = _library().sr_linear_attention_workspace_bytes(ctypes.byref(d), 1 if packed else 0, ctypes.byref(size))
    if code:
        raise SrError(code, call)
    if len(_descs) >= 256:
        _descs.clear()
    _descs[key] = hit = (ctypes.byref(d), size.value, (batch, groups, dk, dv), d)
    return hit


def attention_plan(dtype, batch: int, frames: int, heads: int, groups: int, dk: int, dv: int, packed: bool = False, sms: int = 0) -> dict:
    """How a run over tensors of these sizes is cut (sr_linear_attention_plan) on the current device or one of `sms` SMs; packed: `frames` in all."""
    _counts("attention_plan", batch, heads, groups, dk, dv)
    d = _AttentionDesc(_DTYPES[dtype], batch, heads, groups, dk, dv, frames, 1.0)
    p = _AttentionPlan()
    code = _library().sr_linear_attention_plan(ctypes.byref(d), 1 if packed else 0, sms, ctypes.byref(p))
    if code:
        raise SrError(code, "sr_linear_attention_plan")
    return {n: getattr(p, n) for n, _ in _AttentionPlan._fields_}


def _state_pointer(call: str, state, shape):
    if state.dtype is not torch.float32 or tuple(state.shape) != shape or not state.is_contiguous():
        _refuse(call, "the state has to be float32 [%d][%d][%d][%d] without gaps" % shape)
    return state.data_ptr()


def linear_attention_run(q, k, v, log_decay, state=None, offsets=None, scale: float = 1.0, out=None, state_out=None):
    """S_t = exp(log_decay_t) S_{t-1} + k_t v_t^T, out_t = scale * q_t S_t over all frames; returns (out, the states after the last frame).

    q [frames][sequences][heads][dk], k [..][groups][dk], v [..][groups][dv] (a view of a larger tensor will do as long as the elements of a
    head lie side by side), log_decay [groups] or [frames][sequences][groups]; with `offsets` (int64 [sequences + 1]) packed sequences
    [frames][heads][size], sequence b the frames offsets[b] .. offsets[b + 1] - 1.  state: float32 [sequences][groups][dk][dv] before the first
    frame (None: zeros).  `out` (without gaps; frames that no sequence has keep what it holds) and `state_out` (may be `state`) are written in
    place of new tensors."""
    fast = _compiled.run(q, k, v, log_decay, state, offsets, scale, out, state_out)
    if fast is not None:
        return (fast[0] if out is None else out), (fast[1] if state_out is None else state_out)
    call = "linear_attention_run"
    device = _tensors(call, q, k, v, log_decay, state, offsets, out, state_out)
    packed = offsets is not None
    if packed and (offsets.dtype is not torch.int64 or offsets.dim() != 1 or offsets.shape[0] < 1 or not offsets.is_contiguous()):
        _refuse(call, "offsets have to be int64 [sequences + 1] without gaps")
    if q.dim() < 3 or v.dim() < 3:
        _refuse(call, "q, k and v have to be [frames][sequences][heads][size], or [frames][heads][size] with offsets")
    given = out
    if out is None:
        out = q.new_empty(q.shape[:-1] + v.shape[-1:])
    elif out.shape != q.shape[:-1] + v.shape[-1:] or out.dtype is not q.dtype or not out.is_contiguous():
        _refuse(call, "out has to be %s of q's type without gaps" % (tuple(q.shape[:-1] + v.shape[-1:]),))
    batch = offsets.shape[0] - 1 if packed else q.shape[1]
    desc, size, shape, _ = _desc(call, device, q, k, v, log_decay, packed, False, batch, scale)
    sp = None if state is None else _state_pointer(call, state, shape)
    last = q.new_empty(shape, dtype=torch.float32) if state_out is None else state_out
    lp = _state_pointer(call, last, shape)
    work = q.new_empty(size, dtype=torch.uint8) if size else None
    _call("sr_linear_attention_run", device, _library().sr_linear_attention_run, desc, q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(),
          offsets.data_ptr() if packed else None, sp, lp, out.data_ptr(), work.data_ptr() if size else None, size)
    _written(given, state_out)
    return out, last


def linear_attention_step(q, k, v, log_decay, state, scale: float = 1.0):
    """One frame of every sequence: q [sequences][heads][dk], k [..][groups][dk], v [..][groups][dv], log_decay [groups] or [sequences][groups].
    `state` (float32 [sequences][groups][dk][dv]) is updated in place; returns out [sequences][heads][dv]."""
    fast = _compiled.step(q, k, v, log_decay, state, scale)
    if fast is not None:
        return fast
    call = "linear_attention_step"
    device = _tensors(call, q, k, v, log_decay, state)
    if q.dim() != 3 or v.dim() != 3:
        _refuse(call, "q, k and v have to be [sequences][heads][size]")
    out = q.new_empty(q.shape[:-1] + v.shape[-1:])
    desc, _, shape, _ = _desc(call, device, q, k, v, log_decay, False, True, q.shape[0], scale)
    _call("sr_linear_attention_step", device, _library().sr_linear_attention_step, desc, q.data_ptr(), k.data_ptr(), v.data_ptr(), log_decay.data_ptr(),
          _state_pointer(call, state, shape), out.data_ptr())
    _written(state)
    return out


def _device_index(call: str, device) -> int:
    d = torch.device("cuda" if device is None else device)
    if d.type != "cuda":
        _refuse(call, "a CUDA device is required")
    return torch.cuda.current_device() if d.index is None else d.index


def operator_status(device=None):
    """Waits for the current stream's work; raises `SrError` if it failed or a bounded wait inside an operator's kernel has expired on the device (until
    `operator_reset`)."""
    _call("sr_operator_status", _device_index("operator_status", device), _library().sr_operator_status)


def operator_reset(device=None):
    """Forgets that a wait expired."""
    _call("sr_operator_reset", _device_index("operator_reset", device), _library().sr_operator_reset)


class _Head:
    """What heads behind a rollout share: `batch` sequences, `channels` features of a frame, and a device."""

    def _fits(self, call: str, features, lead: int):
        if not isinstance(features, torch.Tensor) or features.dim() <= lead or features.shape[lead - 1] != self.batch or math.prod(features.shape[lead:]) != self.channels:
            _refuse("%s.%s" % (type(self).__name__, call), "the head takes %s[%d sequences][%d channels]" % ("[frames]" if lead == 2 else "", self.batch, self.channels))

    def check_features(self, shape, device):
        """Refuses features of one frame that the head cannot take: [batch][...channels], on its device."""
        if len(shape) < 1 or shape[0] != self.batch or math.prod(shape[1:]) != self.channels:
            _refuse(type(self).__name__, "the head takes [%d sequences][%d channels]" % (self.batch, self.channels))
        if _device_index(type(self).__name__, device) != self.device.index:
            _refuse(type(self).__name__, "the head lies on %s" % self.device)


class TemporalHead(_Head):
    """A head with a memory over the frames on the features that a rollout gives, per frame and sequence

        q, k, v = Wqkv norm(x)      (microscaled operands)
        S = exp(log_decay) S + k v^T,  o = q S / sqrt(dk)
        h = x + Wo norm(o),   out = Wout norm(h) + bias

    with x the features ([channels], what `Graph` hands out for its output node).  `run` takes whole clips and `step` single frames; both carry
    the states S on, as a rollout carries a network's, and give the same values up to rounding.

    weights: qkv [heads * dk + groups * (dk + dv)][channels], o [channels][heads * dv], out [outputs][channels], bias [outputs]; norm_x [channels],
    norm_o [heads * dv], norm_h [channels]; log_decay [groups] (all float tensors, quantised here once)."""

    def __init__(self, weights: dict, channels: int, heads: int, groups: int, dk: int, dv: int, batch: int, format: str = "mx4", dtype: str = "bf16",
                 eps: float = 1e-6, device: str = "cuda:0"):
        if min(channels, heads, groups, dk, dv) < 1 or batch < 0 or heads % groups or heads // groups > 128 or dk > 256:
            _refuse("TemporalHead", "sizes are positive, heads a multiple of groups (128 times them at most), dk at most 256")
        if dtype not in ("bf16", "fp32") or format not in FORMATS or not eps >= 0:
            _refuse("TemporalHead", "dtype is bf16 or fp32, format one of %s, eps not negative" % ", ".join(FORMATS))
        self.channels, self.heads, self.groups, self.dk, self.dv, self.batch, self.eps, self.format = channels, heads, groups, dk, dv, batch, eps, format
        self.tdtype = {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]
        shapes = {"qkv": (heads * dk + groups * (dk + dv), channels), "o": (channels, heads * dv), "out": (None, channels), "bias": (None,),
                  "norm_x": (channels,), "norm_o": (heads * dv,), "norm_h": (channels,), "log_decay": (groups,)}
        w = {}
        for name, shape in shapes.items():
            if name not in weights:
                _refuse("TemporalHead", "%s is missing" % name)
            t = torch.as_tensor(weights[name], dtype=torch.float32).detach().to(device).contiguous()
            if t.dim() != len(shape) or any(n is not None and n != m for n, m in zip(shape, t.shape)):
                _refuse("TemporalHead", "%s has shape %s" % (name, tuple(t.shape)))
            w[name] = t
        self.outputs = w["out"].shape[0]
        if w["bias"].shape[0] != self.outputs:
            _refuse("TemporalHead", "bias has another number of outputs than out")
        for name in ("qkv", "o", "out"):
            w[name] = quantize(w[name], format)
        self._w = w
        self.scale = float(dk) ** -0.5
        with torch.inference_mode(False):              # (a state of inference mode could not be written outside of it)
            self.state = torch.zeros((batch, groups, dk, dv), dtype=torch.float32, device=device)

    @property
    def device(self):
        return self.state.device

    def reset(self):
        """Before the first frame: no memory."""
        self.state.zero_()

    def get_state(self):
        return self.state.clone()

    def set_state(self, state):
        if not isinstance(state, torch.Tensor) or state.shape != self.state.shape or state.dtype is not torch.float32:
            _refuse("TemporalHead.set_state", "the state has to be float32 %s" % (tuple(self.state.shape),))
        self.state.copy_(state)

    def _attend(self, x):
        n = self.heads * self.dk, self.groups * self.dk
        qkv = product(rms_norm(x, self._w["norm_x"], eps=self.eps, format=self.format), self._w["qkv"], dtype=self.tdtype)
        return qkv[:, :n[0]], qkv[:, n[0]:n[0] + n[1]], qkv[:, n[0] + n[1]:]

    def _answer(self, x, o):
        y = product(rms_norm(o.reshape(x.shape[0], self.heads * self.dv), self._w["norm_o"], eps=self.eps, format=self.format), self._w["o"], dtype=self.tdtype)
        m, _ = rms_norm(y, self._w["norm_h"], residual=x, eps=self.eps, format=self.format)
        return product(m, self._w["out"], bias=self._w["bias"], dtype=torch.float32)

    @torch.no_grad()
    def run(self, features):
        """features [frames][batch][...channels] (float32 or the head's type) -> float32 [frames][batch][outputs]."""
        self._fits("run", features, 2)
        T, B = features.shape[:2]
        x = features.reshape(T * B, self.channels).to(self.tdtype)
        q, k, v = self._attend(x)
        o, _ = linear_attention_run(q.unflatten(0, (T, B)).unflatten(2, (self.heads, self.dk)), k.unflatten(0, (T, B)).unflatten(2, (self.groups, self.dk)),
                                    v.unflatten(0, (T, B)).unflatten(2, (self.groups, self.dv)), self._w["log_decay"], state=self.state,
                                    scale=self.scale, state_out=self.state)
        return self._answer(x, o).view(T, B, self.outputs)

    @torch.no_grad()
    def step(self, features):
        """features [batch][...channels] of one frame -> float32 [batch][outputs]."""
        self._fits("step", features, 1)
        x = features.reshape(self.batch, self.channels).to(self.tdtype)
        q, k, v = self._attend(x)
        o = linear_attention_step(q.unflatten(1, (self.heads, self.dk)), k.unflatten(1, (self.groups, self.dk)), v.unflatten(1, (self.groups, self.dv)),
                                  self._w["log_decay"], self.state, scale=self.scale)
        return self._answer(x, o)
