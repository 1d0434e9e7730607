"""Operators of the selective head behind a rollout (the sr_causal_conv_*, sr_selective_scan_* and sr_block_norm calls of include/sr_rollout.h).

As in operators.py: argument marshalling only, a call's common case in compiled code, tensors on a CUDA device, work on its current stream, outputs and
workspaces from PyTorch's allocator, every refusal an `SrError`, no derivatives.

  causal_conv_run, _step       convolution of every channel over the last frames: whole clips, single frames
  selective_scan_run, _step    a state for every channel whose decay, input and readout go by the frame
  block_norm                   norm of a block's output, gate, scale and residual, and the norm ahead of the next block, in one pass
  SelectiveHead                blocks of these as one head on the features of a rollout (`Graph.rollout(frames, head=...)`)
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional

import torch

from . import operators as ops
from .binding import SrError
from .operators import FORMATS, Microscaled, _call, _counts, _DTYPES, _float_vector, _Head, _refuse, _rows, _Strides, _tensors, _written, product, quantize, rms_norm

_compiled = ops._compiled
_GATES = {"none": 0, "sigmoid": 1, "silu": 2}
_NORMS = {"none": 0, "after": 1, "before": 2, "both": 3}


class _FrameStrides(ctypes.Structure):
    _fields_ = [("frame", ctypes.c_int64), ("sequence", ctypes.c_int64)]


class _ConvDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "batch", "channels", "width", "act")] + [("frames", ctypes.c_int64), ("x", _FrameStrides), ("out", _FrameStrides)]


class _ScanDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "batch", "channels", "states", "groups", "softplus")] + [("frames", ctypes.c_int64)] + \
        [(n, _FrameStrides) for n in ("u", "dt", "z", "out")] + [(n, _Strides) for n in ("b", "c")]


class _ScanPlan(ctypes.Structure):
    _fields_ = [("held", ctypes.c_int32), ("lanes", ctypes.c_int32), ("segment", ctypes.c_int64), ("segments", ctypes.c_int64)]


class _BlockDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "norms", "gate_act", "out_format")] + [("scale", ctypes.c_float), ("eps", ctypes.c_float)] + \
        [(n, ctypes.c_int64) for n in ("rows", "cols", "y_stride", "residual_stride", "gate_stride")]


_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = ops._library()
        vp, size, i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
        conv, scan, block = (ctypes.POINTER(t) for t in (_ConvDesc, _ScanDesc, _BlockDesc))
        for name, args in {
            "sr_causal_conv_run": [conv] + [vp] * 8,
            "sr_causal_conv_step": [conv] + [vp] * 6,
            "sr_selective_scan_workspace_bytes": [scan, i32, ctypes.POINTER(size)],
            "sr_selective_scan_plan": [scan, i32, i32, ctypes.POINTER(_ScanPlan)],
            "sr_selective_scan_run": [scan] + [vp] * 13 + [size, vp],
            "sr_selective_scan_step": [scan] + [vp] * 11,
            "sr_block_norm": [block] + [vp] * 9,
        }.items():
            f = getattr(lib, name)
            f.argtypes, f.restype = args, i32
        _lib = lib
    return _lib


def _there(call: str, **needed):
    """What may not be left out."""
    for name, t in needed.items():
        if not isinstance(t, torch.Tensor):
            _refuse(call, "%s: tensors are required" % name)


def _pointer(t):
    return None if t is None else t.data_ptr()


def _offsets(call: str, offsets):
    if offsets is not None and (offsets.dtype is not torch.int64 or offsets.dim() != 1 or offsets.shape[0] < 1 or not offsets.is_contiguous()):
        _refuse(call, "offsets have to be int64 [sequences + 1] without gaps")


def _frames(call: str, name: str, t, like, lead: int, tail: int = 1):
    """A tensor of `lead` leading sizes and `tail` more, of like's type and leading sizes, whose last ones lie side by side."""
    if t.dim() != lead + tail or t.dtype is not like.dtype or t.shape[:lead] != like.shape[:lead]:
        _refuse(call, "%s has to be %s%s of one type with the others" % (name, ("[sequences]" if lead == 1 else "[frames][sequences]"), "[channels]" if tail == 1 else "[groups][states]"))
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        _refuse(call, "the last elements of %s have to lie side by side" % name)


def _strides(t, lead: int, step: bool, tail: int = 1):
    st = t.stride()
    frame, sequence = (0, st[0]) if step else (st[0], st[1] if lead == 2 else 0)
    return _FrameStrides(frame, sequence) if tail == 1 else _Strides(frame, sequence, st[lead])


def _matrix(call: str, name: str, t, shape):
    if t.dtype is not torch.float32 or tuple(t.shape) != shape or not t.is_contiguous():
        _refuse(call, "%s has to be float32 %s without gaps" % (name, list(shape)))
    return t.data_ptr()


def _plain(call: str, name: str, t, like, shape):
    if t.dtype is not like.dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        _refuse(call, "%s has to be %s of the inputs' type without gaps" % (name, list(shape)))


def _lead(call: str, x, packed: bool, step: bool) -> int:
    lead = 1 if packed or step else 2
    if x.dtype not in _DTYPES:
        _refuse(call, "inputs are float32 or bfloat16")
    if x.dim() != lead + 1:
        _refuse(call, "inputs have to be %s[channels]" % ("[sequences]" if step else "[frames]" if packed else "[frames][sequences]"))
    if x.shape[-1] < 1:
        _refuse(call, "there are no channels")
    return lead


def _conv_desc(call: str, x, weight, bias, silu, lead: int, step: bool, batch: int, out):
    channels = x.shape[-1]
    _frames(call, "x", x, x, lead)
    if weight.dim() != 2 or weight.shape[1] < 1:
        _refuse(call, "the weight has to be [channels][width]")
    _matrix(call, "the weight", weight, (channels, weight.shape[1]))
    _float_vector(call, "the bias", bias, channels)
    _counts(call, batch, channels, weight.shape[1])
    return _ConvDesc(_DTYPES[x.dtype], batch, channels, weight.shape[1], 1 if silu else 0, 1 if step else x.shape[0], _strides(x, lead, step), _strides(out, lead, step))


def causal_conv_run(x, weight, bias=None, silu: bool = False, state=None, offsets=None, out=None, state_out=None):
    """out[t] = act(bias + sum_j weight[:, j] x[t - (width - 1) + j]) for every channel over all frames, act = x sigmoid(x) or nothing; returns (out, the last
    width - 1 frames of every sequence).

    x [frames][sequences][channels] (a view of a larger tensor will do as long as the channels lie side by side), with `offsets` (int64 [sequences + 1])
    packed sequences [frames][channels], sequence b the frames offsets[b] .. offsets[b + 1] - 1.  weight: float32 [channels][width], bias: float32 [channels].
    state: x's type [sequences][width - 1][channels], the frames ahead of the first (None: zeros).  `out` (x's shape, without gaps; frames that no sequence has
    keep what it holds) and `state_out` (may be `state`) are written in place of new tensors."""
    fast = _compiled.conv_run(x, weight, bias, silu, state, offsets, out, state_out)
    if fast is not None:
        return (fast[0] if out is None else out), (fast[1] if state_out is None else state_out)
    call = "causal_conv_run"
    _there(call, x=x, weight=weight)
    device = _tensors(call, x, weight, bias, state, offsets, out, state_out)
    packed = offsets is not None
    _offsets(call, offsets)
    lead = _lead(call, x, packed, False)
    given, channels = out, x.shape[-1]
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    _plain(call, "out", out, x, x.shape)
    batch = offsets.shape[0] - 1 if packed else x.shape[1]
    d = _conv_desc(call, x, weight, bias, silu, lead, False, batch, out)
    shape = (batch, d.width - 1, channels)
    if state is not None:
        _plain(call, "the state", state, x, shape)
    last = torch.empty(shape, dtype=x.dtype, device=x.device) if state_out is None else state_out
    _plain(call, "state_out", last, x, shape)
    _call("sr_causal_conv_run", device, _library().sr_causal_conv_run, ctypes.byref(d), x.data_ptr(), weight.data_ptr(), _pointer(bias), _pointer(offsets), _pointer(state),
          last.data_ptr(), out.data_ptr())
    _written(given, state_out)
    return out, last


def causal_conv_step(x, weight, state, bias=None, silu: bool = False):
    """One frame of every sequence: x [sequences][channels].  `state` (x's type [sequences][width - 1][channels]) is updated in place; returns out
    [sequences][channels]."""
    fast = _compiled.conv_step(x, weight, state, bias, silu)
    if fast is not None:
        return fast
    call = "causal_conv_step"
    _there(call, x=x, weight=weight, state=state)
    device = _tensors(call, x, weight, state, bias)
    lead = _lead(call, x, False, True)
    out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    d = _conv_desc(call, x, weight, bias, silu, lead, True, x.shape[0], out)
    _plain(call, "the state", state, x, (d.batch, d.width - 1, d.channels))
    _call("sr_causal_conv_step", device, _library().sr_causal_conv_step, ctypes.byref(d), x.data_ptr(), weight.data_ptr(), _pointer(bias), state.data_ptr(), out.data_ptr())
    _written(state)
    return out


def _scan_desc(call: str, u, dt, a, b, c, d, z, dt_bias, softplus, lead: int, step: bool, batch: int, out):
    channels = u.shape[-1]
    for name, t in (("u", u), ("dt", dt), ("z", z)):
        if t is not None:
            _frames(call, name, t, u, lead)
            if t.shape[-1] != channels:
                _refuse(call, "u, dt and z have the same channels")
    for name, t in (("b", b), ("c", c)):
        _frames(call, name, t, u, lead, 2)
    groups, states = b.shape[-2:]
    if c.shape != b.shape or groups < 1 or states < 1 or channels % groups:
        _refuse(call, "b and c have the same groups and states, and the channels are a multiple of the groups")
    _matrix(call, "a", a, (channels, states))
    _float_vector(call, "d", d, channels)
    _float_vector(call, "dt_bias", dt_bias, channels)
    _counts(call, batch, channels, states, groups)
    return _ScanDesc(_DTYPES[u.dtype], batch, channels, states, groups, 1 if softplus else 0, 1 if step else u.shape[0], _strides(u, lead, step), _strides(dt, lead, step),
                     _FrameStrides() if z is None else _strides(z, lead, step), _strides(out, lead, step), _strides(b, lead, step, 2), _strides(c, lead, step, 2))


def selective_scan_run(u, dt, a, b, c, d=None, z=None, dt_bias=None, softplus: bool = True, state=None, offsets=None, out=None, state_out=None):
    """r = softplus(dt + dt_bias), h <- exp(r a) h + r u b, out = (c . h + d u) * z sigmoid(z) for every channel over all frames; returns (out, the states after the
    last frame).

    u, dt, z [frames][sequences][channels], b, c [frames][sequences][groups][states] of one type (views of larger tensors will do as long as the last elements lie
    side by side); channels share b and c in groups of channels / groups neighbours.  a: float32 [channels][states]; d, dt_bias: float32 [channels].  With
    `offsets` (int64 [sequences + 1]) packed sequences, without the dimension [sequences].  state: float32 [sequences][channels][states] before the first frame (None:
    zeros).  `out` (u's shape, without gaps; frames that no sequence has keep what it holds) and `state_out` (may be `state`) are written in place of new
    tensors."""
    fast = _compiled.scan_run(u, dt, a, b, c, d, z, dt_bias, softplus, state, offsets, out, state_out)
    if fast is not None:
        return (fast[0] if out is None else out), (fast[1] if state_out is None else state_out)
    call = "selective_scan_run"
    _there(call, u=u, dt=dt, a=a, b=b, c=c)
    device = _tensors(call, u, dt, a, b, c, d, z, dt_bias, state, offsets, out, state_out)
    packed = offsets is not None
    _offsets(call, offsets)
    lead = _lead(call, u, packed, False)
    given = out
    if out is None:
        out = torch.empty(u.shape, dtype=u.dtype, device=u.device)
    _plain(call, "out", out, u, u.shape)
    batch = offsets.shape[0] - 1 if packed else u.shape[1]
    desc = _scan_desc(call, u, dt, a, b, c, d, z, dt_bias, softplus, lead, False, batch, out)
    shape = (batch, desc.channels, desc.states)
    if state is not None:
        _matrix(call, "the state", state, shape)
    last = torch.empty(shape, dtype=torch.float32, device=u.device) if state_out is None else state_out
    _matrix(call, "state_out", last, shape)
    size = ctypes.c_size_t()
    with torch.cuda.device(device):                    # (the workspace goes by the device's SMs)
        code = _library().sr_selective_scan_workspace_bytes(ctypes.byref(desc), 1 if packed else 0, ctypes.byref(size))
    if code:
        raise SrError(code, call)
    work = torch.empty(size.value, dtype=torch.uint8, device=u.device) if size.value else None
    _call("sr_selective_scan_run", device, _library().sr_selective_scan_run, ctypes.byref(desc), u.data_ptr(), dt.data_ptr(), a.data_ptr(), b.data_ptr(), c.data_ptr(),
          _pointer(d), _pointer(z), _pointer(dt_bias), _pointer(offsets), _pointer(state), last.data_ptr(), out.data_ptr(), _pointer(work), size.value)
    _written(given, state_out)
    return out, last


def selective_scan_step(u, dt, a, b, c, state, d=None, z=None, dt_bias=None, softplus: bool = True):
    """One frame of every sequence: u, dt, z [sequences][channels], b, c [sequences][groups][states].  `state` (float32 [sequences][channels][states]) is updated in place;
    returns out [sequences][channels]."""
    fast = _compiled.scan_step(u, dt, a, b, c, state, d, z, dt_bias, softplus)
    if fast is not None:
        return fast
    call = "selective_scan_step"
    _there(call, u=u, dt=dt, a=a, b=b, c=c, state=state)
    device = _tensors(call, u, dt, a, b, c, state, d, z, dt_bias)
    lead = _lead(call, u, False, True)
    out = torch.empty(u.shape, dtype=u.dtype, device=u.device)
    desc = _scan_desc(call, u, dt, a, b, c, d, z, dt_bias, softplus, lead, True, u.shape[0], out)
    _matrix(call, "the state", state, (desc.batch, desc.channels, desc.states))
    _call("sr_selective_scan_step", device, _library().sr_selective_scan_step, ctypes.byref(desc), u.data_ptr(), dt.data_ptr(), a.data_ptr(), b.data_ptr(), c.data_ptr(),
          _pointer(d), _pointer(z), _pointer(dt_bias), state.data_ptr(), out.data_ptr())
    _written(state)
    return out


def scan_plan(dtype, batch: int, frames: int, channels: int, states: int, groups: int = 1, packed: bool = False, sms: int = 0) -> dict:
    """How a run over tensors of these sizes is cut (sr_selective_scan_plan) on the current device or one of `sms` SMs; packed: `frames` in all."""
    _counts("scan_plan", batch, channels, states, groups)
    d = _ScanDesc(_DTYPES[dtype], batch, channels, states, groups, 1, frames)
    p = _ScanPlan()
    code = _library().sr_selective_scan_plan(ctypes.byref(d), 1 if packed else 0, sms, ctypes.byref(p))
    if code:
        raise SrError(code, "sr_selective_scan_plan")
    return {n: getattr(p, n) for n, _ in _ScanPlan._fields_}


def block_norm(y, residual, weight_after=None, weight_before=None, gate=None, gate_act: str = "sigmoid", scale: float = 1.0, eps: float = 1e-6, norms: str = "both",
               format: Optional[str] = None):
    """h = residual + scale * act(gate) * rms(y) * weight_after, out = rms(h) * weight_before, rms(x) = x / sqrt(mean(x^2) + eps), for every row of y [rows][cols].

    residual and gate have y's shape and type (rows may have gaps between them, or all be the same one); act is "none", "sigmoid" or "silu" (x sigmoid(x)); weights are
    float32 [cols].  norms: "both", "after" (no norm of h, and no output of it), "before" (y as it is) or "none".  Returns (out, h rounded to y's type), or h alone; out has y's type,
    or is `Microscaled` where a format is given."""
    kinds = _NORMS.get(norms, -1)
    fast = _compiled.block_norm(y, residual, weight_after, weight_before, gate, _GATES.get(gate_act, -1), scale, eps, kinds, 0 if format is None else FORMATS[format]) \
        if format is None or format in FORMATS else None
    if fast is not None:
        out, h = fast
        if kinds < 2:
            return h
        if format is not None:
            m = Microscaled.__new__(Microscaled)
            m.data, m.scales = out
            m.rows, m.cols = y.shape
            m.format = format
            out = m
        return out, h
    call = "block_norm"
    _there(call, y=y, residual=residual)
    device = _tensors(call, y, residual, weight_after, weight_before, gate)
    if kinds < 0 or gate_act not in _GATES:
        _refuse(call, "norms is one of %s, gate_act one of %s" % (", ".join(_NORMS), ", ".join(_GATES)))
    if format is not None and (format not in FORMATS or kinds < 2):
        _refuse(call, "format is one of %s, and there has to be an output" % ", ".join(FORMATS))
    ys = _rows(call, "y", y)
    rows, cols = y.shape
    strides = []
    for name, t in (("the residual", residual), ("the gate", gate)):
        if t is not None and (t.shape != y.shape or t.dtype is not y.dtype):
            _refuse(call, "%s has y's shape and type" % name)
        strides.append(0 if t is None else _rows(call, name, t))
    after, before = _float_vector(call, "weight_after", weight_after, cols), _float_vector(call, "weight_before", weight_before, cols)
    h = torch.empty((rows, cols), dtype=y.dtype, device=y.device)
    out, op, sp = None, None, None
    if kinds >= 2 and format is None:
        out = torch.empty((rows, cols), dtype=y.dtype, device=y.device)
        op = out.data_ptr()
    elif kinds >= 2:
        out = Microscaled._like(y, rows, cols, format)
        op, sp = out.data.data_ptr(), out.scales.data_ptr()
    desc = _BlockDesc(_DTYPES[y.dtype], kinds, _GATES[gate_act], _DTYPES[y.dtype] if format is None else FORMATS[format], scale, eps, rows, cols, ys, *strides)
    _call("sr_block_norm", device, _library().sr_block_norm, ctypes.byref(desc), y.data_ptr(), residual.data_ptr(), _pointer(gate), after, before, h.data_ptr(), op, sp)
    return h if kinds < 2 else (out, h)


class SelectiveHead(_Head):
    """A head of blocks with a selective memory over the frames on the features that a rollout gives, per frame and sequence

        m = norm(x) * norm_0,  h = x, and for every block i
            u, z, gate = Win m                            (microscaled operands)
            u = silu(conv(u)),  low, b, c = Wx u,  dt = Wdt low
            y = scan(u, dt, a, b, c, d, z)
            h = h + scale * sigmoid(gate) * norm(Wo y) * norm_after,   m = norm(h) * norm of block i + 1, or norm_out
        out = Wout m + bias

    with x the features ([channels], what `Graph` hands out for its output node).  `run` takes whole clips and `step` single frames; both carry the blocks' states on, as
    a rollout carries a network's, and give the same values up to rounding.

    weights: blocks (a list), norm_out [channels], out [outputs][channels], bias [outputs]; a block: norm [channels], in [2 * inner + channels][channels], conv [inner][width],
    conv_bias [inner], x [rank + 2 * groups * states][inner], dt [inner][rank], dt_bias [inner], a [inner][states], d [inner], o [channels][inner], norm_after [channels]
    (all float tensors, quantised here once)."""

    def __init__(self, weights: dict, channels: int, inner: int, states: int, rank: int, width: int, batch: int, groups: int = 1, scale: float = 1.0, format: str = "mx4",
                 dtype: str = "bf16", eps: float = 1e-6, device: str = "cuda:0"):
        if min(channels, inner, states, rank, width, groups) < 1 or batch < 0 or inner % groups or states > 128 or width > 8:
            _refuse("SelectiveHead", "sizes are positive, inner a multiple of groups, states at most 128, width at most 8")
        if dtype not in ("bf16", "fp32") or format not in FORMATS or not eps >= 0:
            _refuse("SelectiveHead", "dtype is bf16 or fp32, format one of %s, eps not negative" % ", ".join(FORMATS))
        if not isinstance(weights.get("blocks"), (list, tuple)) or not weights["blocks"]:
            _refuse("SelectiveHead", "blocks are missing")
        self.channels, self.inner, self.states, self.rank, self.width, self.groups = channels, inner, states, rank, width, groups
        self.batch, self.scale, self.eps, self.format = batch, scale, eps, format
        self.tdtype = {"bf16": torch.bfloat16, "fp32": torch.float32}[dtype]
        self.device = torch.empty(0, device=device).device

        def take(of, shapes):
            w = {}
            for name, shape in shapes.items():
                if name not in of:
                    _refuse("SelectiveHead", "%s is missing" % name)
                t = torch.as_tensor(of[name], dtype=torch.float32).detach().to(self.device).contiguous()
                if t.dim() != len(shape) or any(n is not None and n != m for n, m in zip(shape, t.shape)):
                    _refuse("SelectiveHead", "%s has shape %s" % (name, tuple(t.shape)))
                w[name] = t
            return w

        small = rank + 2 * groups * states
        blocks = [take(b, {"norm": (channels,), "in": (2 * inner + channels, channels), "conv": (inner, width), "conv_bias": (inner,), "x": (small, inner), "dt": (inner, rank),
                           "dt_bias": (inner,), "a": (inner, states), "d": (inner,), "o": (channels, inner), "norm_after": (channels,)}) for b in weights["blocks"]]
        w = take(weights, {"norm_out": (channels,), "out": (None, channels), "bias": (None,)})
        self.outputs = w["out"].shape[0]
        if w["bias"].shape[0] != self.outputs:
            _refuse("SelectiveHead", "bias has another number of outputs than out")
        for b in blocks:
            for name in ("in", "x", "dt", "o"):
                b[name] = quantize(b[name], format)
        w["out"] = quantize(w["out"], format)
        self._w, self._blocks = w, blocks
        with torch.inference_mode(False):              # (states of inference mode could not be written outside of it)
            self._states = [(torch.zeros((batch, width - 1, inner), dtype=self.tdtype, device=self.device),
                             torch.zeros((batch, inner, states), dtype=torch.float32, device=self.device)) for _ in blocks]

    def reset(self):
        """Before the first frame: no memory."""
        for conv, scan in self._states:
            conv.zero_()
            scan.zero_()

    def get_state(self):
        """A copy of every block's states: the last frames ahead of its convolution, and its scan's states."""
        return [(conv.clone(), scan.clone()) for conv, scan in self._states]

    def set_state(self, state):
        def fits(given, own):
            return isinstance(given, (list, tuple)) and len(given) == 2 and all(isinstance(t, torch.Tensor) and t.shape == o.shape and t.dtype is o.dtype for t, o in zip(given, own))

        if not isinstance(state, (list, tuple)) or len(state) != len(self._states) or not all(map(fits, state, self._states)):
            _refuse("SelectiveHead.set_state", "the state has to be what get_state gives")
        for s, (conv, scan) in zip(state, self._states):
            conv.copy_(s[0])
            scan.copy_(s[1])

    def _through(self, x, lead):
        """x [rows][channels] through all blocks; lead: () for one frame of every sequence, (frames,) for whole clips."""
        step, n, gn = not lead, self.inner, self.groups * self.states
        lead = tuple(lead) + (self.batch,)
        m, h = rms_norm(x, self._blocks[0]["norm"], eps=self.eps, format=self.format), x
        for i, (w, (conv, scan)) in enumerate(zip(self._blocks, self._states)):
            p = product(m, w["in"], dtype=self.tdtype)
            u, z = p[:, :n].unflatten(0, lead), p[:, n:2 * n].unflatten(0, lead)
            if step:
                u = causal_conv_step(u, w["conv"], conv, bias=w["conv_bias"], silu=True)
            else:
                u, _ = causal_conv_run(u, w["conv"], bias=w["conv_bias"], silu=True, state=conv, state_out=conv)
            low = product(quantize(u.view(x.shape[0], n), self.format), w["x"], dtype=self.tdtype)
            dt = product(quantize(low[:, :self.rank], self.format), w["dt"], dtype=self.tdtype).view(u.shape)
            b, c = (low[:, self.rank + k * gn:self.rank + (k + 1) * gn].unflatten(1, (self.groups, self.states)).unflatten(0, lead) for k in (0, 1))
            if step:
                y = selective_scan_step(u, dt, w["a"], b, c, scan, d=w["d"], z=z, dt_bias=w["dt_bias"])
            else:
                y, _ = selective_scan_run(u, dt, w["a"], b, c, d=w["d"], z=z, dt_bias=w["dt_bias"], state=scan, state_out=scan)
            o = product(quantize(y.view(x.shape[0], n), self.format), w["o"], dtype=self.tdtype)
            before = self._blocks[i + 1]["norm"] if i + 1 < len(self._blocks) else self._w["norm_out"]
            m, h = block_norm(o, h, w["norm_after"], before, gate=p[:, 2 * n:], scale=self.scale, eps=self.eps, format=self.format)
        return product(m, self._w["out"], bias=self._w["bias"], dtype=torch.float32)

    @torch.no_grad()
    def run(self, features):
        """features [frames][batch][...channels] (float32 or the head's type) -> float32 [frames][batch][outputs]."""
        self._fits("run", features, 2)
        T = features.shape[0]
        return self._through(features.reshape(T * self.batch, self.channels).to(self.tdtype), (T,)).view(T, self.batch, self.outputs)

    @torch.no_grad()
    def step(self, features):
        """features [batch][...channels] of one frame -> float32 [batch][outputs]."""
        self._fits("step", features, 1)
        return self._through(features.reshape(self.batch, self.channels).to(self.tdtype), ())
