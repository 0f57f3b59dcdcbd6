"""Operators of explainer networks (``include/gts_nn.h``): networks that learn to give
the SHAP values ``gts.shap`` computes.

Argument marshalling only; the work runs in libgts' gfx950 kernels.  Tensors are
float32, bfloat16 or float16 on the current HIP device, matrices with unit column stride.
Calls are enqueued on ``stream`` (default: the current one) and do not synchronise.
Outputs and workspaces that a call makes itself are allocated on that stream; inputs
made on another stream must be ready when the call's stream reaches it.
"""
from __future__ import annotations

import array
import contextlib
import ctypes
import functools
import itertools
from typing import NamedTuple, Optional, Sequence

import numpy as np
import torch

from . import gts

ACTS = {"none": 0, "relu": 1, "silu": 2, "gelu": 3}
NORMS = {"rms": 0, "layer": 1}
GATES = {"none": 0, "linear": 1, "sigmoid": 2}
STATE_BLOCK = 256
TYPES = {torch.float32: 0, torch.bfloat16: 2, torch.float16: 3}

_i32, _i64, _vp, _f32, _f64 = (ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p, ctypes.c_float,
                               ctypes.c_double)


class _Linear(ctypes.Structure):
    """gts_linear_args"""
    _fields_ = [("rows", _i64), ("inputs", _i64), ("outputs", _i64), ("dtype", _i32),
                ("act", _i32), ("x", _vp), ("ld_x", _i64), ("w", _vp), ("ld_w", _i64),
                ("bias", _vp), ("residual", _vp), ("ld_r", _i64), ("y", _vp), ("ld_y", _i64),
                ("pre", _vp), ("ld_pre", _i64)]


class _LinearGrad(ctypes.Structure):
    """gts_linear_grad_args"""
    _fields_ = [("rows", _i64), ("inputs", _i64), ("outputs", _i64), ("dtype", _i32),
                ("act", _i32), ("dy", _vp), ("ld_dy", _i64), ("pre", _vp), ("ld_pre", _i64),
                ("x", _vp), ("ld_x", _i64), ("w", _vp), ("ld_w", _i64), ("dx", _vp),
                ("ld_dx", _i64), ("dw", _vp), ("ld_dw", _i64), ("db", _vp)]


class LinearLaunch(ctypes.Structure):
    """gts_linear_launch (include/gts_nn.h)."""
    _fields_ = [("tile_m", _i32), ("tile_n", _i32), ("splits", _i32), ("copies", _i32),
                ("direct", _i32)]


class _Norm(ctypes.Structure):
    """gts_norm_args"""
    _fields_ = [("rows", _i64), ("width", _i64), ("dtype", _i32), ("norm", _i32),
                ("gate_act", _i32), ("eps", _f32), ("x", _vp), ("ld_x", _i64), ("f", _vp),
                ("ld_f", _i64), ("gate", _vp), ("ld_gate", _i64), ("scale", _vp),
                ("w_post", _vp), ("w_pre", _vp), ("u", _vp), ("ld_u", _i64), ("h", _vp),
                ("ld_h", _i64)]


class _NormGrad(ctypes.Structure):
    """gts_norm_grad_args"""
    _fields_ = [("rows", _i64), ("width", _i64), ("dtype", _i32), ("norm", _i32),
                ("gate_act", _i32), ("eps", _f32), ("du", _vp), ("ld_du", _i64), ("dh", _vp),
                ("ld_dh", _i64), ("u", _vp), ("ld_u", _i64), ("f", _vp), ("ld_f", _i64),
                ("gate", _vp), ("ld_gate", _i64), ("scale", _vp), ("w_post", _vp),
                ("w_pre", _vp), ("dx", _vp), ("ld_dx", _i64), ("df", _vp), ("ld_df", _i64),
                ("dgate", _vp), ("ld_dgate", _i64), ("dscale", _vp), ("dw_post", _vp),
                ("dw_pre", _vp)]


class _AdamW(ctypes.Structure):
    """gts_adamw_args"""
    _fields_ = [("tensors", _vp), ("num_tensors", _i64), ("param_dtype", _i32),
                ("grad_dtype", _i32), ("copy_dtype", _i32), ("state_bits", _i32), ("m", _vp),
                ("v", _vp), ("m_scale", _vp), ("v_scale", _vp), ("d_clip", _vp), ("step", _i64),
                ("lr", _f64), ("beta1", _f64), ("beta2", _f64), ("eps", _f64),
                ("weight_decay", _f64)]


_lib = None


def _L() -> ctypes.CDLL:
    global _lib
    if _lib is None:
        L = gts.lib()
        P = ctypes.POINTER
        for name, args in (
                ("gts_linear_workspace_bytes", [_i64, _i64, _i64, _i32, _i32, P(_i64)]),
                ("gts_linear_config", [_i64, _i64, _i64, _i32, _i32, _i32, P(LinearLaunch)]),
                ("gts_linear", [P(_Linear), _vp, _i64, _vp]),
                ("gts_linear_backward_workspace_bytes", [_i64, _i64, _i64, _i32, _i32, P(_i64)]),
                ("gts_linear_backward", [P(_LinearGrad), _vp, _i64, _vp]),
                ("gts_norm_residual", [P(_Norm), _vp]),
                ("gts_norm_residual_backward_workspace_bytes", [_i64, _i64, P(_i64)]),
                ("gts_norm_residual_backward", [P(_NormGrad), _vp, _i64, _vp]),
                ("gts_grad_clip_workspace_bytes", [_vp, _i64, P(_i64)]),
                ("gts_grad_clip", [_vp, _i64, _i32, _f32, _vp, _vp, _i64, _vp]),
                ("gts_adamw", [P(_AdamW), _vp])):
            f = getattr(L, name)
            f.argtypes, f.restype = args, ctypes.c_int
        _lib = L
    return _lib


# ----------------------------------------------------------------------------
# arguments
# ----------------------------------------------------------------------------
#
# The checks take a tensor's attributes as few times as they can: a call on one row is
# shorter on the device than these lines on the host.

def _first(name, t):
    """The type and device that a call's other tensors must share with this one."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) torch tensor")
    dtype, dev = t.dtype, t.get_device()
    if dtype not in TYPES:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, not {dtype}")
    if dev != torch.cuda.current_device():
        raise ValueError(f"{name} is on cuda:{dev}, which is not the current device")
    return dtype, dev


def _same(name, t, dtype, dev):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) torch tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, not on cuda:{dev}")


def _extents(name, t):
    shape = t.shape
    if len(shape) != 2:
        raise ValueError(f"{name} must be a matrix, not of shape {tuple(shape)}")
    return shape


def _matrix(name, t, rows, width, dtype, dev):
    """(address, row stride) of a matrix argument."""
    _same(name, t, dtype, dev)
    shape = t.shape
    if len(shape) != 2 or shape[0] != rows or shape[1] != width:
        raise ValueError(f"{name} must have shape {(rows, width)}, not {tuple(shape)}")
    if t.is_contiguous():
        return t.data_ptr(), width
    ld, step = t.stride()
    if width > 1 and step != 1:
        raise ValueError(f"{name} must have unit column stride")
    if rows > 1 and ld < width:
        raise ValueError(f"{name} has rows that overlap (row stride {ld}, width {width})")
    return t.data_ptr(), (ld if rows > 1 else width)


def _vector(name, t, n, dtype, dev):
    _same(name, t, dtype, dev)
    if t.dim() != 1 or t.shape[0] != n or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous vector of {n}")
    return t.data_ptr()


def _choice(name, value, table):
    try:
        return table[value]
    except (KeyError, TypeError):
        raise ValueError(f"{name} must be one of {', '.join(map(str, table))}, not {value!r}") from None


_HERE = contextlib.nullcontext()


def _on(stream):
    """The context in which a call allocates: its stream's."""
    return _HERE if stream is None else torch.cuda.stream(stream)


def _handle(stream, dev):
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream


def _workspace(need, given, like):
    """(address, size, the tensor) of at least `need` bytes; the caller's where it is given
    and large enough."""
    if need == 0:
        return None, 0, None
    if given is None or given.numel() * given.element_size() < need:
        given = torch.empty(need, dtype=torch.uint8, device=like.device)
    elif not given.is_cuda or given.get_device() != like.get_device() or not given.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the call's device")
    return given.data_ptr(), given.numel() * given.element_size(), given


def _lie(addresses, strides):
    """The workspace queries' `aligned`, of addresses and of row strides in bytes, all of
    each combined by or."""
    return (addresses | strides) & 15 == 0 and strides < 1 << 22


@functools.lru_cache(maxsize=1024)
def _need(query, *sizes):
    """The bytes a workspace query gives: a function of the sizes alone."""
    n = _i64(0)
    gts._check(getattr(_L(), query)(*sizes, n), query)
    return n.value


# ----------------------------------------------------------------------------
# products
# ----------------------------------------------------------------------------

def linear(x, weight, bias=None, *, residual=None, act="none", save_pre=False, out=None,
           workspace=None, stream=None):
    """gts_linear: act(x weight^T + bias) + residual.

    x [rows, inputs], weight [outputs, inputs], bias [outputs], residual [rows, outputs].
    With ``save_pre``, (result, pre-activation), as linear_backward needs it.  ``out``
    may be ``residual``."""
    dtype, dev = _first("x", x)
    rows, inputs = _extents("x", x)
    _same("weight", weight, dtype, dev)
    outputs = _extents("weight", weight)[0]
    a = _Linear(rows, inputs, outputs, TYPES[dtype], _choice("act", act, ACTS))
    a.x, a.ld_x = _matrix("x", x, rows, inputs, dtype, dev)
    a.w, a.ld_w = _matrix("weight", weight, outputs, inputs, dtype, dev)
    if bias is not None:
        a.bias = _vector("bias", bias, outputs, dtype, dev)
    if residual is not None:
        a.residual, a.ld_r = _matrix("residual", residual, rows, outputs, dtype, dev)
    size = 4 if a.dtype == 0 else 2
    aligned = rows * inputs * outputs > 0 and _lie(a.x | a.w, (a.ld_x | a.ld_w) * size)
    need = _need("gts_linear_workspace_bytes", rows, inputs, outputs, a.dtype, aligned)
    pre = None
    with _on(stream):
        if out is None:
            out = x.new_empty((rows, outputs))
            a.y, a.ld_y = out.data_ptr(), outputs
        else:
            a.y, a.ld_y = _matrix("out", out, rows, outputs, dtype, dev)
        if save_pre:
            pre = x.new_empty((rows, outputs))
            a.pre, a.ld_pre = pre.data_ptr(), outputs
        ws, size, keep = _workspace(need, workspace, x)
        gts._check(_L().gts_linear(a, ws, size, _handle(stream, dev)), "gts_linear")
    return (out, pre) if save_pre else out


def linear_config(rows: int, inputs: int, outputs: int, dtype, product: str = "forward",
                  aligned: bool = True) -> dict:
    """gts_linear_config: how a product ("forward", "dx" or "dw") of these extents runs."""
    info = LinearLaunch()
    kind = _choice("product", product, {"forward": 0, "dx": 1, "dw": 2})
    gts._check(_L().gts_linear_config(rows, inputs, outputs, _choice("dtype", dtype, TYPES), aligned,
                                      kind, info), "gts_linear_config")
    return {name: int(getattr(info, name)) for name, _ in LinearLaunch._fields_}


def linear_backward(dy, x, weight, *, pre=None, act="none", bias=True, dx=True, dw=True,
                    workspace=None, stream=None):
    """gts_linear_backward: (dx, dweight, dbias) of ``linear``; dx, dw and bias say
    which are wanted, the others are None.  ``pre`` is the pre-activation that
    linear(..., save_pre=True) returned, for any act but "none".  The gradient of a
    residual is dy."""
    dtype, dev = _first("dy", dy)
    rows, outputs = _extents("dy", dy)
    _same("x", x, dtype, dev)
    inputs = _extents("x", x)[1]
    a = _LinearGrad(rows, inputs, outputs, TYPES[dtype], _choice("act", act, ACTS))
    a.dy, a.ld_dy = _matrix("dy", dy, rows, outputs, dtype, dev)
    a.x, a.ld_x = _matrix("x", x, rows, inputs, dtype, dev)
    a.w, a.ld_w = _matrix("weight", weight, outputs, inputs, dtype, dev)
    if a.act != 0:
        if pre is None:
            raise ValueError(f"act {act!r} needs pre")
        a.pre, a.ld_pre = _matrix("pre", pre, rows, outputs, dtype, dev)
    size = 4 if a.dtype == 0 else 2
    aligned = (rows * inputs * outputs > 0 and
               _lie(a.dy | a.x | a.w, (a.ld_dy | a.ld_x | a.ld_w) * size))
    need = _need("gts_linear_backward_workspace_bytes", rows, inputs, outputs, a.dtype, aligned)
    gx = gw = gb = None
    with _on(stream):
        if dx:
            gx = dy.new_empty((rows, inputs))
            a.dx, a.ld_dx = gx.data_ptr(), inputs
        if dw:
            gw = dy.new_empty((outputs, inputs))
            a.dw, a.ld_dw = gw.data_ptr(), inputs
        if bias:
            gb = dy.new_empty(outputs)
            a.db = gb.data_ptr()
        ws, size, keep = _workspace(need, workspace, dy)
        gts._check(_L().gts_linear_backward(a, ws, size, _handle(stream, dev)),
                   "gts_linear_backward")
    return gx, gw, gb


# ----------------------------------------------------------------------------
# norms
# ----------------------------------------------------------------------------

def _gate_of(gate, gate_act):
    kind = _choice("gate_act", gate_act or ("none" if gate is None else "sigmoid"), GATES)
    if (gate is None) != (kind == 0):
        raise ValueError('gate must be given exactly if gate_act is not "none"')
    return kind


def norm_residual(x, f, w_post, w_pre, *, gate=None, scale=None, norm="rms", gate_act=None,
                  eps=1e-6, u=None, h=None, stream=None):
    """gts_norm_residual: (u, h) with u = x + scale * gate * (N(f) * w_post) and
    h = N(u) * w_pre.

    x, f and gate [rows, width], the others [width].  gate_act is "sigmoid" (default
    with a gate), "linear" (the gate multiplies as it is) or "none".  ``u`` may be x,
    ``h`` may be f."""
    dtype, dev = _first("x", x)
    rows, width = _extents("x", x)
    a = _Norm(rows, width, TYPES[dtype], _choice("norm", norm, NORMS), _gate_of(gate, gate_act),
              eps)
    a.x, a.ld_x = _matrix("x", x, rows, width, dtype, dev)
    a.f, a.ld_f = _matrix("f", f, rows, width, dtype, dev)
    if gate is not None:
        a.gate, a.ld_gate = _matrix("gate", gate, rows, width, dtype, dev)
    a.w_post = _vector("w_post", w_post, width, dtype, dev)
    a.w_pre = _vector("w_pre", w_pre, width, dtype, dev)
    if scale is not None:
        a.scale = _vector("scale", scale, width, dtype, dev)
    with _on(stream):
        if u is None:
            u = x.new_empty((rows, width))
            a.u, a.ld_u = u.data_ptr(), width
        else:
            a.u, a.ld_u = _matrix("u", u, rows, width, dtype, dev)
        if h is None:
            h = x.new_empty((rows, width))
            a.h, a.ld_h = h.data_ptr(), width
        else:
            a.h, a.ld_h = _matrix("h", h, rows, width, dtype, dev)
        gts._check(_L().gts_norm_residual(a, _handle(stream, dev)), "gts_norm_residual")
    return u, h


def norm_residual_backward(du, dh, u, f, w_post, w_pre, *, gate=None, scale=None, norm="rms",
                           gate_act=None, eps=1e-6, workspace=None, stream=None):
    """gts_norm_residual_backward: a dict of the gradients "dx", "df", "dw_post", "dw_pre",
    and "dgate" and "dscale" where there is a gate and a scale.  du and dh are the
    gradients of norm_residual's results (du may be None: zero), u its first result."""
    dtype, dev = _first("dh", dh)
    rows, width = _extents("dh", dh)
    a = _NormGrad(rows, width, TYPES[dtype], _choice("norm", norm, NORMS),
                  _gate_of(gate, gate_act), eps)
    a.dh, a.ld_dh = _matrix("dh", dh, rows, width, dtype, dev)
    if du is not None:
        a.du, a.ld_du = _matrix("du", du, rows, width, dtype, dev)
    a.u, a.ld_u = _matrix("u", u, rows, width, dtype, dev)
    a.f, a.ld_f = _matrix("f", f, rows, width, dtype, dev)
    a.w_post = _vector("w_post", w_post, width, dtype, dev)
    a.w_pre = _vector("w_pre", w_pre, width, dtype, dev)
    need = _need("gts_norm_residual_backward_workspace_bytes", rows, width)
    out = {}
    with _on(stream):
        out["dx"], out["df"] = dh.new_empty((rows, width)), dh.new_empty((rows, width))
        a.dx, a.df = out["dx"].data_ptr(), out["df"].data_ptr()
        a.ld_dx = a.ld_df = a.ld_dgate = width
        if gate is not None:
            a.gate, a.ld_gate = _matrix("gate", gate, rows, width, dtype, dev)
            out["dgate"] = dh.new_empty((rows, width))
            a.dgate = out["dgate"].data_ptr()
        if scale is not None:
            a.scale = _vector("scale", scale, width, dtype, dev)
            out["dscale"] = dh.new_empty(width)
            a.dscale = out["dscale"].data_ptr()
        out["dw_post"], out["dw_pre"] = dh.new_empty(width), dh.new_empty(width)
        a.dw_post, a.dw_pre = out["dw_post"].data_ptr(), out["dw_pre"].data_ptr()
        ws, size, keep = _workspace(need, workspace, dh)
        gts._check(_L().gts_norm_residual_backward(a, ws, size, _handle(stream, dev)),
                   "gts_norm_residual_backward")
    return out


# ----------------------------------------------------------------------------
# the optimizer's step
# ----------------------------------------------------------------------------

# gts_tensor
_TENSOR = np.dtype([("param", np.uint64), ("grad", np.uint64), ("copy", np.uint64),
                    ("count", np.int64), ("state_offset", np.int64)])
assert _TENSOR.itemsize == 40


class AdamWState(NamedTuple):
    """The moments of a list of parameters, in flat buffers: tensor i's start at
    state_offsets(params)[0][i].  In 32 bits m and v are the moments; in 8 bits, m and
    v are float8_e4m3fn codes, m = code * m_scale and sqrt(v) = code * v_scale with a
    scale for each 256."""
    m: torch.Tensor
    v: torch.Tensor
    m_scale: Optional[torch.Tensor]
    v_scale: Optional[torch.Tensor]


def state_offsets(tensors: Sequence):
    """(where each tensor's state starts, the flat buffers' length)."""
    starts, total = _starts(tuple(t.numel() for t in tensors))
    return list(starts), total


def adamw_state(params: Sequence, bits: int = 32) -> AdamWState:
    """Zero moments for these parameters, in 32 or 8 bits."""
    if bits not in (8, 32):
        raise ValueError("bits must be 8 or 32")
    n = state_offsets(params)[1]
    dev = params[0].device if params else "cuda"
    if bits == 32:
        return AdamWState(torch.zeros(n, device=dev), torch.zeros(n, device=dev), None, None)
    codes = [torch.zeros(n, dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn)
             for _ in range(2)]
    scales = [torch.full((n // STATE_BLOCK,), 2.0 ** -126, device=dev) for _ in range(2)]
    return AdamWState(*codes, *scales)


def _addresses(name, tensors, dtype, dev, sizes=None):
    """Addresses of a list of contiguous tensors of one type, of the given sizes."""
    try:
        out = [t.data_ptr() for t in tensors
               if t.dtype is dtype and t.get_device() == dev and t.is_contiguous()]
    except AttributeError:
        out = ()
    if len(out) != len(tensors):
        for i, t in enumerate(tensors):
            _same(f"{name}[{i}]", t, dtype, dev)
            if not t.is_contiguous():
                raise ValueError(f"{name}[{i}] must be contiguous")
    if sizes is not None:
        for i, t in enumerate(tensors):
            if t.numel() != sizes[i]:
                raise ValueError(f"{name}[{i}] has {t.numel()} elements, its parameter {sizes[i]}")
    return out


@functools.lru_cache(maxsize=64)
def _starts(sizes):
    """(where the states of tensors of these sizes start, the states' length)."""
    at, starts = 0, []
    for n in sizes:
        starts.append(at)
        at += -(-n // STATE_BLOCK) * STATE_BLOCK
    return tuple(starts), at


def _table(params, grads, copies, sizes, starts):
    """An array of gts_tensor."""
    return array.array("q", itertools.chain.from_iterable(zip(params, grads, copies, sizes, starts)))


@functools.lru_cache(maxsize=64)
def _clip_bytes(sizes):
    """What gts_grad_clip_workspace_bytes gives for gradients of these sizes."""
    none, n = (0,) * len(sizes), _i64(0)
    tab = _table(none, none, none, sizes, none)
    gts._check(_L().gts_grad_clip_workspace_bytes(tab.buffer_info()[0], len(sizes), n),
               "gts_grad_clip_workspace_bytes")
    return n.value


def grad_clip(grads: Sequence, max_norm: float, *, out=None, workspace=None, stream=None):
    """gts_grad_clip: a tensor of two, the norm of all gradients together and the factor
    that holds it to max_norm (NaN if it is not finite), for adamw_step."""
    if not grads:
        raise ValueError("grads must not be empty")
    like = grads[0]
    dtype, dev = _first("grads[0]", like)
    at = _addresses("grads", grads, dtype, dev)
    sizes = tuple([t.numel() for t in grads])
    none = (0,) * len(at)
    tab = _table(none, at, none, sizes, none)
    with _on(stream):
        if out is None:
            out = torch.empty(2, dtype=torch.float32, device=like.device)
            address = out.data_ptr()
        else:
            address = _vector("out", out, 2, torch.float32, dev)
        ws, size, keep = _workspace(_clip_bytes(sizes), workspace, like)
        gts._check(_L().gts_grad_clip(tab.buffer_info()[0], len(at), TYPES[dtype], max_norm,
                                      address, ws, size, _handle(stream, dev)), "gts_grad_clip")
    return out


def adamw_step(params: Sequence, grads: Sequence, m, v, *, step: int, lr: float,
               beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
               weight_decay: float = 0.0, m_scale=None, v_scale=None, copies=None, clip=None,
               stream=None):
    """gts_adamw: one AdamW step, in place, on params and on the state (m, v and, in 8
    bits, their scales: the fields of adamw_state).  ``copies`` are bfloat16 or float16
    tensors that receive the new values, ``clip`` the result of grad_clip; with gradients
    that are not finite, the step then changes no parameter or state."""
    if len(grads) != len(params) or (copies is not None and len(copies) != len(params)):
        raise ValueError("params, grads and copies must be of one length")
    if not params:
        return
    dtype, dev = _first("params[0]", params[0])
    grad_dtype = _first("grads[0]", grads[0])[0]
    copy_dtype = _first("copies[0]", copies[0])[0] if copies is not None else torch.bfloat16
    at = _addresses("params", params, dtype, dev)
    sizes = tuple([t.numel() for t in params])
    starts, total = _starts(sizes)
    tab = _table(at, _addresses("grads", grads, grad_dtype, dev, sizes), (0,) * len(sizes)
                 if copies is None else _addresses("copies", copies, copy_dtype, dev, sizes),
                 sizes, starts)
    bits = 8 if isinstance(m, torch.Tensor) and m.dtype is torch.float8_e4m3fn else 32
    kind = torch.float8_e4m3fn if bits == 8 else torch.float32
    a = _AdamW(tab.buffer_info()[0], len(sizes), TYPES[dtype], TYPES[grad_dtype],
               TYPES[copy_dtype], bits, _vector("m", m, total, kind, dev),
               _vector("v", v, total, kind, dev))
    if bits == 8:
        a.m_scale = _vector("m_scale", m_scale, total // STATE_BLOCK, torch.float32, dev)
        a.v_scale = _vector("v_scale", v_scale, total // STATE_BLOCK, torch.float32, dev)
    if clip is not None:
        a.d_clip = _vector("clip", clip, 2, torch.float32, dev)
    a.step, a.lr, a.beta1, a.beta2 = step, lr, beta1, beta2
    a.eps, a.weight_decay = eps, weight_decay
    gts._check(_L().gts_adamw(a, _handle(stream, dev)), "gts_adamw")
