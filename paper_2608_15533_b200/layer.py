"""What a recurrent layer runs around its scan: the short causal convolution, the norm and rotation of query and key heads, and
the selective state space scan that takes the scan's place in other layers.

Python face of the "Around the scan" part of ``include/deltalog.h``: checks of types, shapes and devices (``ValueError``),
argument marshalling, and one ``torch.autograd.Function`` per operator.  The work is done by the CUDA kernels behind the C ABI.

Tokens are packed as for the scan (``plan.starts`` says where each row's begin); the single-token calls take one token per row
and a slot list.  A token's own values are dense, while the tokens may be columns of a wider tensor (``proj[:, a:b]``) wherever
the row stride and the address are multiples of 16 bytes.
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass
from typing import Optional, Tuple

import torch
from torch.autograd import forward_ad

from .binding import BF16, HINT_ZERO_UNWRITTEN, _DT_TO_TORCH, _check, _ConvDesc, _ConvGrads, _NormDesc, _SsmDesc, _SsmGrads, _SsmInputs, load_library
from .sequence import Plan, _bytes, _eager, _gpu, _on, _refuse_capture_beside_eager, _want

NORM_L2, NORM_RMS, NORM_NONE = 0, 1, 2


class _Described:
    """A descriptor whose C struct is made once per set of values; the second form asks for zeros in unwritten rows."""

    def __setattr__(self, name, value):
        self.__dict__.pop("_c", None)
        object.__setattr__(self, name, value)

    def _forms(self):
        made = self.__dict__.get("_c")
        if made is None:
            second = self._struct(*self._key())
            second.hints |= HINT_ZERO_UNWRITTEN
            made = self.__dict__["_c"] = (self._struct(*self._key()), second)
        return made

    def c_struct(self, zero: bool = False):
        return self._forms()[1 if zero else 0]


@dataclass
class ConvDesc(_Described):
    """Mirror of ``deltalog_conv_desc``."""

    channels: int
    width: int = 4
    io_dtype: int = BF16
    silu: bool = True
    num_slots: int = 1
    hints: int = 0
    _struct = _ConvDesc

    def _key(self):
        return self.channels, self.width, self.io_dtype, int(self.silu), self.num_slots, self.hints


@dataclass
class SsmDesc(_Described):
    """Mirror of ``deltalog_ssm_desc``."""

    channels: int
    d_state: int = 16
    groups: int = 1
    io_dtype: int = BF16
    softplus: bool = True
    num_slots: int = 1
    hints: int = 0
    _struct = _SsmDesc

    def _key(self):
        return self.channels, self.d_state, self.groups, self.io_dtype, int(self.softplus), self.num_slots, self.hints


@dataclass
class NormDesc(_Described):
    """``deltalog_norm_desc`` without ``table_rows``, which the tables' shape gives."""

    H_q: int
    H_k: int
    d: int
    io_dtype: int = BF16
    norm: int = NORM_L2
    eps: float = 1e-6
    rot: int = 0
    interleaved: bool = False
    q_scale: float = 1.0

    def c_struct(self, table_rows: int = 0):
        made = self.__dict__.get("_c")
        if made is None or made[0] != table_rows:
            made = self.__dict__["_c"] = (table_rows, _NormDesc(self.H_q, self.H_k, self.d, self.io_dtype, self.norm, self.rot, int(self.interleaved),
                                                                table_rows, self.eps, self.q_scale))
        return made[1]


class _Pool:
    """A pool of per-slot states and the status word that step and prefill set bits in.  ``tensor`` None: zeros."""

    def __init__(self, desc, tensor, shape, dtype, device, name):
        self.desc = desc
        if tensor is None:
            tensor = torch.zeros(shape, dtype=dtype, device=device)
        else:
            _want(name, tensor, shape, dtype, tensor.device)
        self._status = torch.zeros(1, dtype=torch.int32, device=tensor.device)
        self._tensor, self._shape, self._seen = tensor, shape, None

    @property
    def status(self) -> torch.Tensor:
        return self._status

    def _fits(self, desc, device):
        """Addresses of the pool and of the status word for a call with this descriptor."""
        forms = desc._forms()
        if forms is not self._seen:  # (a descriptor whose values change makes new ones)
            if self._shape != self._want(desc) or self._tensor.dtype is not self._dtype(desc):
                raise ValueError("state: its tensor was laid out for another descriptor")
            self._seen = forms
        if self._tensor.device != device:
            raise ValueError(f"state: expected a tensor on {device}, got one on {self._tensor.device}")
        return self._tensor.data_ptr(), self._status.data_ptr()


class ConvState(_Pool):
    """``window [num_slots, width - 1, channels]``: the last inputs of every slot's sequence, oldest first.  (A new request whose
    first call is a single token needs its window cleared: ``state.window[slot] = 0``.)"""

    def __init__(self, desc: ConvDesc, window: Optional[torch.Tensor] = None, device="cuda"):
        super().__init__(desc, window, self._want(desc), self._dtype(desc), device, "window")

    @property
    def window(self) -> torch.Tensor:
        return self._tensor

    @staticmethod
    def _want(desc):
        return desc.num_slots, desc.width - 1, desc.channels

    @staticmethod
    def _dtype(desc):
        return _DT_TO_TORCH[desc.io_dtype]


class SsmState(_Pool):
    """``S [num_slots, channels, d_state]`` fp32.  (A new request whose first call is a single token needs its state cleared:
    ``state.S[slot] = 0``.)"""

    def __init__(self, desc: SsmDesc, S: Optional[torch.Tensor] = None, device="cuda"):
        super().__init__(desc, S, self._want(desc), torch.float32, device, "S")

    @property
    def S(self) -> torch.Tensor:
        return self._tensor

    @staticmethod
    def _want(desc):
        return desc.num_slots, desc.channels, desc.d_state

    @staticmethod
    def _dtype(desc):
        return torch.float32


def _tokens(name: str, t, shape: Tuple[int, ...], dtype, device) -> Tuple[int, int]:
    """Pointer and token stride of a tensor [tokens, width] or [tokens, heads, width] of this shape whose tokens are dense."""
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.device == device and t.shape == shape):
        if not isinstance(t, torch.Tensor):
            raise ValueError(f"{name}: a tensor is needed")
        raise ValueError(f"{name}: expected {dtype} {shape} on {device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    width = shape[-1]
    dense = width if len(shape) == 2 else shape[1] * width
    if t.is_contiguous():
        return t.data_ptr() or 16, dense
    strides = t.stride()
    if (strides[-1] != 1 and width != 1) or (len(shape) == 3 and strides[1] != width and shape[1] != 1):
        raise ValueError(f"{name}: a token's values have to be dense, the strides are {strides}")
    stride, at = strides[0] if shape[0] > 1 else dense, t.data_ptr()
    if stride < dense or stride * t.element_size() % 16 or at % 16:
        raise ValueError(f"{name}: the tokens have to start on 16-byte boundaries and not overlap, the strides are {strides}")
    return at, stride


_MOST_ROWS = 0x7fffffff - 64  # the C ABI counts rows in 31 bits


def _rows(name: str, t) -> int:
    if not isinstance(t, torch.Tensor) or t.dim() == 0:
        raise ValueError(f"{name}: a tensor of tokens is needed")
    rows = t.shape[0]
    if rows > _MOST_ROWS:
        raise ValueError(f"{name}: at most {_MOST_ROWS} rows, got {rows}")
    return rows


class _Here:
    """A stream handle as a context: nothing to switch."""

    __slots__ = ("handle",)

    def __init__(self, handle):
        self.handle = handle

    def __enter__(self):
        return self.handle

    def __exit__(self, *exc):
        pass


def _stream_of(device, stream):
    """The context of a call: the current stream as it is, if the device is current and no other stream is asked for; ``_on``
    otherwise."""
    if device.type != "cuda":
        _gpu(device)
    if stream is None and torch._C._cuda_getDevice() == device.index:
        return _Here(torch._C._cuda_getCurrentRawStream(device.index))
    return _on(device, stream)


def _empty(shape: Tuple[int, ...], dtype, device) -> torch.Tensor:
    """A new dense tensor of one to three axes (torch.empty with the strides worked out: half of its time on the host)."""
    if len(shape) == 2:
        strides = shape[1], 1
    else:
        strides = (1,) if len(shape) == 1 else (shape[1] * shape[2], shape[2], 1)
    return torch.empty_strided(shape, strides, dtype=dtype, device=device)


def _zeros(shape, dtype, device) -> torch.Tensor:
    return torch.zeros(shape, dtype=dtype, device=device)


def _param(name: str, t, shape, device) -> Optional[int]:
    return None if t is None else _want(name, t, shape, torch.float32, device)


def _new_out(out, rows: int, shape, dtype, device, plan: Plan) -> Tuple[torch.Tensor, bool]:
    """The caller's output, or a new one whose rows that the call does not write are to be zero (the kernels see to those below
    ``plan.max_tokens``)."""
    if out is not None:
        _want("out", out, shape, dtype, device)
        return out, False
    out = _empty(shape, dtype, device)
    first = plan.max_tokens if plan.n > 0 else 0
    if first < rows:
        out[first:].zero_()
    return out, True


def _plan_rows(name: str, t, plan: Plan) -> int:
    rows = _rows(name, t)
    if rows < plan.max_tokens:
        raise ValueError(f"{name}: the plan reaches over {plan.max_tokens} tokens, the tensor has {rows}")
    return rows


def _slot_list(slot_idx, B: int, num_slots: int, device) -> Optional[int]:
    if slot_idx is None:
        if B > num_slots:
            raise ValueError(f"slot_idx: {B} rows without a list need as many slots, the pool has {num_slots}")
        return None
    return _want("slot_idx", slot_idx, (B,), torch.int32, device)


def _no_tangent(what: str, tensors) -> None:
    if any(isinstance(t, torch.Tensor) and forward_ad.unpack_dual(t).tangent is not None for t in tensors):
        raise RuntimeError(f"{what} has no forward-mode derivative: an argument carries a tangent")


def _entered(ctx, inputs, device) -> None:
    """The rules of scan's captures: no capture beside an eager graph of the same leaves."""
    if torch.cuda.is_current_stream_capturing():
        _refuse_capture_beside_eager(inputs)
    elif torch.cuda.current_stream(device) == torch.cuda.default_stream(device):
        _eager.add(ctx)


def _gradient(g, like: torch.Tensor) -> Optional[torch.Tensor]:
    """A gradient as the kernels want it: dense, of its output's type, on a 16-byte boundary."""
    g = g.to(like.dtype).contiguous()
    return g.clone() if g.data_ptr() % 16 else g


def _differentiable(tensors) -> bool:
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


def _want_workspace(workspace, device) -> torch.Tensor:
    if workspace.device != device or not workspace.is_contiguous():
        raise ValueError(f"workspace: expected a contiguous tensor on {device}")
    return workspace


# ---- causal convolution -------------------------------------------------------------------------------------------------
def conv_step(desc: ConvDesc, state: ConvState, x, weight, bias=None, slot_idx=None, out=None, stream=None) -> torch.Tensor:
    """``deltalog_conv_step``: one token ``x [B, channels]`` per row; row b advances window ``slot_idx[b]`` (b without a list).
    Padding rows (negative slots) and rows outside the pool stay as they were in the caller's ``out`` and are not defined in a
    tensor that the call makes."""
    dev, io, C = state._tensor.device, _DT_TO_TORCH[desc.io_dtype], desc.channels
    B = _rows("x", x)
    p_x, stride = _tokens("x", x, (B, C), io, dev)
    p_w, p_b = _want("weight", weight, (C, desc.width), torch.float32, dev), _param("bias", bias, (C,), dev)
    p_slots = _slot_list(slot_idx, B, desc.num_slots, dev)
    p_win, p_status = state._fits(desc, dev)
    if out is not None:
        _want("out", out, (B, C), io, dev)
    with _stream_of(dev, stream) as handle:
        if out is None:
            out = _empty((B, C), io, dev)
        rc = load_library().deltalog_conv_step(ctypes.byref(desc.c_struct()), p_win, p_x, stride, p_w, p_b, p_slots, B, out.data_ptr() or 16, p_status, handle)
    _check(rc, "deltalog_conv_step")
    return out


def conv_prefill(desc: ConvDesc, state: ConvState, plan: Plan, x, weight, bias=None, fresh=None, out=None, stream=None) -> torch.Tensor:
    """``deltalog_conv_prefill``: the rows of ``plan.scan_slots`` run their tokens ``x [tokens, channels]`` behind their slots'
    windows, which hold the rows' last inputs afterwards.  ``fresh [n]`` int32: rows that start from zeros.  Rows of the output that
    the call does not write: as in ``prefill``."""
    dev, io, C = plan.device, _DT_TO_TORCH[desc.io_dtype], desc.channels
    rows = _plan_rows("x", x, plan)
    p_x, stride = _tokens("x", x, (rows, C), io, dev)
    p_w, p_b = _want("weight", weight, (C, desc.width), torch.float32, dev), _param("bias", bias, (C,), dev)
    p_fresh = None if fresh is None else _want("fresh", fresh, (plan.n,), torch.int32, dev)
    p_win, p_status = state._fits(desc, dev)
    with _stream_of(dev, stream) as handle:
        out, zero = _new_out(out, rows, (rows, C), io, dev, plan)
        rc = load_library().deltalog_conv_prefill(ctypes.byref(desc.c_struct(zero)), p_win, ctypes.byref(plan.c_struct()), p_x, stride, p_w, p_b, p_fresh,
                                                  out.data_ptr() or 16, p_status, handle)
    _check(rc, "deltalog_conv_prefill")
    return out


def conv_forward(desc: ConvDesc, plan: Plan, x, weight, bias=None, init=None, out=None, stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """``deltalog_conv_forward``: row i of the plan starts from ``init[i]`` (zeros without it); returns ``(out, final)`` with
    ``final [n, width - 1, channels]``, the rows' last inputs."""
    dev, io, C = plan.device, _DT_TO_TORCH[desc.io_dtype], desc.channels
    rows, window = _plan_rows("x", x, plan), (plan.n, desc.width - 1, C)
    p_x, stride = _tokens("x", x, (rows, C), io, dev)
    p_w, p_b = _want("weight", weight, (C, desc.width), torch.float32, dev), _param("bias", bias, (C,), dev)
    p_init = None if init is None else _want("init", init, window, io, dev)
    with _stream_of(dev, stream) as handle:
        out, zero = _new_out(out, rows, (rows, C), io, dev, plan)
        final = _empty(window, io, dev)
        rc = load_library().deltalog_conv_forward(ctypes.byref(desc.c_struct(zero)), ctypes.byref(plan.c_struct()), p_init, p_x, stride, p_w, p_b,
                                                  out.data_ptr() or 16, final.data_ptr(), handle)
    _check(rc, "deltalog_conv_forward")
    return out, final


@dataclass
class ConvGrads:
    """Gradients of a convolution, typed like its inputs and dense."""

    x: torch.Tensor
    weight: torch.Tensor
    bias: Optional[torch.Tensor]
    init: torch.Tensor


def conv_workspace(desc: ConvDesc, rows: int, device="cuda") -> torch.Tensor:
    """Workspace for ``conv_backward`` over ``rows`` tokens."""
    bytes_ = load_library().deltalog_conv_workspace_bytes(ctypes.byref(desc.c_struct()), int(rows))
    if bytes_ == 0:
        raise ValueError("the descriptor or the size is not supported")
    return torch.empty(bytes_, dtype=torch.uint8, device=device)


def conv_backward(desc: ConvDesc, plan: Plan, x, weight, bias, dout, init=None, dfinal=None, workspace=None, stream=None) -> ConvGrads:
    """``deltalog_conv_backward``: gradients of ``conv_forward`` for ``dout`` and ``dfinal`` (zeros without it)."""
    dev, io, C = plan.device, _DT_TO_TORCH[desc.io_dtype], desc.channels
    rows, window = _plan_rows("x", x, plan), (plan.n, desc.width - 1, C)
    p_x, stride = _tokens("x", x, (rows, C), io, dev)
    p_w, p_b = _want("weight", weight, (C, desc.width), torch.float32, dev), _param("bias", bias, (C,), dev)
    p_init = None if init is None else _want("init", init, window, io, dev)
    p_dfinal = None if dfinal is None else _want("dfinal", dfinal, window, io, dev)
    p_dout = _want("dout", dout, (rows, C), io, dev) or 16
    with _stream_of(dev, stream) as handle:
        ws = _want_workspace(workspace, dev) if workspace is not None else conv_workspace(desc, rows, dev)
        make = _zeros if plan.n == 0 else _empty  # without rows nothing is launched
        new = ConvGrads(make((rows, C), io, dev), make((C, desc.width), torch.float32, dev), None if bias is None else make((C,), torch.float32, dev),
                        _empty(window, io, dev))
        ptr = _ConvGrads(new.x.data_ptr() or 16, new.weight.data_ptr(), None if bias is None else new.bias.data_ptr(), new.init.data_ptr())
        rc = load_library().deltalog_conv_backward(ctypes.byref(desc.c_struct()), ctypes.byref(plan.c_struct()), p_init, p_x, stride, p_w, p_b, p_dout,
                                                   p_dfinal, ctypes.byref(ptr), rows, ws.data_ptr(), _bytes(ws), handle)
    _check(rc, "deltalog_conv_backward")
    return new


class _Conv(torch.autograd.Function):
    @staticmethod
    def forward(ctx, desc, plan, x, weight, bias, init):
        _entered(ctx, (x, weight, bias, init), plan.device)
        out, final = conv_forward(desc, plan, x, weight, bias, init=init)
        ctx.set_materialize_grads(False)
        ctx.desc, ctx.plan, ctx.builds = desc, plan, plan.builds
        ctx.save_for_backward(x, weight, bias, init)
        return out, final

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout, dfinal):
        x, weight, bias, init = ctx.saved_tensors
        if ctx.plan.builds != ctx.builds:
            raise RuntimeError("the plan of this convolution was rebuilt before its backward pass")
        dout = torch.zeros(x.shape, dtype=x.dtype, device=x.device) if dout is None else _gradient(dout, x)
        dfinal = None if dfinal is None else _gradient(dfinal, x)
        d = conv_backward(ctx.desc, ctx.plan, x, weight, bias, dout, init=init, dfinal=dfinal)
        return None, None, d.x, d.weight, d.bias, None if init is None else d.init


def conv(desc: ConvDesc, plan: Plan, x, weight, bias=None, init=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """The differentiable convolution: ``(out, final)`` of the plan's rows with gradients for every tensor argument.  What
    ``scan`` says about rows behind the last sequence, rebuilt plans, captures and forward mode holds here too."""
    _no_tangent("conv", (x, weight, bias, init))
    _gpu(plan.device)
    if _differentiable((x, weight, bias, init)):
        return _Conv.apply(desc, plan, x, weight, bias, init)
    return conv_forward(desc, plan, x, weight, bias, init=init)


# ---- selective state space scan -----------------------------------------------------------------------------------------
def ssm_workspace(desc: SsmDesc, n: int, max_tokens: int, train: bool = False, device="cuda") -> torch.Tensor:
    """Workspace for ``ssm_prefill`` / ``ssm_forward`` (``train=False``), or for ``save=True`` and ``ssm_backward`` (then
    ``max_tokens`` is the rows of the token tensors)."""
    bytes_ = load_library().deltalog_ssm_workspace_bytes(ctypes.byref(desc.c_struct()), int(n), int(max_tokens), int(bool(train)))
    if bytes_ == 0:
        raise ValueError("the descriptor or the sizes are not supported")
    return torch.empty(bytes_, dtype=torch.uint8, device=device)


def _ssm_inputs(desc: SsmDesc, rows: int, x, dt, A, B, C, D, z, dt_bias, dev) -> _SsmInputs:
    io, ch = _DT_TO_TORCH[desc.io_dtype], desc.channels
    tokens, states = (rows, ch), (rows, desc.groups, desc.d_state)
    p_x, s_x = _tokens("x", x, tokens, io, dev)
    p_dt, s_dt = _tokens("dt", dt, tokens, io, dev)
    p_B, s_B = _tokens("B", B, states, io, dev)
    p_C, s_C = _tokens("C", C, states, io, dev)
    p_z, s_z = (None, 0) if z is None else _tokens("z", z, tokens, io, dev)
    p_A = _want("A", A, (ch, desc.d_state), torch.float32, dev)
    return _SsmInputs(p_x, p_dt, p_B, p_C, p_z, s_x, s_dt, s_B, s_C, s_z, p_A, _param("D", D, (ch,), dev), _param("dt_bias", dt_bias, (ch,), dev))


def ssm_step(desc: SsmDesc, state: SsmState, x, dt, A, B, C, D=None, z=None, dt_bias=None, slot_idx=None, out=None, stream=None) -> torch.Tensor:
    """``deltalog_ssm_step``: one token per row; row b advances state ``slot_idx[b]`` (b without a list).  Rows that the call
    skips: as in ``conv_step``."""
    dev, io = state._tensor.device, _DT_TO_TORCH[desc.io_dtype]
    rows = _rows("x", x)
    inputs = _ssm_inputs(desc, rows, x, dt, A, B, C, D, z, dt_bias, dev)
    p_slots = _slot_list(slot_idx, rows, desc.num_slots, dev)
    p_S, p_status = state._fits(desc, dev)
    if (p_S | inputs.A) % 32:
        raise ValueError("state, A: the single-token call wants them on 32-byte boundaries")
    if out is not None:
        _want("out", out, (rows, desc.channels), io, dev)
    with _stream_of(dev, stream) as handle:
        if out is None:
            out = _empty((rows, desc.channels), io, dev)
        rc = load_library().deltalog_ssm_step(ctypes.byref(desc.c_struct()), p_S, ctypes.byref(inputs), p_slots, rows, out.data_ptr() or 16, p_status, handle)
    _check(rc, "deltalog_ssm_step")
    return out


def ssm_prefill(desc: SsmDesc, state: SsmState, plan: Plan, x, dt, A, B, C, D=None, z=None, dt_bias=None, fresh=None, out=None, workspace=None,
                stream=None) -> torch.Tensor:
    """``deltalog_ssm_prefill``: the rows of ``plan.scan_slots`` run their tokens through their slots' states; returns ``out
    [tokens, channels]``.  ``fresh`` and rows that the call does not write: as in ``prefill``."""
    dev, io = plan.device, _DT_TO_TORCH[desc.io_dtype]
    rows = _plan_rows("x", x, plan)
    inputs = _ssm_inputs(desc, rows, x, dt, A, B, C, D, z, dt_bias, dev)
    p_fresh = None if fresh is None else _want("fresh", fresh, (plan.n,), torch.int32, dev)
    p_S, p_status = state._fits(desc, dev)
    with _stream_of(dev, stream) as handle:
        out, zero = _new_out(out, rows, (rows, desc.channels), io, dev, plan)
        ws = _want_workspace(workspace, dev) if workspace is not None else ssm_workspace(desc, plan.n, plan.max_tokens, device=dev)
        rc = load_library().deltalog_ssm_prefill(ctypes.byref(desc.c_struct(zero)), p_S, ctypes.byref(plan.c_struct()), ctypes.byref(inputs), p_fresh,
                                                 out.data_ptr() or 16, p_status, ws.data_ptr(), _bytes(ws), handle)
    _check(rc, "deltalog_ssm_prefill")
    return out


def ssm_forward(desc: SsmDesc, plan: Plan, x, dt, A, B, C, D=None, z=None, dt_bias=None, S_init=None, out=None, workspace=None, save: bool = False,
                stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """``deltalog_ssm_forward``: row i of the plan starts from ``S_init[i]`` (zeros without it); returns ``(out, S_final)`` with
    ``S_final [n, channels, d_state]`` fp32.  ``save``: the workspace (``ssm_workspace(.., train=True)``) keeps what
    ``ssm_backward(.., saved=True)`` reads."""
    dev, io = plan.device, _DT_TO_TORCH[desc.io_dtype]
    rows = _plan_rows("x", x, plan)
    inputs = _ssm_inputs(desc, rows, x, dt, A, B, C, D, z, dt_bias, dev)
    s_shape = (plan.n, desc.channels, desc.d_state)
    p_init = None if S_init is None else _want("S_init", S_init, s_shape, torch.float32, dev)
    if save and workspace is None:
        raise ValueError("workspace: save=True needs the caller's workspace, which ssm_backward reads")
    with _stream_of(dev, stream) as handle:
        out, zero = _new_out(out, rows, (rows, desc.channels), io, dev, plan)
        ws = _want_workspace(workspace, dev) if workspace is not None else ssm_workspace(desc, plan.n, plan.max_tokens, device=dev)
        S_final = _empty(s_shape, torch.float32, dev)
        rc = load_library().deltalog_ssm_forward(ctypes.byref(desc.c_struct(zero)), ctypes.byref(plan.c_struct()), p_init, ctypes.byref(inputs),
                                                 out.data_ptr() or 16, S_final.data_ptr(), int(bool(save)), ws.data_ptr(), _bytes(ws), handle)
    _check(rc, "deltalog_ssm_forward")
    return out, S_final


@dataclass
class SsmGrads:
    """Gradients of a state space scan, typed like its inputs and dense; None where there is no such input."""

    x: torch.Tensor
    dt: torch.Tensor
    A: torch.Tensor
    B: torch.Tensor
    C: torch.Tensor
    D: Optional[torch.Tensor]
    z: Optional[torch.Tensor]
    dt_bias: Optional[torch.Tensor]
    S_init: torch.Tensor


def ssm_backward(desc: SsmDesc, plan: Plan, x, dt, A, B, C, D, z, dt_bias, dout, S_init=None, dS_final=None, workspace=None, saved: bool = False,
                 stream=None) -> SsmGrads:
    """``deltalog_ssm_backward``: gradients of ``ssm_forward`` for ``dout`` and ``dS_final`` (zeros without it).  ``saved``: the
    workspace is the one that ``ssm_forward(.., save=True)`` left for these inputs; otherwise its states are computed again."""
    dev, io, ch = plan.device, _DT_TO_TORCH[desc.io_dtype], desc.channels
    rows = _plan_rows("x", x, plan)
    inputs = _ssm_inputs(desc, rows, x, dt, A, B, C, D, z, dt_bias, dev)
    s_shape = (plan.n, ch, desc.d_state)
    p_init = None if S_init is None else _want("S_init", S_init, s_shape, torch.float32, dev)
    p_dS = None if dS_final is None else _want("dS_final", dS_final, s_shape, torch.float32, dev)
    p_dout = _want("dout", dout, (rows, ch), io, dev) or 16
    if saved and workspace is None:
        raise ValueError("workspace: saved=True needs the workspace of ssm_forward")
    with _stream_of(dev, stream) as handle:
        ws = _want_workspace(workspace, dev) if workspace is not None else ssm_workspace(desc, plan.n, rows, train=True, device=dev)
        make = _zeros if plan.n == 0 else _empty  # without rows nothing is launched

        def grad(t, dtype):
            return None if t is None else make(tuple(t.shape), dtype, dev)

        new = SsmGrads(grad(x, io), grad(dt, io), grad(A, torch.float32), grad(B, io), grad(C, io), grad(D, torch.float32), grad(z, io),
                       grad(dt_bias, torch.float32), _empty(s_shape, torch.float32, dev))
        ptr = _SsmGrads(*(None if t is None else t.data_ptr() or 16 for t in (new.x, new.dt, new.B, new.C, new.z, new.A, new.D, new.dt_bias)),
                        new.S_init.data_ptr())
        rc = load_library().deltalog_ssm_backward(ctypes.byref(desc.c_struct()), ctypes.byref(plan.c_struct()), p_init, ctypes.byref(inputs), p_dout, p_dS,
                                                  int(bool(saved)), ctypes.byref(ptr), rows, ws.data_ptr(), _bytes(ws), handle)
    _check(rc, "deltalog_ssm_backward")
    return new


class _Ssm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, desc, plan, x, dt, A, B, C, D, z, dt_bias, S_init):
        inputs = (x, dt, A, B, C, D, z, dt_bias, S_init)
        _entered(ctx, inputs, plan.device)
        ws = ssm_workspace(desc, plan.n, x.shape[0], train=True, device=plan.device)
        out, S_final = ssm_forward(desc, plan, x, dt, A, B, C, D, z, dt_bias, S_init=S_init, workspace=ws, save=True)
        ctx.set_materialize_grads(False)
        ctx.desc, ctx.plan, ctx.builds = desc, plan, plan.builds
        ctx.save_for_backward(*inputs, ws)
        return out, S_final

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout, dS_final):
        x, dt, A, B, C, D, z, dt_bias, S_init, ws = ctx.saved_tensors
        if ctx.plan.builds != ctx.builds:
            raise RuntimeError("the plan of this scan was rebuilt before its backward pass")
        dout = torch.zeros(x.shape, dtype=x.dtype, device=x.device) if dout is None else _gradient(dout, x)
        dS_final = None if dS_final is None else _gradient(dS_final, A)
        d = ssm_backward(ctx.desc, ctx.plan, x, dt, A, B, C, D, z, dt_bias, dout, S_init=S_init, dS_final=dS_final, workspace=ws, saved=True)
        return None, None, d.x, d.dt, d.A, d.B, d.C, d.D, d.z, d.dt_bias, None if S_init is None else d.S_init


def ssm(desc: SsmDesc, plan: Plan, x, dt, A, B, C, D=None, z=None, dt_bias=None, S_init=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """The differentiable state space scan: ``(out, S_final)`` of the plan's rows with gradients for every tensor argument.  What
    ``scan`` says about rows behind the last sequence, rebuilt plans, captures and forward mode holds here too."""
    tensors = (x, dt, A, B, C, D, z, dt_bias, S_init)
    _no_tangent("ssm", tensors)
    _gpu(plan.device)
    if _differentiable(tensors):
        _plan_rows("x", x, plan)
        return _Ssm.apply(desc, plan, *tensors)
    return ssm_forward(desc, plan, x, dt, A, B, C, D, z, dt_bias, S_init=S_init)


# ---- norm and rotation of heads -----------------------------------------------------------------------------------------
def _norm_inputs(desc: NormDesc, q, k, w_q, w_k, cos, sin, positions):
    """The call's descriptor and the pointers of its inputs, checked; and the tokens."""
    rows = _rows("q", q)
    dev, io, d = q.device, _DT_TO_TORCH[desc.io_dtype], desc.d
    p_q, s_q = _tokens("q", q, (rows, desc.H_q, d), io, dev)
    if desc.H_k:
        p_k, s_k = _tokens("k", k, (rows, desc.H_k, d), io, dev)
    elif k is not None:
        raise ValueError("k: the descriptor has no key heads")
    else:
        p_k, s_k = None, 0
    if (w_q is not None or w_k is not None) and desc.norm != NORM_RMS:
        raise ValueError("w_q, w_k: only the RMS norm has weights")
    if desc.H_k and (w_q is None) != (w_k is None):
        raise ValueError("w_q, w_k: both or neither")
    p_wq, p_wk = _param("w_q", w_q, (d,), dev), _param("w_k", w_k, (d,), dev)
    p_cos = p_sin = p_pos = None
    c = desc
    if desc.rot:
        p_cos = _want("cos", cos, (None, desc.rot // 2), torch.float32, dev)
        p_sin = _want("sin", sin, tuple(cos.shape), torch.float32, dev)
        p_pos = _want("positions", positions, (rows,), torch.int32, dev) or 16
        c = desc.c_struct(cos.shape[0])
    else:
        c = desc.c_struct()
    return c, rows, (p_q, s_q, p_k, s_k, p_wq, p_wk, p_cos, p_sin, p_pos, rows)


def head_norm_forward(desc: NormDesc, q, k, w_q=None, w_k=None, cos=None, sin=None, positions=None, out_q=None, out_k=None, status=None,
                      stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """``deltalog_head_norm_forward``: ``q [tokens, H_q, d]`` and ``k [tokens, H_k, d]`` normalised, rotated by their tokens'
    ``positions [tokens]`` and, the queries, scaled.  ``status`` (int32, one word) receives ``STATUS_BAD_POSITION``."""
    c, rows, ptr = _norm_inputs(desc, q, k, w_q, w_k, cos, sin, positions)
    dev, io, d = q.device, q.dtype, desc.d
    if out_q is not None:
        _want("out_q", out_q, (rows, desc.H_q, d), io, dev)
    if out_k is not None:
        _want("out_k", out_k, (rows, desc.H_k, d), io, dev)
    p_status = None if status is None else _want("status", status, (1,), torch.int32, dev)
    with _stream_of(dev, stream) as handle:
        if out_q is None:
            out_q = _empty((rows, desc.H_q, d), io, dev)
        if out_k is None and desc.H_k:
            out_k = _empty((rows, desc.H_k, d), io, dev)
        rc = load_library().deltalog_head_norm_forward(ctypes.byref(c), *ptr, out_q.data_ptr() or 16, (out_k.data_ptr() or 16) if desc.H_k else None,
                                                       p_status, handle)
    _check(rc, "deltalog_head_norm_forward")
    return out_q, out_k


@dataclass
class HeadNormGrads:
    """Gradients of head_norm, typed like its inputs and dense; None where there is no such input."""

    q: torch.Tensor
    k: Optional[torch.Tensor]
    w_q: Optional[torch.Tensor]
    w_k: Optional[torch.Tensor]


def head_norm_backward(desc: NormDesc, q, k, w_q, w_k, cos, sin, positions, dout_q, dout_k, workspace=None, stream=None) -> HeadNormGrads:
    """``deltalog_head_norm_backward``: gradients of ``head_norm_forward``; cos and sin have none."""
    c, rows, ptr = _norm_inputs(desc, q, k, w_q, w_k, cos, sin, positions)
    dev, io, d = q.device, q.dtype, desc.d
    p_dq = _want("dout_q", dout_q, (rows, desc.H_q, d), io, dev) or 16
    p_dk = (_want("dout_k", dout_k, (rows, desc.H_k, d), io, dev) or 16) if desc.H_k else None
    with _stream_of(dev, stream) as handle:
        lib = load_library()
        if workspace is None:
            bytes_ = lib.deltalog_head_norm_workspace_bytes(ctypes.byref(c), rows) if w_q is not None else 0
            workspace = torch.empty(max(bytes_, 16), dtype=torch.uint8, device=dev)
        ws = _want_workspace(workspace, dev)
        new = HeadNormGrads(_empty((rows, desc.H_q, d), io, dev), _empty((rows, desc.H_k, d), io, dev) if desc.H_k else None,
                            None if w_q is None else torch.empty_like(w_q), None if w_k is None else torch.empty_like(w_k))
        rc = lib.deltalog_head_norm_backward(ctypes.byref(c), *ptr, p_dq, p_dk, new.q.data_ptr() or 16, None if new.k is None else new.k.data_ptr() or 16,
                                             None if w_q is None else new.w_q.data_ptr(), None if w_k is None else new.w_k.data_ptr(), ws.data_ptr(),
                                             _bytes(ws), handle)
    _check(rc, "deltalog_head_norm_backward")
    return new


class _HeadNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, desc, q, k, w_q, w_k, cos, sin, positions):
        _entered(ctx, (q, k, w_q, w_k), q.device)
        out = head_norm_forward(desc, q, k, w_q, w_k, cos, sin, positions)
        ctx.set_materialize_grads(False)
        ctx.desc = desc
        ctx.save_for_backward(q, k, w_q, w_k, cos, sin, positions)
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout_q, dout_k):
        q, k, w_q, w_k, cos, sin, positions = ctx.saved_tensors

        def whole(g, like):
            if like is None:
                return None
            return torch.zeros(like.shape, dtype=like.dtype, device=like.device) if g is None else _gradient(g, like)

        d = head_norm_backward(ctx.desc, q, k, w_q, w_k, cos, sin, positions, whole(dout_q, q), whole(dout_k, k))
        return None, d.q, d.k, d.w_q, d.w_k, None, None, None


def head_norm(desc: NormDesc, q, k, w_q=None, w_k=None, cos=None, sin=None, positions=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """The differentiable form of ``head_norm_forward``, with gradients for q, k and the weights.  Captures and forward mode: as
    in ``scan``."""
    tensors = (q, k, w_q, w_k)
    _no_tangent("head_norm", tensors + (cos, sin))
    if any(isinstance(t, torch.Tensor) and t.requires_grad for t in (cos, sin)):
        raise ValueError("cos, sin: the rotation's tables have no gradient")
    if _differentiable(tensors):
        _norm_inputs(desc, q, k, w_q, w_k, cos, sin, positions)
        _gpu(q.device)
        return _HeadNorm.apply(desc, q, k, w_q, w_k, cos, sin, positions)
    return head_norm_forward(desc, q, k, w_q, w_k, cos, sin, positions)
