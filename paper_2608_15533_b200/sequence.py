"""Whole sequences: the plan of a step, prefill into the slot pool, and the trainable scan.

Python face of the "Sequences" part of ``include/deltalog.h``: checks of types, shapes and devices (``ValueError``),
argument marshalling, and one ``torch.autograd.Function``.  The work is done by the CUDA kernels behind the C ABI.

Token tensors are packed: ``q, k [tokens, H_qk, d_k]``, ``v [tokens, H, d_v]``, ``g [tokens, H]`` or ``[tokens, H, d_k]``
fp32 log-decay, ``beta [tokens, H]`` fp32, ``u_bonus [H, d_k]`` fp32; ``plan.starts`` says where each row's tokens begin.
"""
from __future__ import annotations

import ctypes
import weakref
from dataclasses import dataclass
from typing import Optional, Tuple

import torch
from torch.autograd import forward_ad

from . import binding
from .binding import (
    BF16, F32, HINT_ZERO_UNWRITTEN, RWKV6, Desc, State, _DELTA_RULE, _DT_TO_TORCH, _check, _Desc, _Plan, _ScanGrads, _VEC_DECAY, load_library,
)

SCAN_CHUNK = 64
_STATE_FIELDS = ("num_slots", "H", "d_k", "d_v", "cap", "d_lambda", "base_dtype", "klog_dtype", "ulog_dtype")


def _want(name: str, t: Optional[torch.Tensor], shape, dtype, device) -> Optional[int]:
    """Pointer of a contiguous tensor of this shape, type and device; ValueError otherwise.  A shape entry of None is any
    size."""
    if isinstance(t, torch.Tensor) and t.shape == shape and t.dtype is dtype and t.device == device and t.is_contiguous():
        return t.data_ptr()
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name}: a tensor is needed")
    if t.dtype != dtype or t.device != device or t.dim() != len(shape) or any(s is not None and s != x for s, x in zip(shape, t.shape)):
        raise ValueError(f"{name}: expected {dtype} {tuple(shape)} on {device}, got {t.dtype} {tuple(t.shape)} on {t.device}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: the tensor has to be contiguous")
    return t.data_ptr()


class _on:
    """A call's device and stream made current around it, where they are not already: the call's own buffers then belong to
    the stream that its kernels run on.  Yields the stream's handle."""

    __slots__ = ("index", "stream", "before")

    def __init__(self, device, stream):
        if stream is not None and not isinstance(stream, torch.cuda.Stream):
            handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
            stream = torch.cuda.ExternalStream(handle, device=device) if handle else torch.cuda.default_stream(device)
        if stream is not None and stream.device != device:
            raise ValueError(f"stream: the tensors are on {device}, the stream is of {stream.device}")
        self.index, self.stream = device.index, stream

    def __enter__(self):
        self.before = torch.cuda.current_device()
        if self.before != self.index:
            torch.cuda.set_device(self.index)
        if self.stream is None:
            return torch.cuda.current_stream().cuda_stream
        self.stream, asked = torch.cuda.current_stream(), self.stream
        torch.cuda.set_stream(asked)
        return asked.cuda_stream

    def __exit__(self, *exc):
        if self.stream is not None:
            torch.cuda.set_stream(self.stream)
        if self.before != self.index:
            torch.cuda.set_device(self.before)


def _gpu(device) -> None:
    if device.type != "cuda":
        raise ValueError(f"the plan's tables are on {device}: there is no path but the GPU's")


class Plan:
    """Device tables of a plan for ``n`` rows of ``max_tokens`` tokens together at most (``build_plan`` fills them)."""

    def __init__(self, n: int, max_tokens: int, device="cuda", token_map: bool = True):
        if n < 0 or max_tokens < 0 or n + max_tokens > 2 ** 31 - 65:
            raise ValueError("a plan needs 0 <= n, 0 <= max_tokens and a sum below 2^31 - 64")
        self.n, self.max_tokens = int(n), int(max_tokens)

        def table(size):
            return torch.zeros(size, dtype=torch.int32, device=device)

        self.starts, self.chunk_starts = table(n + 1), table(n + 1)
        self.chunk_seq = torch.full((max(1, max_tokens // SCAN_CHUNK + n),), -1, dtype=torch.int32, device=device)[: max_tokens // SCAN_CHUNK + n]
        self.token_seq = table(max_tokens) if token_map and max_tokens > 0 else None
        self.scan_slots, self.append_slots, self.merge_slots = (torch.full((max(1, n),), -1, dtype=torch.int32, device=device)[:n] for _ in range(3))
        self.totals = table(4)
        self.status = table(1)   # STATUS_* bits of the scans over this plan
        self.builds = 0   # how often build_plan has filled the tables
        self.device = self.starts.device

    def c_struct(self) -> _Plan:
        if "_c" not in self.__dict__:
            # zero-sized views keep the address of their one-element storage
            ptr = [None if t is None else t.untyped_storage().data_ptr() + t.storage_offset() * 4 for t in (
                self.starts, self.chunk_starts, self.chunk_seq, self.token_seq, self.scan_slots, self.append_slots, self.merge_slots, self.totals, self.status)]
            self._c = _Plan(self.n, self.max_tokens, *ptr)
        return self._c


def build_plan(lens: torch.Tensor, plan: Plan, slots: Optional[torch.Tensor] = None, log_len: Optional[torch.Tensor] = None, cap: int = 0,
               decode_rows: bool = False, stream=None) -> Plan:
    """``deltalog_build_plan``: fill ``plan`` from ``lens [n]`` (tokens that each row brings), on the GPU and without a
    synchronisation.

    ``slots [n]``: the rows' slots (row i: slot i without it).  ``decode_rows``: rows with one token decode; they are listed in
    ``plan.append_slots`` or, where ``log_len [num_slots, H]`` holds ``cap`` entries, in ``plan.merge_slots``, and the longer
    ones in ``plan.scan_slots``.  Returns ``plan``.
    """
    dev = plan.device
    p_lens = _want("lens", lens, (plan.n,), torch.int32, dev)
    p_slots = None if slots is None else _want("slots", slots, (plan.n,), torch.int32, dev)
    p_log, H, num = None, 0, 0
    if log_len is not None:
        p_log = _want("log_len", log_len, (None, None), torch.int32, dev)
        num, H = log_len.shape
    _gpu(dev)
    with _on(dev, stream) as handle:
        rc = load_library().deltalog_build_plan(p_lens if plan.n else None, p_slots, p_log, int(H), int(cap), int(num), int(bool(decode_rows)),
                                                ctypes.byref(plan.c_struct()), handle)
    _check(rc, "deltalog_build_plan")
    plan.builds += 1
    return plan


def scan_workspace(desc: Desc, n: int, max_tokens: int, train: bool = False, device="cuda") -> torch.Tensor:
    """Workspace for ``prefill`` / ``scan_forward`` (``train=False``) or for ``save=True`` and ``scan_backward``."""
    bytes_ = load_library().deltalog_scan_workspace_bytes(ctypes.byref(desc.c_struct()), int(n), int(max_tokens), int(bool(train)))
    if bytes_ == 0 and n > 0:
        raise ValueError("the descriptor or the sizes are not supported")
    return torch.empty(bytes_, dtype=torch.uint8, device=device)


class _Tokens:
    """Checked pointers of a call's token tensors."""

    def __init__(self, desc: Desc, plan: Plan, q, k, v, g, beta, u_bonus):
        io, H = _DT_TO_TORCH[desc.io_dtype], desc.H
        Hqk = desc.H_qk or H
        self.device, self.rows = plan.device, q.shape[0] if isinstance(q, torch.Tensor) else 0
        if self.rows < plan.max_tokens:
            raise ValueError(f"q: the plan reaches over {plan.max_tokens} tokens, the tensor has {self.rows}")
        rows = self.rows
        gate = (rows, H, desc.d_k) if desc.op in _VEC_DECAY else (rows, H)
        self.ptr = [_want("q", q, (rows, Hqk, desc.d_k), io, self.device), _want("k", k, (rows, Hqk, desc.d_k), io, self.device),
                    _want("v", v, (rows, H, desc.d_v), io, self.device),
                    None if desc.op == binding.LINATTN else _want("g", g, gate, torch.float32, self.device),
                    _want("beta", beta, (rows, H), torch.float32, self.device) if desc.op in _DELTA_RULE else None,
                    _want("u_bonus", u_bonus, (H, desc.d_k), torch.float32, self.device) if desc.op == RWKV6 else None]
        self.out_shape, self.io = (rows, H, desc.d_v), io
        if rows == 0:  # an empty tensor has no address; the calls see that there is nothing to do
            self.ptr = [p or 16 if p is not None else None for p in self.ptr]


def _workspace(desc, plan, workspace, train) -> torch.Tensor:
    if workspace is None:
        return scan_workspace(desc, plan.n, plan.max_tokens, train=train, device=plan.device)
    if workspace.device != plan.device or not workspace.is_contiguous():
        raise ValueError(f"workspace: expected a contiguous tensor on {plan.device}")
    return workspace


def _out_ok(out, tk: _Tokens) -> None:
    if out is not None:
        _want("out", out, tk.out_shape, tk.io, tk.device)


def _out(out, tk: _Tokens, desc: Desc, plan: Plan):
    """The output tensor and the call's descriptor: the caller's own, or a new tensor whose rows that the call does not write
    are to be zero (the kernels see to those below ``plan.max_tokens``)."""
    d = desc.c_struct()
    if out is not None:
        return out, d
    out = torch.empty(tk.out_shape, dtype=tk.io, device=tk.device)
    first = plan.max_tokens if plan.n > 0 else 0
    if first < tk.rows:
        out[first:].zero_()
    cached = desc.__dict__.get("_c_zero")
    if cached is None or cached[0] is not d:
        zero = _Desc.from_buffer_copy(d)
        zero.hints |= HINT_ZERO_UNWRITTEN
        cached = desc.__dict__["_c_zero"] = (d, zero)
    return out, cached[1]


def _bytes(t: torch.Tensor) -> int:
    return t.numel() * t.element_size()


def prefill(desc: Desc, state: State, plan: Plan, q, k, v, g=None, beta=None, u_bonus=None, fresh: Optional[torch.Tensor] = None, out=None,
            workspace=None, stream=None) -> torch.Tensor:
    """``deltalog_prefill``: the rows of ``plan.scan_slots`` run their tokens through their slots' states; returns
    ``out [tokens, H, d_v]``.  ``fresh [n]`` int32: rows that start from a zero state.  The slots' logs are empty afterwards.
    Output rows that no row of the call writes (decoding, padding and dropped rows, behind the last sequence) stay as they were
    in the caller's ``out``; in a tensor that the call makes they are zero."""
    tk = _Tokens(desc, plan, q, k, v, g, beta, u_bonus)
    dev = tk.device
    p_fresh = None if fresh is None else _want("fresh", fresh, (plan.n,), torch.int32, dev)
    if state.S_base.device != dev:
        raise ValueError(f"state: expected tensors on {dev}")
    if state.desc is not desc and any(getattr(state.desc, x) != getattr(desc, x) for x in _STATE_FIELDS):
        raise ValueError("state: its tensors were laid out for another descriptor")
    _out_ok(out, tk)
    _gpu(dev)
    with _on(dev, stream) as handle:
        (out, d), ws = _out(out, tk, desc, plan), _workspace(desc, plan, workspace, False)
        rc = load_library().deltalog_prefill(ctypes.byref(d), ctypes.byref(state.c_struct()), ctypes.byref(plan.c_struct()), *tk.ptr,
                                             p_fresh, out.data_ptr() or 16, ws.data_ptr(), _bytes(ws), handle)
    _check(rc, "deltalog_prefill")
    return out


def scan_forward(desc: Desc, plan: Plan, q, k, v, g=None, beta=None, u_bonus=None, S_init=None, out=None, workspace=None, save: bool = False,
                 stream=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """``deltalog_scan_forward``: row i of the plan starts from ``S_init[i]`` (zeros without it); returns ``(out, S_final)``
    with ``S_final [n, H, d_k, d_v]`` fp32.  ``save``: the workspace (``scan_workspace(.., train=True)``) keeps what
    ``scan_backward(.., saved=True)`` reads.  Rows behind the last sequence: as in ``prefill``."""
    tk = _Tokens(desc, plan, q, k, v, g, beta, u_bonus)
    dev, s_shape = tk.device, (plan.n, desc.H, desc.d_k, desc.d_v)
    p_init = None if S_init is None else _want("S_init", S_init, s_shape, torch.float32, dev)
    if save and workspace is None:
        raise ValueError("workspace: save=True needs the caller's workspace, which scan_backward reads")
    _out_ok(out, tk)
    _gpu(dev)
    with _on(dev, stream) as handle:
        (out, d), ws = _out(out, tk, desc, plan), _workspace(desc, plan, workspace, save)
        S_final = torch.empty(s_shape, dtype=torch.float32, device=dev)
        rc = load_library().deltalog_scan_forward(ctypes.byref(d), ctypes.byref(plan.c_struct()), p_init, *tk.ptr,
                                                  out.data_ptr() or 16, S_final.data_ptr(), int(bool(save)), ws.data_ptr(), _bytes(ws), handle)
    _check(rc, "deltalog_scan_forward")
    return out, S_final


@dataclass
class ScanGrads:
    """Gradients of a scan, typed and laid out like its inputs; None where the operator has no such input."""

    q: torch.Tensor
    k: torch.Tensor
    v: torch.Tensor
    g: Optional[torch.Tensor]
    beta: Optional[torch.Tensor]
    u_bonus: Optional[torch.Tensor]
    S_init: torch.Tensor


def scan_backward(desc: Desc, plan: Plan, q, k, v, g, beta, u_bonus, dout, S_init=None, dS_final=None, workspace=None, saved: bool = False,
                  stream=None) -> ScanGrads:
    """``deltalog_scan_backward``: gradients of ``scan_forward`` for ``dout`` and ``dS_final`` (zeros without it).  ``saved``: the
    workspace is the one that ``scan_forward(.., save=True)`` left for these inputs; otherwise its states are computed again."""
    tk = _Tokens(desc, plan, q, k, v, g, beta, u_bonus)
    dev, s_shape = tk.device, (plan.n, desc.H, desc.d_k, desc.d_v)
    p_init = None if S_init is None else _want("S_init", S_init, s_shape, torch.float32, dev)
    p_dS = None if dS_final is None else _want("dS_final", dS_final, s_shape, torch.float32, dev)
    p_dout = _want("dout", dout, tk.out_shape, tk.io, dev) or 16
    if saved and workspace is None:
        raise ValueError("workspace: saved=True needs the workspace of scan_forward")
    _gpu(dev)
    with _on(dev, stream) as handle:
        ws = _workspace(desc, plan, workspace, True)
        # without rows nothing is launched, and the token tensors' rows are all behind the last sequence
        make = torch.zeros_like if plan.n == 0 else torch.empty_like
        new = ScanGrads(*(None if p is None else make(t) for p, t in zip(tk.ptr, (q, k, v, g, beta, u_bonus))),
                        torch.empty(s_shape, dtype=torch.float32, device=dev))
        ptr = _ScanGrads(*(None if t is None else t.data_ptr() or 16 for t in (new.q, new.k, new.v, new.g, new.beta, new.u_bonus, new.S_init)))
        rc = load_library().deltalog_scan_backward(ctypes.byref(desc.c_struct()), ctypes.byref(plan.c_struct()), p_init, *tk.ptr, p_dout, p_dS,
                                                   int(bool(saved)), ctypes.byref(ptr), tk.rows, ws.data_ptr(), _bytes(ws), handle)
    _check(rc, "deltalog_scan_backward")
    return new


_eager = weakref.WeakSet()  # graph nodes of the scans that ran on the default stream, outside of a capture


def _leaves(nodes) -> list:
    """The leaf tensors whose gradients graphs with these nodes at their ends accumulate."""
    found, seen, todo = [], set(), [n for n in nodes if n is not None]
    while todo:
        node = todo.pop()
        if node in seen:
            continue
        seen.add(node)
        if hasattr(node, "variable"):
            found.append(node.variable)
        todo += [n for n, _ in node.next_functions if n is not None]
    return found


def _refuse_capture_beside_eager(inputs) -> None:
    """A leaf's gradient is accumulated on the stream that its first graph was built on, and as long as that graph lives a later
    one shares the place.  A captured backward pass would have to leave for the default stream, which a capture does not
    survive, and with it the process may end.  The leaves are the inputs themselves or what they were computed from."""
    eager = _leaves(list(_eager))
    asked = [t for t in inputs if t is not None and t.requires_grad]
    mine = [t for t in asked if t.is_leaf] + _leaves([t.grad_fn for t in asked])
    if any(x is y for x in mine for y in eager):
        raise RuntimeError("a graph of the same leaves, built on the default stream, is alive: drop its outputs before the capture, or "
                           "build it on a side stream")


class _Scan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, desc, plan, q, k, v, g, beta, u_bonus, S_init):
        inputs = (q, k, v, g, beta, u_bonus, S_init)
        if torch.cuda.is_current_stream_capturing():
            _refuse_capture_beside_eager(inputs)
        elif torch.cuda.current_stream(plan.device) == torch.cuda.default_stream(plan.device):
            _eager.add(ctx)
        ws = scan_workspace(desc, plan.n, plan.max_tokens, train=True, device=plan.device)
        out, S_final = scan_forward(desc, plan, q, k, v, g, beta, u_bonus, S_init=S_init, workspace=ws, save=True)
        ctx.set_materialize_grads(False)
        ctx.desc, ctx.plan, ctx.builds = desc, plan, plan.builds
        ctx.save_for_backward(*inputs, ws)
        return out, S_final

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout, dS_final):
        q, k, v, g, beta, u_bonus, S_init, ws = ctx.saved_tensors
        if ctx.plan.builds != ctx.builds:
            raise RuntimeError("the plan of this scan was rebuilt before its backward pass")
        dout = torch.zeros_like(v) if dout is None else dout.to(v.dtype).contiguous()
        if dout.data_ptr() % 16:  # a gradient is a view of whatever autograd hands over; the kernels want 16-byte boundaries
            dout = dout.clone()
        dS_final = None if dS_final is None else dS_final.float().contiguous()
        d = scan_backward(ctx.desc, ctx.plan, q, k, v, g, beta, u_bonus, dout, S_init=S_init, dS_final=dS_final, workspace=ws, saved=True)
        return None, None, d.q, d.k, d.v, d.g, d.beta, d.u_bonus, None if S_init is None else d.S_init


def scan(desc: Desc, plan: Plan, q, k, v, g=None, beta=None, u_bonus=None, S_init=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """The differentiable scan: ``(out, S_final)`` of the plan's rows with gradients for every tensor argument; ``out`` rows
    behind the last sequence are zero.  The plan's tables belong to the graph until its backward pass has run: rebuilding
    the plan in between is an error (a build that a replayed graph makes changes the tables just the same, but is not
    noticed), and so is capturing a scan while an eager graph of the same leaves lives.  Forward-mode
    differentiation is refused."""
    _Tokens(desc, plan, q, k, v, g, beta, u_bonus)
    if any(isinstance(t, torch.Tensor) and forward_ad.unpack_dual(t).tangent is not None for t in (q, k, v, g, beta, u_bonus, S_init)):
        # (a dual tensor need not require a gradient, and the kernels would read its value alone: a derivative of zero)
        raise RuntimeError("scan has no forward-mode derivative: an argument carries a tangent")
    _gpu(plan.device)
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (q, k, v, g, beta, u_bonus, S_init)):
        return _Scan.apply(desc, plan, q, k, v, g, beta, u_bonus, S_init)
    return scan_forward(desc, plan, q, k, v, g, beta, u_bonus, S_init=S_init)
