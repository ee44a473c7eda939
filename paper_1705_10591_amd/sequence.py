"""Operators over the tokens of sequences: the short causal convolution and the selective scan (dconv.h says what they compute).

Token tensors are [N, L, C] (B and C of the scan [N, L, G, S]) with the last dimension contiguous and any strides before
it; a step has no L.  As everywhere in this package, functions check and marshal arguments, enqueue on the current stream
of the tensors' device and return; outputs that are not passed in, and workspaces, come from torch's allocator, which
is safe for streams and captured graphs.  Outputs must not share memory with inputs, but for the states that a call says it may
write over.  Gradients are explicit calls: nothing is recorded for torch.autograd.
"""
from __future__ import annotations

import ctypes
import struct
import sys
from functools import lru_cache
from typing import NamedTuple, Optional

import torch

EXPORTS = ("dconv_causal", "dconv_causal_grad", "dconv_causal_step", "dconv_causal_workspace",
           "dconv_scan", "dconv_scan_grad", "dconv_scan_step", "dconv_scan_workspace", "dconv_scan_starts")
DTYPE_F32 = 3
_DTYPES = {torch.float16: 0, torch.bfloat16: 1, torch.float32: DTYPE_F32}

# The argument structs of dconv.h, packed at once: filling a ctypes structure field by field takes several times as long
# as a single token takes the GPU.  A token tensor is four fields: pointer, strides of sequence, token and group.
_CAUSAL = struct.Struct("8i" + 4 * "4q" + "12q")
_SCAN = struct.Struct("8i" + 12 * "4q" + "15q")
# ... of each form, without the fields that it leaves empty
_CAUSAL_PROMPT = struct.Struct("8i" + 2 * "3q8x" + "64x" + "4q" + "32x" + "q" + "24x")
_CAUSAL_GRAD = struct.Struct("8i" + "3q8x" + "32x" + 2 * "3q8x" + "3q8x" + "4q" + "q8x" + "2q")
_CAUSAL_STEP = struct.Struct("8i" + 2 * "2q16x" + "64x" + "2q8xq40xq16x")
_SCAN_PROMPT = struct.Struct("8i" + 4 * "3q8x" + 2 * "4q" + "192x" + "5q" + "40x" + "2q8x" + "2q")
_SCAN_GRAD = struct.Struct("8i" + 3 * "3q8x" + "32x" + 2 * "4q" + 4 * "3q8x" + 2 * "4q" + "4q8x" + "5q" + "2q8x" + "2q")
_SCAN_STEP = struct.Struct("8i" + 4 * "2q16x" + 2 * "2q8xq" + "192x" + "3q8xq56xq16x")
_NONE, _NONE3 = (0, 0, 0, 0), (0, 0, 0)
_INT32, _FLOAT32 = torch.int32, torch.float32
# (torch.cuda.current_device and a Stream object take as long as all checks of a call)
_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def declare(lib: ctypes.CDLL) -> None:
    for name in EXPORTS:
        fn = getattr(lib, name)
        if name.endswith(("_workspace", "_starts")):
            fn.argtypes = [ctypes.c_char_p] + ([ctypes.c_int] if name == "dconv_scan_workspace" else [])
            fn.restype = ctypes.c_longlong
        else:
            fn.argtypes = [ctypes.c_char_p, ctypes.c_void_p]
            fn.restype = ctypes.c_int


_loaded = _package = _raw_stream = None


def _lib():
    global _loaded, _package, _raw_stream
    if _loaded is None:
        _package = sys.modules[__package__]
        _raw_stream = _package._raw_stream
        _loaded = _package.load_library()
    return _loaded


def _run(fn, index, args):
    if index != _device():
        return _package._enqueue(fn, index, args)
    rc = fn(args, _raw_stream(index))
    if rc:
        _package._raise(rc)


def _beyond():
    """A size that the structs' 32 bits do not hold is one that the library refuses."""
    _lib()
    _package._raise(_package.STATUS_BAD_SHAPE)


# One token of one row takes the GPU 2.4 us and the host two to three times as long, most of it in the checks below: a tensor that
# fits is looked at in one expression, and what does not fit is looked into afterwards.  (Sizes of zero are the library's to refuse.)

def _like(t):
    """A dense tensor of t's shape; a third faster than asking for the shape."""
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _first(t, dims, what):
    """Type, its number, device and shape that the other tensors of a call have to agree with."""
    try:
        dtype, shape = t.dtype, t.shape
        code, index = _DTYPES.get(dtype), t.get_device()
        if code is not None and index >= 0 and len(shape) == dims:
            return dtype, code, index, shape
    except AttributeError:
        pass
    raise TypeError(f"{what} must be a float16, bfloat16 or float32 CUDA tensor with {dims} dims")


def _refuse(t, shape, dtype, index, what):
    """Says what does not fit."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype):
        raise TypeError(f"{what} must be a CUDA tensor of type {dtype}")
    if t.get_device() != index:
        raise ValueError(f"{what} is on another device")
    if t.shape != shape:
        raise ValueError(f"{what} must have the shape {tuple(shape)}, not {tuple(t.shape)}")
    raise TypeError(f"{what} must be contiguous")


def _strides(t, shape, dtype, index, what):
    try:
        if t.dtype is dtype and t.get_device() == index and t.shape == shape:
            s = t.stride()
            if s[-1] == 1 or shape[-1] == 1:
                return s
            raise TypeError(f"the last dimension of {what} must be contiguous")
    except AttributeError:
        pass
    _refuse(t, shape, dtype, index, what)


def _row(t, shape, dtype, index, what):
    """(pointer, stride) of the rows of a step's token tensor."""
    s = _strides(t, shape, dtype, index, what)
    return t.data_ptr(), s[0]


def _rows(t, shape, dtype, index, what):
    """(pointer, strides of sequence and token) of a token tensor."""
    if t is None:
        return _NONE3
    s = _strides(t, shape, dtype, index, what)
    return t.data_ptr(), s[0], s[1]


def _groups(t, shape, dtype, index, what):
    """(pointer, strides of sequence, token and group) of B, C and their gradients."""
    if t is None:
        return _NONE
    s = _strides(t, shape, dtype, index, what)
    return t.data_ptr(), s[0], s[1], s[2]


def _output(t, shape, dtype, index, what):
    """_rows of an output that the caller gives.  Tokens that share memory would be written by several workgroups."""
    s = _strides(t, shape, dtype, index, what)
    span = shape[-1]
    for stride, size in sorted(zip(s[:-1], shape[:-1])):
        if size > 1:
            if stride < span:
                raise ValueError(f"elements of {what} overlap")
            span += stride * (size - 1)
    return (t.data_ptr(), *s[:-1])


def _dense(t, shape, dtype, index, what):
    if t is None:
        return 0
    try:
        if t.dtype is dtype and t.get_device() == index and t.shape == shape and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    _refuse(t, shape, dtype, index, what)


def _cache(t, tail, dtype, index, what, rows, slots):
    """(pointer, rows) of a cache of states that a step updates."""
    if not isinstance(t, torch.Tensor) or t.dim() != 3:
        raise ValueError(f"{what} must have the shape (rows, {', '.join(map(str, tail))})")
    M = t.shape[0]
    p = _dense(t, (M, *tail), dtype, index, what)
    if M == 0 or (slots is None and M < rows):
        raise ValueError(f"{what} has too few rows")
    return p, M


@lru_cache(maxsize=4096)
def _causal_bytes(code, N, L, C, F):
    try:
        args = _CAUSAL.pack(code, N, L, C, F, 0, 0, 0, *(4 * _NONE), *(12 * (0,)))
    except struct.error:
        _beyond()
    return _lib().dconv_causal_workspace(args)


@lru_cache(maxsize=4096)
def _scan_bytes(code, N, L, C, S, G, form):
    """Of the workspace of a prompt ("scan"), a gradient with and without starts ("grad", "starts grad"), of the starts."""
    tokens = (*(3 * _NONE), 16, 0, 0, 0, *(8 * _NONE))               # (a prompt that has an output)
    try:
        args = _SCAN.pack(code, N, L, C, S, G, 0, 0, *tokens, *(10 * (0,)), 16 if form == "starts grad" else 0, 0, 0, 0, 0)
    except struct.error:
        _beyond()
    if form == "starts":
        return _lib().dconv_scan_starts(args)
    return _lib().dconv_scan_workspace(args, 0 if form == "scan" else 1)


def _workspace(bytes_, like):
    """From torch's allocator, in fp32 elements; sizes that are not valid are refused by the call itself."""
    return like.new_empty((max(bytes_, 16) + 3) // 4, dtype=_FLOAT32)


class CausalGrad(NamedTuple):
    """Gradients of dconv_causal: of x (its type), filt and bias (fp32), and of the state where there is one."""
    dx: torch.Tensor
    dfilt: torch.Tensor
    dbias: torch.Tensor
    dstate: Optional[torch.Tensor]


class ScanGrad(NamedTuple):
    """Gradients of dconv_scan: of the token tensors in their type, of A, D, delta_bias and the state in fp32; None for what
    the call was not given."""
    du: torch.Tensor
    ddelta: torch.Tensor
    dA: torch.Tensor
    dB: torch.Tensor
    dC: torch.Tensor
    dD: Optional[torch.Tensor]
    dz: Optional[torch.Tensor]
    ddelta_bias: Optional[torch.Tensor]
    dstate: Optional[torch.Tensor]


def dconv_causal(x: torch.Tensor, filt: torch.Tensor, bias: torch.Tensor | None = None, *, silu: bool = True,
                 state: torch.Tensor | None = None, lengths: torch.Tensor | None = None,
                 out: torch.Tensor | None = None, state_out: torch.Tensor | None = None) -> torch.Tensor:
    """out[n,t,c] = act(bias[c] + sum_j filt[c,j] * x[n, t-(F-1)+j, c]), act = silu or nothing.

    x [N,L,C], filt [C,F] (F <= 8), bias [C], all of one type.  state [N,F-1,C]: the rows before token 0 (default: zeros);
    state_out, which may be `state`, receives the last F-1 rows of each sequence.  lengths [N] int32: the tokens of each
    sequence that count; out is 0 behind them."""
    dtype, code, index, shape = _first(x, 3, "x")
    N, L, C = shape
    F = _taps(filt, C)
    if out is None:
        out = _like(x)
        o = out.data_ptr(), L * C, C
    else:
        o = _output(out, shape, dtype, index, "out")
    rows = (N, F - 1, C)
    try:
        args = _CAUSAL_PROMPT.pack(
            code, N, L, C, F, 0, bool(silu), 0, *_rows(x, shape, dtype, index, "x"), *o,
            _dense(filt, (C, F), dtype, index, "filt"), 0 if bias is None else _dense(bias, (C,), dtype, index, "bias"),
            0 if state is None else _dense(state, rows, dtype, index, "state"),
            0 if state_out is None else _dense(state_out, rows, dtype, index, "state_out"),
            0 if lengths is None else _dense(lengths, (N,), _INT32, index, "lengths"))
    except struct.error:
        _beyond()
    _run(_lib().dconv_causal, index, args)
    return out


def dconv_causal_grad(dout: torch.Tensor, x: torch.Tensor, filt: torch.Tensor, bias: torch.Tensor | None = None, *,
                      silu: bool = True, state: torch.Tensor | None = None, lengths: torch.Tensor | None = None,
                      dstate_out: torch.Tensor | None = None, dx: torch.Tensor | None = None) -> CausalGrad:
    """Gradients of dconv_causal(x, filt, bias, ...) from dout, the gradient of its output, and dstate_out, that of state_out.

    dx may be given (a slice of a wider gradient, say); it is 0 behind `lengths`.  dstate is None without a state."""
    dtype, code, index, shape = _first(x, 3, "x")
    N, L, C = shape
    F = _taps(filt, C)
    rows = (N, F - 1, C)
    if dx is None:
        dx = _like(x)
        d = dx.data_ptr(), L * C, C
    else:
        d = _output(dx, shape, dtype, index, "dx")
    dfilt, dbias = torch.empty_like(filt, dtype=_FLOAT32), x.new_empty((C,), dtype=_FLOAT32)
    dstate = None if state is None else _like(state)
    need = _causal_bytes(code, N, L, C, F)
    ws = _workspace(need, x)
    try:
        args = _CAUSAL_GRAD.pack(
            code, N, L, C, F, 0, bool(silu), 0, *_rows(x, shape, dtype, index, "x"), *_rows(dout, shape, dtype, index, "dout"), *d,
            _dense(filt, (C, F), dtype, index, "filt"), _dense(bias, (C,), dtype, index, "bias"),
            _dense(state, rows, dtype, index, "state"), _dense(dstate_out, rows, dtype, index, "dstate_out"),
            0 if dstate is None else dstate.data_ptr(), dfilt.data_ptr(), dbias.data_ptr(),
            _dense(lengths, (N,), _INT32, index, "lengths"), ws.data_ptr(), need)
    except struct.error:
        _beyond()
    _run(_lib().dconv_causal_grad, index, args)
    return CausalGrad(dx, dfilt, dbias, dstate)


def dconv_causal_step(x: torch.Tensor, state: torch.Tensor, filt: torch.Tensor, bias: torch.Tensor | None = None, *,
                      silu: bool = True, slots: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """One token x [N,C] of each row: out [N,C], and the windows of `state` [M,F-1,C] move on by it.

    slots [N] int32: the window of each row (default: row n has window n); rows with a slot outside the cache, or
    one that an earlier row has, are padding: out is 0 there and no window changes."""
    dtype, code, index, shape = _first(x, 2, "x")
    N, C = shape
    F = _taps(filt, C)
    if out is None:
        out = _like(x)
        o = out.data_ptr(), C
    else:
        o = _output(out, shape, dtype, index, "out")
    cache, M = _cache(state, (F - 1, C), dtype, index, "state", N, slots)
    try:
        args = _CAUSAL_STEP.pack(
            code, N, 1, C, F, M, bool(silu), 0, *_row(x, shape, dtype, index, "x"), *o,
            _dense(filt, (C, F), dtype, index, "filt"), 0 if bias is None else _dense(bias, (C,), dtype, index, "bias"), cache,
            0 if slots is None else _dense(slots, (N,), _INT32, index, "slots"))
    except struct.error:
        _beyond()
    _run(_lib().dconv_causal_step, index, args)
    return out


def _taps(filt, C):
    try:
        c, F = filt.shape
        if c == C:
            return F
    except (AttributeError, ValueError):
        pass
    raise ValueError(f"filt must have the shape ({C}, F)")


def _scan_sizes(u, A, B, dims):
    dtype, code, index, shape = _first(u, dims, "u")
    if not isinstance(A, torch.Tensor) or A.dim() != 2 or A.shape[0] != shape[-1]:
        raise ValueError("A must have the shape (C, S)")
    if not isinstance(B, torch.Tensor) or B.dim() != dims + 1:
        raise ValueError(f"B must have {dims + 1} dims")
    return dtype, code, index, shape, A.shape[1], B.shape[-2]


def scan_starts(N: int, L: int, C: int, S: int, G: int = 1, device="cuda") -> torch.Tensor:
    """An empty tensor for the `starts` of dconv_scan and dconv_scan_grad on sequences of these sizes."""
    need = _scan_bytes(DTYPE_F32, N, L, C, S, G, "starts")
    if need < 0:
        _package._raise(_package.STATUS_BAD_SHAPE)
    return torch.empty(need // 4, dtype=torch.float32, device=device)


def _starts(starts, N, L, C, S, G, index):
    if starts is None:
        return 0
    need = _scan_bytes(DTYPE_F32, N, L, C, S, G, "starts")
    return _dense(starts, (max(need, 0) // 4,), torch.float32, index, "starts")


def dconv_scan(u: torch.Tensor, delta: torch.Tensor, A: torch.Tensor, B: torch.Tensor, C: torch.Tensor,
               D: torch.Tensor | None = None, z: torch.Tensor | None = None, delta_bias: torch.Tensor | None = None, *,
               softplus: bool = True, state: torch.Tensor | None = None, lengths: torch.Tensor | None = None,
               out: torch.Tensor | None = None, state_out: torch.Tensor | None = None,
               starts: torch.Tensor | None = None) -> torch.Tensor:
    """The selective scan: with d = softplus(delta + delta_bias) (without softplus: delta + delta_bias),
    h[t] = exp(d[t] A) h[t-1] + d[t] u[t] B[t],  y[t] = sum_s C[t] h[t] + D u[t],  out = y silu(z) or y.

    u, delta, z [N,L,C]; B, C [N,L,G,S], group g for channels g*C/G onwards; one type for all of these.  A [C,S] (S <= 32),
    D and delta_bias [C], fp32.  state [N,C,S] fp32: h before token 0 (default: zeros); state_out, which may be `state`,
    receives h behind the last token.  lengths [N] int32: the tokens that count; out is 0 behind them.
    starts (of scan_starts): receives what lets dconv_scan_grad go back without running the scan again."""
    dtype, code, index, wide, S, G = _scan_sizes(u, A, B, 3)
    N, L, ch = wide
    narrow = (N, L, G, S)
    if out is None:
        out = _like(u)
        o = out.data_ptr(), L * ch, ch
    else:
        o = _output(out, wide, dtype, index, "out")
    need = _scan_bytes(code, N, L, ch, S, G, "scan")
    ws = _workspace(need, u) if need else None
    try:
        args = _SCAN_PROMPT.pack(
            code, N, L, ch, S, G, 0, bool(softplus), *_rows(u, wide, dtype, index, "u"), *_rows(delta, wide, dtype, index, "delta"),
            *_rows(z, wide, dtype, index, "z"), *o, *_groups(B, narrow, dtype, index, "B"), *_groups(C, narrow, dtype, index, "C"),
            _dense(A, (ch, S), _FLOAT32, index, "A"), _dense(D, (ch,), _FLOAT32, index, "D"),
            _dense(delta_bias, (ch,), _FLOAT32, index, "delta_bias"),
            0 if state is None else _dense(state, (N, ch, S), _FLOAT32, index, "state"),
            0 if state_out is None else _dense(state_out, (N, ch, S), _FLOAT32, index, "state_out"),
            0 if starts is None else _starts(starts, N, L, ch, S, G, index),
            0 if lengths is None else _dense(lengths, (N,), _INT32, index, "lengths"), 0 if ws is None else ws.data_ptr(), need)
    except struct.error:
        _beyond()
    _run(_lib().dconv_scan, index, args)
    return out


def dconv_scan_grad(dout: torch.Tensor, u: torch.Tensor, delta: torch.Tensor, A: torch.Tensor, B: torch.Tensor,
                    C: torch.Tensor, D: torch.Tensor | None = None, z: torch.Tensor | None = None,
                    delta_bias: torch.Tensor | None = None, *, softplus: bool = True, state: torch.Tensor | None = None,
                    lengths: torch.Tensor | None = None, starts: torch.Tensor | None = None,
                    dstate_out: torch.Tensor | None = None, du: torch.Tensor | None = None,
                    ddelta: torch.Tensor | None = None, dz: torch.Tensor | None = None) -> ScanGrad:
    """Gradients of dconv_scan(u, ...) from dout, the gradient of its output, and dstate_out, that of state_out.

    starts: what dconv_scan left there for the same inputs; without it the states are made again.  du, ddelta and dz may be
    given (slices of a wider gradient, say); gradients are 0 behind `lengths`."""
    dtype, code, index, wide, S, G = _scan_sizes(u, A, B, 3)
    N, L, ch = wide
    narrow = (N, L, G, S)

    def wide_out(t, what):
        if t is not None:
            return t, _output(t, wide, dtype, index, what)
        t = _like(u)
        return t, (t.data_ptr(), L * ch, ch)

    du, du_ = wide_out(du, "du")
    ddelta, ddelta_ = wide_out(ddelta, "ddelta")
    dz, dz_ = (None, _NONE3) if z is None else wide_out(dz, "dz")
    dB, dC, dA = _like(B), _like(B), _like(A)
    dD = None if D is None else _like(D)
    dbias = None if delta_bias is None else _like(delta_bias)
    dstate = None if state is None else _like(state)
    need = _scan_bytes(code, N, L, ch, S, G, "grad" if starts is None else "starts grad")
    ws = _workspace(need, u)
    try:
        args = _SCAN_GRAD.pack(
            code, N, L, ch, S, G, 0, bool(softplus), *_rows(u, wide, dtype, index, "u"), *_rows(delta, wide, dtype, index, "delta"),
            *_rows(z, wide, dtype, index, "z"), *_groups(B, narrow, dtype, index, "B"), *_groups(C, narrow, dtype, index, "C"),
            *_rows(dout, wide, dtype, index, "dout"), *du_, *ddelta_, *dz_,
            dB.data_ptr(), L * G * S, G * S, S, dC.data_ptr(), L * G * S, G * S, S,
            _dense(A, (ch, S), _FLOAT32, index, "A"), _dense(D, (ch,), _FLOAT32, index, "D"),
            _dense(delta_bias, (ch,), _FLOAT32, index, "delta_bias"), _dense(state, (N, ch, S), _FLOAT32, index, "state"),
            _dense(dstate_out, (N, ch, S), _FLOAT32, index, "dstate_out"), 0 if dstate is None else dstate.data_ptr(),
            dA.data_ptr(), 0 if dD is None else dD.data_ptr(), 0 if dbias is None else dbias.data_ptr(),
            0 if starts is None else _starts(starts, N, L, ch, S, G, index), _dense(lengths, (N,), _INT32, index, "lengths"),
            ws.data_ptr(), need)
    except struct.error:
        _beyond()
    _run(_lib().dconv_scan_grad, index, args)
    return ScanGrad(du, ddelta, dA, dB, dC, dD, dz, dbias, dstate)


def dconv_scan_step(u: torch.Tensor, delta: torch.Tensor, A: torch.Tensor, B: torch.Tensor, C: torch.Tensor,
                    state: torch.Tensor, D: torch.Tensor | None = None, z: torch.Tensor | None = None,
                    delta_bias: torch.Tensor | None = None, *, softplus: bool = True, slots: torch.Tensor | None = None,
                    out: torch.Tensor | None = None) -> torch.Tensor:
    """One token of each row: u, delta, z [N,C], B, C [N,G,S]; out [N,C], and `state` [M,C,S] (fp32) is updated.

    slots as for dconv_causal_step."""
    dtype, code, index, wide, S, G = _scan_sizes(u, A, B, 2)
    N, ch = wide
    narrow = (N, G, S)
    if out is None:
        out = _like(u)
        o = out.data_ptr(), ch
    else:
        o = _output(out, wide, dtype, index, "out")
    cache, M = _cache(state, (ch, S), _FLOAT32, index, "state", N, slots)
    try:
        args = _SCAN_STEP.pack(
            code, N, 1, ch, S, G, M, bool(softplus), *_row(u, wide, dtype, index, "u"), *_row(delta, wide, dtype, index, "delta"),
            *((0, 0) if z is None else _row(z, wide, dtype, index, "z")), *o,
            *_rows(B, narrow, dtype, index, "B"), *_rows(C, narrow, dtype, index, "C"),          # (sequence and group)
            _dense(A, (ch, S), _FLOAT32, index, "A"), _dense(D, (ch,), _FLOAT32, index, "D"),
            _dense(delta_bias, (ch,), _FLOAT32, index, "delta_bias"), cache,
            0 if slots is None else _dense(slots, (N,), _INT32, index, "slots"))
    except struct.error:
        _beyond()
    _run(_lib().dconv_scan_step, index, args)
    return out
