"""Python binding of ``include/lbi_block.h``, the operators of a state-space region block
(argument marshalling only, like ``binding``).

Every function has the name of the C entry point it calls.  Token tensors are [T, D], or
[B, L, D] for B sequences of L tokens; rows may lie at any stride (halves and slices of a
projection's output are taken as they are), the values of a row side by side.  Without
``offsets`` a [T, D] tensor holds ``sequences`` sequences of the same length.  Outputs and the
workspace are allocated unless they are given.

``stream`` (a torch stream or a handle): where the call runs instead of the current stream.  What the
call allocates is that stream's own.  Waiting is left to the caller, in both directions, and so is
keeping the inputs and the given tensors alive until the call is done.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from . import binding
from .binding import _DTYPES, _check, _stream_ptr

LBI_Q8_E4M3 = 0
LBI_Q8_INT8 = 1
LBI_NORM_MAX_D = 16384
LBI_SSM_MAX_D = 65536
LBI_SSM_MAX_N = 64
LBI_CONV_MAX_W = 4

_Q8_TYPES = {LBI_Q8_E4M3: torch.float8_e4m3fn, LBI_Q8_INT8: torch.int8}


class SsmInputs(ctypes.Structure):
    """lbi_ssm_inputs."""

    _fields_ = [(n, t) for names, t in (
        (("u",), ctypes.c_void_p), (("ld_u",), ctypes.c_int64),
        (("delta",), ctypes.c_void_p), (("ld_delta",), ctypes.c_int64),
        (("z",), ctypes.c_void_p), (("ld_z",), ctypes.c_int64),
        (("B",), ctypes.c_void_p), (("ld_B",), ctypes.c_int64),
        (("C",), ctypes.c_void_p), (("ld_C",), ctypes.c_int64),
        (("A", "skip", "delta_bias", "state_in", "offsets"), ctypes.c_void_p),
        (("T", "sequences"), ctypes.c_int64),
        (("D", "N", "G", "softplus"), ctypes.c_int32),
        (("dt",), ctypes.c_int)) for n in names]


class SsmGradients(ctypes.Structure):
    """lbi_ssm_gradients."""

    _fields_ = [(n, t) for names, t in (
        (("du",), ctypes.c_void_p), (("ld_du",), ctypes.c_int64),
        (("ddelta",), ctypes.c_void_p), (("ld_ddelta",), ctypes.c_int64),
        (("dz",), ctypes.c_void_p), (("ld_dz",), ctypes.c_int64),
        (("dB",), ctypes.c_void_p), (("ld_dB",), ctypes.c_int64),
        (("dC",), ctypes.c_void_p), (("ld_dC",), ctypes.c_int64),
        (("dA", "dskip", "ddelta_bias", "dstate_in"), ctypes.c_void_p)) for n in names]


_lib = None


def load() -> ctypes.CDLL:
    """The HIP library with these entry points declared (raises RuntimeError when not built)."""
    global _lib
    if _lib is not None:
        return _lib
    lib = binding.load()
    vp, i64, i32, sz, f32 = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t,
                             ctypes.c_float)
    en = ctypes.c_int
    inputs, grads = ctypes.POINTER(SsmInputs), ctypes.POINTER(SsmGradients)
    for name, args, res in (
            ("lbi_rms_norm", [vp, i64, vp, i64, vp, vp, i64, vp, i64, i64, i32, f32, en, en, vp],
             en),
            ("lbi_rms_norm_q8", [vp, i64, vp, i64, vp, vp, i64, vp, vp, i64, i64, i32, f32, i32,
                                 en, en, en, vp], en),
            ("lbi_rms_norm_backward_workspace_bytes", [i64, i32], sz),
            ("lbi_rms_norm_backward", [vp, i64, vp, i64, vp, vp, i64, vp, i64, vp, i64, i32, f32,
                                       en, en, vp, sz, vp], en),
            ("lbi_ssm_conv", [vp, i64, vp, vp, vp, i64, vp, vp, vp, i32, vp, i64, i64, i32, i32,
                              i32, en, vp], en),
            ("lbi_ssm_conv_backward_workspace_bytes", [i64, i32, i32], sz),
            ("lbi_ssm_conv_backward", [vp, i64, vp, vp, vp, i64, vp, vp, vp, i64, vp, vp, vp, vp,
                                       i64, i64, i32, i32, i32, en, vp, sz, vp], en),
            ("lbi_ssm_conv_step", [vp, i64, vp, vp, vp, i64, vp, vp, vp, i32, i64, i32, i32, i32,
                                   en, vp], en),
            ("lbi_ssm_scan_workspace_bytes", [i64, i64, i32, i32, i32, i32], sz),
            ("lbi_ssm_scan", [inputs, vp, i64, vp, vp, i32, vp, sz, vp], en),
            ("lbi_ssm_scan_backward_workspace_bytes", [i64, i64, i32, i32, i32, i32], sz),
            ("lbi_ssm_scan_backward", [inputs, vp, i64, vp, grads, vp, sz, vp], en),
            ("lbi_ssm_scan_step", [inputs, vp, i64, vp, vp, i32, vp], en)):
        fn = getattr(lib, name)
        fn.argtypes, fn.restype = args, res
    _lib = lib
    return lib


# The checks below are what a small call spends most of its host time on: they compare with `is`
# and by device index, and take shapes and strides once.

def _int32(name: str, value: int) -> int:
    """The library takes it in 32 bits, and a larger one would be cut to them."""
    if not -(1 << 31) <= value < 1 << 31:
        raise ValueError(f"{name} is out of range: {value}")
    return value


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _rows(name: str, t: torch.Tensor, shape, dtype, dev: int) -> int:
    """Checks a token tensor and returns its row stride."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != dev:
        raise ValueError(f"{name} must be a {dtype} {tuple(shape)} tensor on cuda:{dev}, got "
                         f"{t.dtype} {tuple(t.shape)} on {t.device}")
    return _row_stride(name, shape, t.stride())


def _row_stride(name: str, shape, stride) -> int:
    """The stride between the rows of all tokens."""
    if stride[-1] != 1 and shape[-1] > 1:
        raise ValueError(f"{name}: the values of a row must lie side by side")
    if len(shape) == 2:
        return stride[0] if shape[0] > 1 else shape[1]
    if shape[1] > 1:
        if shape[0] > 1 and stride[0] != shape[1] * stride[1]:
            raise ValueError(f"{name}: the rows of all sequences must lie at one stride")
        return stride[1]
    return stride[0] if shape[0] > 1 else shape[2]


def _vector(name: str, t: Optional[torch.Tensor], shape, dev: int, dtype=torch.float32):
    """Checks a dense tensor (None passes) and returns its pointer."""
    if t is None:
        return None
    if t.shape != shape or t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} {tuple(shape)} tensor on "
                         f"cuda:{dev}")
    return t.data_ptr()


def _tokens(name: str, x: torch.Tensor):
    """(shape, tokens, dtype, device index, row stride) of the token tensor that leads a call."""
    shape, dtype = x.shape, x.dtype
    if dtype not in _DTYPES:
        raise TypeError(f"{name} must be float32 or bfloat16, got {dtype}")
    if len(shape) not in (2, 3) or not x.is_cuda:
        raise ValueError(f"{name} must be a [T, D] or [B, L, D] GPU tensor")
    T = shape[0] if len(shape) == 2 else shape[0] * shape[1]
    _int32(f"{name}'s row", shape[-1])
    return shape, T, dtype, x.get_device(), _row_stride(name, shape, x.stride())


def _batch(shape, offsets, sequences, dev: int) -> int:
    """The number of packed sequences."""
    if offsets is not None:
        if len(shape) != 2:
            raise ValueError("offsets go with packed [T, D] tensors")
        n = offsets.numel() - 1
        if n < 0:
            raise ValueError("offsets must hold at least one value")
        _vector("offsets", offsets, (n + 1,), dev, torch.int64)
    else:
        n = shape[0] if len(shape) == 3 else (1 if sequences is None else int(sequences))
        if n >> 62 not in (0, -1):
            raise ValueError(f"sequences is out of range: {n}")
    if sequences is not None and int(sequences) != n:
        raise ValueError(f"sequences is {sequences}, the tensors hold {n}")
    return n


def _states(state_in, state_out, slots, n: int, tail, dtype, dev: int, names=("state_in",
                                                                            "state_out")):
    """Checks the states ([n or the slots' rows, *tail], None passes) and the slots; returns
    (state_in pointer, state_out pointer, slots pointer, rows)."""
    rows, ptrs = n, []
    if slots is not None:
        some = state_in if state_in is not None else state_out
        rows = 0 if some is None else _int32("the states' rows", some.shape[0])
    for name, t in zip(names, (state_in, state_out)):
        ptrs.append(_vector(name, t, (rows, *tail), dev, dtype))
    if slots is None:
        return ptrs[0], ptrs[1], None, 0
    return ptrs[0], ptrs[1], _vector("slots", slots, (n,), dev, torch.int32), rows


def _scratch(need: int, workspace, dev: int):
    """(the workspace, its pointer and bytes), allocated when needed and not given."""
    if workspace is None:
        if need == 0:
            return None, None, 0
        workspace = torch.empty((need,), dtype=torch.uint8, device=f"cuda:{dev}")
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError(f"workspace must be a contiguous tensor on cuda:{dev}")
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(dev: int) -> int:
    """The current stream of the device, as the library takes it."""
    if _raw_stream is not None:
        return _raw_stream(dev)
    return _stream_ptr(None, torch.device("cuda", dev))


_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _run(dev: int, entry, *args):
    """Calls an entry point with the tensors' device current: the default stream's handle is the same
    for every device."""
    if _current_device() == dev:
        _check(entry(*args))
    else:
        with torch.cuda.device(dev):
            _check(entry(*args))


def _aside(call, stream, x, *args, **outputs):
    """The call on ``stream``, made the current one: what the call allocates then comes from that
    stream's memory, in its order.  Results are recorded on the caller's stream, where they may be
    used (behind a wait) and dropped."""
    if not x.is_cuda:
        return call(x, *args, **outputs)  # which refuses it
    if not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(int(stream), device=x.device) if int(stream) \
            else torch.cuda.default_stream(x.device)
    if stream.device != x.device:
        raise ValueError(f"stream belongs to {stream.device}, the tensors to {x.device}")
    here = torch.cuda.current_stream(x.device)
    with torch.cuda.stream(stream):
        results = call(x, *args, **outputs)
    for t in (results.values() if isinstance(results, dict) else
              results if isinstance(results, tuple) else (results,)):
        if t is not None:
            t.record_stream(here)
    return results


# ---- norm --------------------------------------------------------------------

def _norm_inputs(x, weight, residual, residual_out):
    shape, T, dtype, dev, ld_x = _tokens("x", x)
    D = shape[-1]
    w = _vector("weight", weight, (D,), dev)
    if residual is None:
        if residual_out is not None:
            raise ValueError("residual_out goes with a residual")
        return shape, D, T, dtype, dev, ld_x, w, 0, 0, _DTYPES[dtype], None
    rt = residual.dtype
    if rt not in _DTYPES:
        raise TypeError(f"residual must be float32 or bfloat16, got {rt}")
    ld_r = _rows("residual", residual, shape, rt, dev)
    if residual_out is None:
        residual_out = x.new_empty(shape, dtype=rt)
    ld_o = _rows("residual_out", residual_out, shape, rt, dev)
    return shape, D, T, dtype, dev, ld_x, w, ld_r, ld_o, _DTYPES[rt], residual_out


def lbi_rms_norm(x: torch.Tensor, weight: torch.Tensor, residual: Optional[torch.Tensor] = None,
                 eps: float = 1e-5, out: Optional[torch.Tensor] = None,
                 residual_out: Optional[torch.Tensor] = None, stream=None):
    """(out, residual_out): the root-mean-square norm of s = x + residual, and s (None without a
    residual).  residual_out may be residual itself."""
    if stream is not None:
        return _aside(lbi_rms_norm, stream, x, weight, residual, eps, out=out,
                      residual_out=residual_out)
    shape, D, T, dtype, dev, ld_x, w, ld_r, ld_o, rdt, residual_out = _norm_inputs(
        x, weight, residual, residual_out)
    if out is None:
        out = x.new_empty(shape)
    _run(dev, load().lbi_rms_norm,
         x.data_ptr(), ld_x, _ptr(residual), ld_r, w, out.data_ptr(),
         _rows("out", out, shape, dtype, dev), _ptr(residual_out), ld_o, T, D, eps,
         _DTYPES[dtype], rdt, _stream(dev))
    return out, residual_out


def lbi_rms_norm_q8(x: torch.Tensor, weight: torch.Tensor,
                    residual: Optional[torch.Tensor] = None, eps: float = 1e-5,
                    format: int = LBI_Q8_E4M3, group: int = 0, q: Optional[torch.Tensor] = None,
                    scales: Optional[torch.Tensor] = None,
                    residual_out: Optional[torch.Tensor] = None, stream=None):
    """(q, scales, residual_out): the norm's output in 8 bits, q * scale, with one float32 scale
    for each ``group`` features of a token (0: for the token)."""
    if stream is not None:
        return _aside(lbi_rms_norm_q8, stream, x, weight, residual, eps, format, group, q=q,
                      scales=scales, residual_out=residual_out)
    shape, D, T, dtype, dev, ld_x, w, ld_r, ld_o, rdt, residual_out = _norm_inputs(
        x, weight, residual, residual_out)
    if format not in _Q8_TYPES:
        raise ValueError(f"format must be LBI_Q8_E4M3 or LBI_Q8_INT8, got {format}")
    groups = (*shape[:-1], -(-D // group) if _int32("group", group) > 0 else 1)
    if q is None:
        q = x.new_empty(shape, dtype=_Q8_TYPES[format])
    if scales is None:
        scales = x.new_empty(groups, dtype=torch.float32)
    _run(dev, load().lbi_rms_norm_q8,
         x.data_ptr(), ld_x, _ptr(residual), ld_r, w, q.data_ptr(),
         _rows("q", q, shape, _Q8_TYPES[format], dev), _vector("scales", scales, groups, dev),
         _ptr(residual_out), ld_o, T, D, eps, group, format, _DTYPES[dtype], rdt,
         _stream(dev))
    return q, scales, residual_out


def lbi_rms_norm_backward_workspace_bytes(T: int, D: int) -> int:
    return int(load().lbi_rms_norm_backward_workspace_bytes(int(T), int(D)))


def lbi_rms_norm_backward(dout: torch.Tensor, s: torch.Tensor, weight: torch.Tensor,
                          dresidual: Optional[torch.Tensor] = None, eps: float = 1e-5,
                          ds: Optional[torch.Tensor] = None,
                          dweight: Optional[torch.Tensor] = None,
                          workspace: Optional[torch.Tensor] = None, stream=None):
    """(ds, dweight): the gradient of what was normalised (of x and of residual alike), with
    ``dresidual`` added, and of the weight.  ds may be dresidual itself."""
    if stream is not None:
        return _aside(lbi_rms_norm_backward, stream, dout, s, weight, dresidual, eps, ds=ds,
                      dweight=dweight, workspace=workspace)
    shape, T, dtype, dev, ld_dout = _tokens("dout", dout)
    D, st = shape[-1], s.dtype
    if st not in _DTYPES:
        raise TypeError(f"s must be float32 or bfloat16, got {st}")
    ld_s = _rows("s", s, shape, st, dev)
    ld_r = 0 if dresidual is None else _rows("dresidual", dresidual, shape, st, dev)
    w = _vector("weight", weight, (D,), dev)
    if ds is None:
        ds = s.new_empty(shape)
    if dweight is None:
        dweight = weight.new_empty((D,))
    workspace, ws, wb = _scratch(load().lbi_rms_norm_backward_workspace_bytes(T, D), workspace, dev)
    _run(dev, load().lbi_rms_norm_backward,
         dout.data_ptr(), ld_dout, s.data_ptr(), ld_s, w, _ptr(dresidual), ld_r, ds.data_ptr(),
         _rows("ds", ds, shape, st, dev), _vector("dweight", dweight, (D,), dev), T, D, eps,
         _DTYPES[dtype], _DTYPES[st], ws, wb, _stream(dev))
    return ds, dweight


# ---- convolution -------------------------------------------------------------

def _conv_inputs(x, weight, bias):
    shape, T, dtype, dev, ld_x = _tokens("x", x)
    D = shape[-1]
    if weight.dim() != 2:
        raise ValueError("weight must be [D, W]")
    W = _int32("W", weight.shape[1])
    return (shape, D, T, dtype, dev, ld_x, W, _vector("weight", weight, (D, W), dev),
            _vector("bias", bias, (D,), dev))


def lbi_ssm_conv(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None,
                 silu: bool = True, offsets: Optional[torch.Tensor] = None,
                 sequences: Optional[int] = None, state_in: Optional[torch.Tensor] = None,
                 state_out: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None,
                 out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """The causal convolution of every channel with its W = 2 .. 4 taps weight [D, W] along the
    tokens of each sequence.  state_in, state_out [B, W - 1, D]: the tokens before each sequence
    and the last ones after it."""
    if stream is not None:
        return _aside(lbi_ssm_conv, stream, x, weight, bias, silu, offsets, sequences, state_in,
                      state_out=state_out, slots=slots, out=out)
    shape, D, T, dtype, dev, ld_x, W, w, b = _conv_inputs(x, weight, bias)
    n = _batch(shape, offsets, sequences, dev)
    si, so, sp, ns = _states(state_in, state_out, slots, n, (W - 1, D), dtype, dev)
    if out is None:
        out = x.new_empty(shape)
    _run(dev, load().lbi_ssm_conv,
         x.data_ptr(), ld_x, w, b, out.data_ptr(), _rows("out", out, shape, dtype, dev), si, so, sp,
         ns, _ptr(offsets), T, n, D, W, int(silu), _DTYPES[dtype], _stream(dev))
    return out


def lbi_ssm_conv_backward_workspace_bytes(T: int, D: int, W: int) -> int:
    return int(load().lbi_ssm_conv_backward_workspace_bytes(int(T), int(D), int(W)))


def lbi_ssm_conv_backward(x: torch.Tensor, weight: torch.Tensor, dout: torch.Tensor,
                          bias: Optional[torch.Tensor] = None, silu: bool = True,
                          offsets: Optional[torch.Tensor] = None,
                          sequences: Optional[int] = None,
                          state_in: Optional[torch.Tensor] = None,
                          dstate_out: Optional[torch.Tensor] = None,
                          dx: Optional[torch.Tensor] = None,
                          workspace: Optional[torch.Tensor] = None, stream=None):
    """(dx, dweight, dbias, dstate_in): dbias None without a bias, dstate_in None without
    state_in."""
    if stream is not None:
        return _aside(lbi_ssm_conv_backward, stream, x, weight, dout, bias, silu, offsets, sequences,
                      state_in, dstate_out, dx=dx, workspace=workspace)
    shape, D, T, dtype, dev, ld_x, W, w, b = _conv_inputs(x, weight, bias)
    n = _batch(shape, offsets, sequences, dev)
    si, so, _, _ = _states(state_in, dstate_out, None, n, (W - 1, D), dtype, dev,
                           ("state_in", "dstate_out"))
    ld_dout = _rows("dout", dout, shape, dtype, dev)
    if dx is None:
        dx = x.new_empty(shape)
    dweight = weight.new_empty((D, W))
    dbias = None if bias is None else bias.new_empty((D,))
    dstate_in = None if state_in is None else torch.empty_like(state_in)
    workspace, ws, wb = _scratch(load().lbi_ssm_conv_backward_workspace_bytes(T, D, W), workspace,
                                 dev)
    _run(dev, load().lbi_ssm_conv_backward,
         x.data_ptr(), ld_x, w, b, dout.data_ptr(), ld_dout, si, so, dx.data_ptr(),
         _rows("dx", dx, shape, dtype, dev), dweight.data_ptr(), _ptr(dbias), _ptr(dstate_in),
         _ptr(offsets), T, n, D, W, int(silu), _DTYPES[dtype], ws, wb, _stream(dev))
    return dx, dweight, dbias, dstate_in


def lbi_ssm_conv_step(x: torch.Tensor, weight: torch.Tensor, state_in: torch.Tensor,
                      state_out: torch.Tensor, bias: Optional[torch.Tensor] = None,
                      silu: bool = True, slots: Optional[torch.Tensor] = None,
                      out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """One token for each of n sequences, x [n, D]; state_out may be state_in."""
    if stream is not None:
        return _aside(lbi_ssm_conv_step, stream, x, weight, state_in, state_out, bias, silu, slots,
                      out=out)
    shape, D, n, dtype, dev, ld_x, W, w, b = _conv_inputs(x, weight, bias)
    if len(shape) != 2:
        raise ValueError("x must be [n, D]")
    si, so, sp, ns = _states(state_in, state_out, slots, n, (W - 1, D), dtype, dev)
    if out is None:
        out = x.new_empty(shape)
    _run(dev, load().lbi_ssm_conv_step,
         x.data_ptr(), ld_x, w, b, out.data_ptr(), _rows("out", out, shape, dtype, dev), si, so, sp,
         ns, n, D, W, int(silu), _DTYPES[dtype], _stream(dev))
    return out


# ---- scan --------------------------------------------------------------------

def _groups(name, t, lead, N: int, dtype, dev: int):
    """(row stride, groups) of B or C: [..., N] or [..., G, N]."""
    shape, stride, k = t.shape, t.stride(), len(lead)
    if (t.dtype is not dtype or t.get_device() != dev or shape[:k] != lead
            or len(shape) - k not in (1, 2) or shape[-1] != N):
        raise ValueError(f"{name} must be a {dtype} {(*lead, 'G', N)} or {(*lead, N)} tensor on "
                         f"cuda:{dev}")
    G = shape[k] if len(shape) > k + 1 else 1
    if (N > 1 and stride[-1] != 1) or (G > 1 and stride[-2] != N):
        raise ValueError(f"{name}: a token's values must lie side by side")
    return _row_stride(name, (*lead, G * N), (*stride[:k], 1)), _int32("G", G)


def _scan_inputs(u, delta, A, B, C, skip, z, delta_bias, softplus, offsets, sequences, state_in):
    """(the struct, shape, dtype, device index); state_in: its pointer."""
    shape, T, dtype, dev, ld_u = _tokens("u", u)
    D, lead = shape[-1], shape[:-1]
    if A.dim() != 2:
        raise ValueError("A must be [D, N]")
    N = _int32("N", A.shape[1])
    ld_B, G = _groups("B", B, lead, N, dtype, dev)
    ld_C, G2 = _groups("C", C, lead, N, dtype, dev)
    if G != G2:
        raise ValueError("B and C must have the same groups")
    n = _batch(shape, offsets, sequences, dev)
    return SsmInputs(
        u.data_ptr(), ld_u, delta.data_ptr(), _rows("delta", delta, shape, dtype, dev), _ptr(z),
        0 if z is None else _rows("z", z, shape, dtype, dev), B.data_ptr(), ld_B, C.data_ptr(),
        ld_C, _vector("A", A, (D, N), dev), _vector("skip", skip, (D,), dev),
        _vector("delta_bias", delta_bias, (D,), dev), state_in, _ptr(offsets), T, n, D, N, G,
        int(softplus), _DTYPES[dtype]), shape, dtype, dev


def lbi_ssm_scan_workspace_bytes(T: int, sequences: int, D: int, N: int, G: int,
                                 ragged: bool) -> int:
    return int(load().lbi_ssm_scan_workspace_bytes(int(T), int(sequences), int(D), int(N), int(G),
                                                   int(ragged)))


def lbi_ssm_scan(u: torch.Tensor, delta: torch.Tensor, A: torch.Tensor, B: torch.Tensor,
                 C: torch.Tensor, skip: Optional[torch.Tensor] = None,
                 z: Optional[torch.Tensor] = None, delta_bias: Optional[torch.Tensor] = None,
                 softplus: bool = True, offsets: Optional[torch.Tensor] = None,
                 sequences: Optional[int] = None, state_in: Optional[torch.Tensor] = None,
                 state_out: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None,
                 out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                 stream=None) -> torch.Tensor:
    """The selective scan of u under the steps softplus(delta + delta_bias), A [D, N] and the
    tokens' B, C [..., G, N] (or [..., N]), gated by silu(z).  state_in, state_out [B, D, N]
    float32: the states before and after each sequence; they may be the same tensor."""
    if stream is not None:
        return _aside(lbi_ssm_scan, stream, u, delta, A, B, C, skip, z, delta_bias, softplus,
                      offsets, sequences, state_in, state_out=state_out, slots=slots, out=out,
                      workspace=workspace)
    si, shape, dtype, dev = _scan_inputs(u, delta, A, B, C, skip, z, delta_bias, softplus, offsets,
                                         sequences, None)
    si.state_in, so, sp, ns = _states(state_in, state_out, slots, si.sequences, (si.D, si.N),
                                      torch.float32, dev)
    if out is None:
        out = u.new_empty(shape)
    lib = load()
    need = lib.lbi_ssm_scan_workspace_bytes(si.T, si.sequences, si.D, si.N, si.G,
                                            int(offsets is not None))
    workspace, w, wb = _scratch(need, workspace, dev)
    _run(dev, lib.lbi_ssm_scan,
         ctypes.byref(si), out.data_ptr(), _rows("out", out, shape, dtype, dev), so, sp, ns, w, wb,
         _stream(dev))
    return out


def lbi_ssm_scan_backward_workspace_bytes(T: int, sequences: int, D: int, N: int, G: int,
                                          ragged: bool) -> int:
    return int(load().lbi_ssm_scan_backward_workspace_bytes(int(T), int(sequences), int(D),
                                                            int(N), int(G), int(ragged)))


def lbi_ssm_scan_backward(u: torch.Tensor, delta: torch.Tensor, A: torch.Tensor,
                          B: torch.Tensor, C: torch.Tensor, dout: torch.Tensor,
                          skip: Optional[torch.Tensor] = None, z: Optional[torch.Tensor] = None,
                          delta_bias: Optional[torch.Tensor] = None, softplus: bool = True,
                          offsets: Optional[torch.Tensor] = None,
                          sequences: Optional[int] = None,
                          state_in: Optional[torch.Tensor] = None,
                          dstate_out: Optional[torch.Tensor] = None,
                          outputs: Optional[dict] = None,
                          workspace: Optional[torch.Tensor] = None, stream=None) -> dict:
    """The gradients by input: "u", "delta", "A", "B", "C", "skip", "z", "delta_bias" and
    "state_in", None where the input is.  ``outputs``: tensors to write some of them to."""
    if stream is not None:
        return _aside(lbi_ssm_scan_backward, stream, u, delta, A, B, C, dout, skip, z, delta_bias,
                      softplus, offsets, sequences, state_in, dstate_out, outputs=outputs,
                      workspace=workspace)
    si, shape, dtype, dev = _scan_inputs(u, delta, A, B, C, skip, z, delta_bias, softplus, offsets,
                                         sequences, None)
    si.state_in, so, _, _ = _states(state_in, dstate_out, None, si.sequences, (si.D, si.N),
                                    torch.float32, dev, ("state_in", "dstate_out"))
    ld_dout = _rows("dout", dout, shape, dtype, dev)
    g = {} if outputs is None else dict(outputs)
    of = {"u": u, "delta": delta, "A": A, "B": B, "C": C, "skip": skip, "z": z,
          "delta_bias": delta_bias, "state_in": state_in}
    if not g.keys() <= of.keys():
        raise ValueError(f"outputs go by the inputs' names, got {sorted(g.keys() - of.keys())}")
    for name, t in of.items():
        if t is None:
            if g.get(name) is not None:
                raise ValueError(f"outputs[{name!r}]: there is no such input")
            g[name] = None
        elif g.get(name) is None:
            g[name] = t.new_empty(t.shape)
    ld_B, G = _groups("outputs['B']", g["B"], shape[:-1], si.N, dtype, dev)
    ld_C, G2 = _groups("outputs['C']", g["C"], shape[:-1], si.N, dtype, dev)
    if G != si.G or G2 != si.G:
        raise ValueError(f"outputs['B'] and outputs['C'] must have {si.G} groups")
    sg = SsmGradients(
        g["u"].data_ptr(), _rows("outputs['u']", g["u"], shape, dtype, dev),
        g["delta"].data_ptr(), _rows("outputs['delta']", g["delta"], shape, dtype, dev),
        _ptr(g["z"]), 0 if z is None else _rows("outputs['z']", g["z"], shape, dtype, dev),
        g["B"].data_ptr(), ld_B, g["C"].data_ptr(), ld_C,
        _vector("outputs['A']", g["A"], (si.D, si.N), dev),
        _vector("outputs['skip']", g["skip"], (si.D,), dev),
        _vector("outputs['delta_bias']", g["delta_bias"], (si.D,), dev),
        _vector("outputs['state_in']", g["state_in"], (si.sequences, si.D, si.N), dev))
    lib = load()
    need = lib.lbi_ssm_scan_backward_workspace_bytes(si.T, si.sequences, si.D, si.N, si.G,
                                                     int(offsets is not None))
    workspace, w, wb = _scratch(need, workspace, dev)
    _run(dev, lib.lbi_ssm_scan_backward, ctypes.byref(si), dout.data_ptr(), ld_dout, so,
         ctypes.byref(sg), w, wb, _stream(dev))
    return g


def lbi_ssm_scan_step(u: torch.Tensor, delta: torch.Tensor, A: torch.Tensor, B: torch.Tensor,
                      C: torch.Tensor, state_in: torch.Tensor, state_out: torch.Tensor,
                      skip: Optional[torch.Tensor] = None, z: Optional[torch.Tensor] = None,
                      delta_bias: Optional[torch.Tensor] = None, softplus: bool = True,
                      slots: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                      stream=None) -> torch.Tensor:
    """One token for each of n sequences, u [n, D]; state_out may be state_in."""
    if stream is not None:
        return _aside(lbi_ssm_scan_step, stream, u, delta, A, B, C, state_in, state_out, skip, z,
                      delta_bias, softplus, slots, out=out)
    if u.dim() != 2:
        raise ValueError("u must be [n, D]")
    si, shape, dtype, dev = _scan_inputs(u, delta, A, B, C, skip, z, delta_bias, softplus, None,
                                         u.shape[0], None)
    si.state_in, so, sp, ns = _states(state_in, state_out, slots, si.sequences, (si.D, si.N),
                                      torch.float32, dev)
    if out is None:
        out = u.new_empty(shape)
    _run(dev, load().lbi_ssm_scan_step,
         ctypes.byref(si), out.data_ptr(), _rows("out", out, shape, dtype, dev), so, sp, ns,
         _stream(dev))
    return out
