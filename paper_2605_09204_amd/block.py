"""Python binding of ``include/lbi_block.h``, the operators of a state-space region block
(argument marshalling only, like ``binding``).

Every function has the name of the C entry point it calls.  Token tensors are [T, D], or
[B, L, D] for B sequences of L tokens; rows may lie at any stride (halves and slices of a
projection's output are taken as they are), the values of a row side by side.  Without
``offsets`` a [T, D] tensor holds ``sequences`` sequences of the same length.  Outputs and the
workspace are allocated unless they are given.
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


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _rows(name: str, t: torch.Tensor, lead, cols: int, dtype, device) -> int:
    """Checks a token tensor of shape lead + (cols,) and returns its row stride."""
    if t.dtype != dtype or t.device != device or tuple(t.shape) != (*lead, cols):
        raise ValueError(f"{name} must be a {dtype} {(*lead, cols)} tensor on {device}, got "
                         f"{t.dtype} {tuple(t.shape)} on {t.device}")
    return _row_stride(name, t)


def _row_stride(name: str, t: torch.Tensor) -> int:
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: the values of a row must lie side by side")
    if t.dim() == 2:
        return t.stride(0) if t.shape[0] > 1 else t.shape[1]
    if t.shape[1] > 1:
        ld = t.stride(1)
        if t.shape[0] > 1 and t.stride(0) != t.shape[1] * ld:
            raise ValueError(f"{name}: the rows of all sequences must lie at one stride")
        return ld
    return t.stride(0) if t.shape[0] > 1 else t.shape[2]


def _vector(name: str, t: Optional[torch.Tensor], shape, device, dtype=torch.float32):
    if t is not None and (tuple(t.shape) != tuple(shape) or t.dtype != dtype
                          or t.device != device or not t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous {dtype} {tuple(shape)} tensor on {device}")
    return t


def _tokens(name: str, x: torch.Tensor):
    """(leading shape, width, tokens) of a token tensor."""
    if x.dim() not in (2, 3) or x.dtype not in _DTYPES or not x.is_cuda:
        raise ValueError(f"{name} must be a [T, D] or [B, L, D] float32/bfloat16 GPU tensor")
    lead = tuple(x.shape[:-1])
    return lead, int(x.shape[-1]), lead[0] if len(lead) == 1 else lead[0] * lead[1]


def _batch(lead, offsets, sequences, device) -> int:
    """The number of packed sequences."""
    if offsets is not None:
        if len(lead) != 1:
            raise ValueError("offsets go with packed [T, D] tensors")
        if (offsets.dim() != 1 or offsets.numel() < 1 or offsets.dtype != torch.int64
                or offsets.device != device or not offsets.is_contiguous()):
            raise ValueError(f"offsets must be a contiguous int64 [B + 1] tensor on {device}")
        n = offsets.numel() - 1
    else:
        n = lead[0] if len(lead) == 2 else (1 if sequences is None else int(sequences))
    if sequences is not None and int(sequences) != n:
        raise ValueError(f"sequences is {sequences}, the tensors hold {n}")
    return n


def _states(name, t, slots, n, tail, dtype, device):
    """Checks a state tensor: [n or slots' rows, *tail]."""
    if t is None:
        return
    if (t.dim() != 1 + len(tail) or tuple(t.shape[1:]) != tail or t.dtype != dtype
            or t.device != device or not t.is_contiguous() or (slots is None and t.shape[0] != n)):
        raise ValueError(f"{name} must be a contiguous {dtype} "
                         f"{(n if slots is None else 'slots', *tail)} tensor on {device}")


def _slots(slots, states, n, device):
    """(pointer, rows of the state tensors)."""
    if slots is None:
        return None, 0
    if (slots.dim() != 1 or slots.numel() != n or slots.dtype != torch.int32
            or slots.device != device or not slots.is_contiguous()):
        raise ValueError(f"slots must be a contiguous int32 [{n}] tensor on {device}")
    rows = {t.shape[0] for t in states if t is not None}
    if len(rows) > 1:
        raise ValueError("state_in and state_out must have the same number of rows")
    return slots.data_ptr(), rows.pop() if rows else 0


def _scratch(need: int, workspace, device):
    """(the workspace, its pointer and bytes), allocated when needed and not given."""
    if workspace is None and need > 0:
        workspace = torch.empty((need,), dtype=torch.uint8, device=device)
    if workspace is None:
        return None, None, 0
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


# ---- norm --------------------------------------------------------------------

def _norm_inputs(x, weight, residual, residual_out):
    lead, D, T = _tokens("x", x)
    dev = x.device
    _vector("weight", weight, (D,), dev)
    ld_x = _row_stride("x", x)
    if residual is None:
        if residual_out is not None:
            raise ValueError("residual_out goes with a residual")
        return lead, D, T, ld_x, 0, 0, _DTYPES[x.dtype], None
    if residual.dtype not in _DTYPES:
        raise TypeError(f"residual must be float32 or bfloat16, got {residual.dtype}")
    ld_r = _rows("residual", residual, lead, D, residual.dtype, dev)
    if residual_out is None:
        residual_out = torch.empty((*lead, D), dtype=residual.dtype, device=dev)
    ld_o = _rows("residual_out", residual_out, lead, D, residual.dtype, dev)
    return lead, D, T, ld_x, ld_r, ld_o, _DTYPES[residual.dtype], residual_out


def lbi_rms_norm(x: torch.Tensor, weight: torch.Tensor, residual: Optional[torch.Tensor] = None,
                 eps: float = 1e-5, out: Optional[torch.Tensor] = None,
                 residual_out: Optional[torch.Tensor] = None, stream=None):
    """(out, residual_out): the root-mean-square norm of s = x + residual, and s (None without a
    residual).  residual_out may be residual itself."""
    lead, D, T, ld_x, ld_r, ld_o, rdt, residual_out = _norm_inputs(x, weight, residual,
                                                                   residual_out)
    if out is None:
        out = torch.empty((*lead, D), dtype=x.dtype, device=x.device)
    _check(load().lbi_rms_norm(
        x.data_ptr(), ld_x, _ptr(residual), ld_r, weight.data_ptr(), out.data_ptr(),
        _rows("out", out, lead, D, x.dtype, x.device), _ptr(residual_out), ld_o, T, D, eps,
        _DTYPES[x.dtype], rdt, _stream_ptr(stream, x.device)))
    return out, residual_out


def lbi_rms_norm_q8(x: torch.Tensor, weight: torch.Tensor,
                    residual: Optional[torch.Tensor] = None, eps: float = 1e-5,
                    format: int = LBI_Q8_E4M3, group: int = 0, q: Optional[torch.Tensor] = None,
                    scales: Optional[torch.Tensor] = None,
                    residual_out: Optional[torch.Tensor] = None, stream=None):
    """(q, scales, residual_out): the norm's output in 8 bits, q * scale, with one float32 scale
    for each ``group`` features of a token (0: for the token)."""
    lead, D, T, ld_x, ld_r, ld_o, rdt, residual_out = _norm_inputs(x, weight, residual,
                                                                   residual_out)
    if format not in _Q8_TYPES:
        raise ValueError(f"format must be LBI_Q8_E4M3 or LBI_Q8_INT8, got {format}")
    ngroups = -(-D // group) if group > 0 else 1
    if q is None:
        q = torch.empty((*lead, D), dtype=_Q8_TYPES[format], device=x.device)
    if scales is None:
        scales = torch.empty((*lead, ngroups), dtype=torch.float32, device=x.device)
    _vector("scales", scales, (*lead, ngroups), x.device)
    _check(load().lbi_rms_norm_q8(
        x.data_ptr(), ld_x, _ptr(residual), ld_r, weight.data_ptr(), q.data_ptr(),
        _rows("q", q, lead, D, _Q8_TYPES[format], x.device), scales.data_ptr(),
        _ptr(residual_out), ld_o, T, D, eps, group, format, _DTYPES[x.dtype], rdt,
        _stream_ptr(stream, x.device)))
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
    lead, D, T = _tokens("dout", dout)
    dev = dout.device
    if s.dtype not in _DTYPES:
        raise TypeError(f"s must be float32 or bfloat16, got {s.dtype}")
    ld_s = _rows("s", s, lead, D, s.dtype, dev)
    ld_r = 0 if dresidual is None else _rows("dresidual", dresidual, lead, D, s.dtype, dev)
    _vector("weight", weight, (D,), dev)
    if ds is None:
        ds = torch.empty((*lead, D), dtype=s.dtype, device=dev)
    if dweight is None:
        dweight = torch.empty((D,), dtype=torch.float32, device=dev)
    _vector("dweight", dweight, (D,), dev)
    workspace, w, wb = _scratch(lbi_rms_norm_backward_workspace_bytes(T, D), workspace, dev)
    _check(load().lbi_rms_norm_backward(
        dout.data_ptr(), _row_stride("dout", dout), s.data_ptr(), ld_s, weight.data_ptr(),
        _ptr(dresidual), ld_r, ds.data_ptr(), _rows("ds", ds, lead, D, s.dtype, dev),
        dweight.data_ptr(), T, D, eps, _DTYPES[dout.dtype], _DTYPES[s.dtype], w, wb,
        _stream_ptr(stream, dev)))
    return ds, dweight


# ---- convolution -------------------------------------------------------------

def _conv_inputs(x, weight, bias):
    lead, D, T = _tokens("x", x)
    if weight.dim() != 2:
        raise ValueError("weight must be [D, W]")
    W = int(weight.shape[1])
    _vector("weight", weight, (D, W), x.device)
    _vector("bias", bias, (D,), x.device)
    return lead, D, T, W, _row_stride("x", x)


def lbi_ssm_conv(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None,
                 silu: bool = True, offsets: Optional[torch.Tensor] = None,
                 sequences: Optional[int] = None, state_in: Optional[torch.Tensor] = None,
                 state_out: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None,
                 out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """The causal convolution of every channel with its W = 2 .. 4 taps weight [D, W] along the
    tokens of each sequence.  state_in, state_out [B, W - 1, D]: the tokens before each sequence
    and the last ones after it."""
    lead, D, T, W, ld_x = _conv_inputs(x, weight, bias)
    dev = x.device
    n = _batch(lead, offsets, sequences, dev)
    for name, t in (("state_in", state_in), ("state_out", state_out)):
        _states(name, t, slots, n, (W - 1, D), x.dtype, dev)
    sp, ns = _slots(slots, (state_in, state_out), n, dev)
    if out is None:
        out = torch.empty((*lead, D), dtype=x.dtype, device=dev)
    _check(load().lbi_ssm_conv(
        x.data_ptr(), ld_x, weight.data_ptr(), _ptr(bias), out.data_ptr(),
        _rows("out", out, lead, D, x.dtype, dev), _ptr(state_in), _ptr(state_out), sp, ns,
        _ptr(offsets), T, n, D, W, int(silu), _DTYPES[x.dtype], _stream_ptr(stream, dev)))
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
    lead, D, T, W, ld_x = _conv_inputs(x, weight, bias)
    dev = x.device
    n = _batch(lead, offsets, sequences, dev)
    for name, t in (("state_in", state_in), ("dstate_out", dstate_out)):
        _states(name, t, None, n, (W - 1, D), x.dtype, dev)
    ld_dout = _rows("dout", dout, lead, D, x.dtype, dev)
    if dx is None:
        dx = torch.empty((*lead, D), dtype=x.dtype, device=dev)
    dweight = torch.empty((D, W), dtype=torch.float32, device=dev)
    dbias = None if bias is None else torch.empty((D,), dtype=torch.float32, device=dev)
    dstate_in = None if state_in is None else torch.empty_like(state_in)
    workspace, w, wb = _scratch(lbi_ssm_conv_backward_workspace_bytes(T, D, W), workspace, dev)
    _check(load().lbi_ssm_conv_backward(
        x.data_ptr(), ld_x, weight.data_ptr(), _ptr(bias), dout.data_ptr(), ld_dout,
        _ptr(state_in), _ptr(dstate_out), dx.data_ptr(), _rows("dx", dx, lead, D, x.dtype, dev),
        dweight.data_ptr(), _ptr(dbias), _ptr(dstate_in), _ptr(offsets), T, n, D, W, int(silu),
        _DTYPES[x.dtype], w, wb, _stream_ptr(stream, dev)))
    return dx, dweight, dbias, dstate_in


def lbi_ssm_conv_step(x: torch.Tensor, weight: torch.Tensor, state_in: torch.Tensor,
                      state_out: torch.Tensor, bias: Optional[torch.Tensor] = None,
                      silu: bool = True, slots: Optional[torch.Tensor] = None,
                      out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """One token for each of n sequences, x [n, D]; state_out may be state_in."""
    lead, D, n, W, ld_x = _conv_inputs(x, weight, bias)
    if len(lead) != 1:
        raise ValueError("x must be [n, D]")
    dev = x.device
    for name, t in (("state_in", state_in), ("state_out", state_out)):
        _states(name, t, slots, n, (W - 1, D), x.dtype, dev)
    sp, ns = _slots(slots, (state_in, state_out), n, dev)
    if out is None:
        out = torch.empty((n, D), dtype=x.dtype, device=dev)
    _check(load().lbi_ssm_conv_step(
        x.data_ptr(), ld_x, weight.data_ptr(), _ptr(bias), out.data_ptr(),
        _rows("out", out, lead, D, x.dtype, dev), state_in.data_ptr(), state_out.data_ptr(), sp,
        ns, n, D, W, int(silu), _DTYPES[x.dtype], _stream_ptr(stream, dev)))
    return out


# ---- scan --------------------------------------------------------------------

def _groups(name, t, lead, N, dtype, device):
    """(row stride, groups) of B or C: [..., N] or [..., G, N]."""
    if (t.dtype != dtype or t.device != device or t.shape[:len(lead)] != lead
            or t.dim() - len(lead) not in (1, 2) or t.shape[-1] != N):
        raise ValueError(f"{name} must be a {dtype} {(*lead, 'G', N)} or {(*lead, N)} tensor on "
                         f"{device}")
    G = 1
    if t.dim() > len(lead) + 1:
        G = int(t.shape[-2])
        if G > 1 and t.stride(-2) != N:
            raise ValueError(f"{name}: a token's values must lie side by side")
        t = t.as_strided((*lead, G * N), (*t.stride()[:len(lead)], 1)) if t.stride(-1) == 1 or \
            N == 1 else t.flatten(-2)
    return _row_stride(name, t), G


def _scan_inputs(u, delta, A, B, C, skip, z, delta_bias, softplus, offsets, sequences, state_in):
    lead, D, T = _tokens("u", u)
    dev = u.device
    if A.dim() != 2:
        raise ValueError("A must be [D, N]")
    N = int(A.shape[1])
    _vector("A", A, (D, N), dev)
    _vector("skip", skip, (D,), dev)
    _vector("delta_bias", delta_bias, (D,), dev)
    ld_B, G = _groups("B", B, lead, N, u.dtype, dev)
    ld_C, G2 = _groups("C", C, lead, N, u.dtype, dev)
    if G != G2:
        raise ValueError("B and C must have the same groups")
    n = _batch(lead, offsets, sequences, dev)
    si = SsmInputs(u.data_ptr(), _row_stride("u", u), delta.data_ptr(),
                   _rows("delta", delta, lead, D, u.dtype, dev), _ptr(z),
                   0 if z is None else _rows("z", z, lead, D, u.dtype, dev), B.data_ptr(), ld_B,
                   C.data_ptr(), ld_C, A.data_ptr(), _ptr(skip), _ptr(delta_bias),
                   _ptr(state_in), _ptr(offsets), T, n, D, N, G, int(softplus),
                   _DTYPES[u.dtype])
    return si, lead, dev


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
    si, lead, dev = _scan_inputs(u, delta, A, B, C, skip, z, delta_bias, softplus, offsets,
                                 sequences, state_in)
    for name, t in (("state_in", state_in), ("state_out", state_out)):
        _states(name, t, slots, si.sequences, (si.D, si.N), torch.float32, dev)
    sp, ns = _slots(slots, (state_in, state_out), si.sequences, dev)
    if out is None:
        out = torch.empty((*lead, si.D), dtype=u.dtype, device=dev)
    need = lbi_ssm_scan_workspace_bytes(si.T, si.sequences, si.D, si.N, si.G, offsets is not None)
    workspace, w, wb = _scratch(need, workspace, dev)
    _check(load().lbi_ssm_scan(
        ctypes.byref(si), out.data_ptr(), _rows("out", out, lead, si.D, u.dtype, dev),
        _ptr(state_out), sp, ns, w, wb, _stream_ptr(stream, dev)))
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
    si, lead, dev = _scan_inputs(u, delta, A, B, C, skip, z, delta_bias, softplus, offsets,
                                 sequences, state_in)
    for name, t in (("state_in", state_in), ("dstate_out", dstate_out)):
        _states(name, t, None, si.sequences, (si.D, si.N), torch.float32, dev)
    ld_dout = _rows("dout", dout, lead, si.D, u.dtype, dev)
    grads = {}
    for name, t in (("u", u), ("delta", delta), ("A", A), ("B", B), ("C", C), ("skip", skip),
                    ("z", z), ("delta_bias", delta_bias), ("state_in", state_in)):
        g = None if outputs is None else outputs.get(name)
        if t is None:
            if g is not None:
                raise ValueError(f"outputs[{name!r}]: there is no such input")
        elif g is None:
            g = torch.empty(t.shape, dtype=t.dtype, device=dev)
        elif name in ("A", "skip", "delta_bias", "state_in"):
            _vector(f"outputs[{name!r}]", g, t.shape, dev)
        grads[name] = g
    ld = {k: 0 if grads[k] is None else _rows(f"outputs[{k!r}]", grads[k], lead, si.D, u.dtype,
                                              dev) for k in ("u", "delta", "z")}
    for k in ("B", "C"):
        ld[k], G = _groups(f"outputs[{k!r}]", grads[k], lead, si.N, u.dtype, dev)
        if G != si.G:
            raise ValueError(f"outputs[{k!r}] must have {si.G} groups")
    sg = SsmGradients(grads["u"].data_ptr(), ld["u"], grads["delta"].data_ptr(), ld["delta"],
                      _ptr(grads["z"]), ld["z"], grads["B"].data_ptr(), ld["B"],
                      grads["C"].data_ptr(), ld["C"], grads["A"].data_ptr(),
                      _ptr(grads["skip"]), _ptr(grads["delta_bias"]), _ptr(grads["state_in"]))
    need = lbi_ssm_scan_backward_workspace_bytes(si.T, si.sequences, si.D, si.N, si.G,
                                                 offsets is not None)
    workspace, w, wb = _scratch(need, workspace, dev)
    _check(load().lbi_ssm_scan_backward(
        ctypes.byref(si), dout.data_ptr(), ld_dout, _ptr(dstate_out), ctypes.byref(sg), w, wb,
        _stream_ptr(stream, dev)))
    return grads


def lbi_ssm_scan_step(u: torch.Tensor, delta: torch.Tensor, A: torch.Tensor, B: torch.Tensor,
                      C: torch.Tensor, state_in: torch.Tensor, state_out: torch.Tensor,
                      skip: Optional[torch.Tensor] = None, z: Optional[torch.Tensor] = None,
                      delta_bias: Optional[torch.Tensor] = None, softplus: bool = True,
                      slots: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                      stream=None) -> torch.Tensor:
    """One token for each of n sequences, u [n, D]; state_out may be state_in."""
    si, lead, dev = _scan_inputs(u, delta, A, B, C, skip, z, delta_bias, softplus, None,
                                 u.shape[0], state_in)
    if len(lead) != 1:
        raise ValueError("u must be [n, D]")
    for name, t in (("state_in", state_in), ("state_out", state_out)):
        _states(name, t, slots, si.sequences, (si.D, si.N), torch.float32, dev)
    sp, ns = _slots(slots, (state_in, state_out), si.sequences, dev)
    if out is None:
        out = torch.empty((lead[0], si.D), dtype=u.dtype, device=dev)
    _check(load().lbi_ssm_scan_step(
        ctypes.byref(si), out.data_ptr(), _rows("out", out, lead, si.D, u.dtype, dev),
        state_out.data_ptr(), sp, ns, _stream_ptr(stream, dev)))
    return out
