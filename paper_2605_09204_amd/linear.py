"""Python binding of ``include/lbi_linear.h``, the operators of a region block with linear attention
(argument marshalling only, in the manner of ``block``, whose conventions hold here too).

Token tensors are [T, D], or [B, L, D] for B sequences of L tokens; queries, keys and values have
their heads behind the tokens, [T, H, DK] or [B, L, H, DK], the values of a token side by side.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from . import block
from .binding import _DTYPES
from .block import (_aside, _batch, _int32, _norm_inputs, _ptr, _row_stride, _rows, _run, _scratch,
                    _states, _stream, _tokens, _vector)

LBI_ACT_NONE = 0
LBI_ACT_SILU = 1
LBI_ACT_GELU = 2
LBI_PROJECTION_MAX = 65536
LBI_ATTENTION_MAX_DIM = 128
LBI_ATTENTION_MAX_H = 1024
LBI_ATTENTION_MAX_LD = 1 << 23


class AttentionInputs(ctypes.Structure):
    """lbi_attention_inputs."""

    _fields_ = [(n, t) for names, t in (
        (("q",), ctypes.c_void_p), (("ld_q",), ctypes.c_int64),
        (("k",), ctypes.c_void_p), (("ld_k",), ctypes.c_int64),
        (("v",), ctypes.c_void_p), (("ld_v",), ctypes.c_int64),
        (("log_decay", "state_in", "offsets"), ctypes.c_void_p),
        (("T", "sequences"), ctypes.c_int64), (("H", "KH", "DK", "DV"), ctypes.c_int32),
        (("scale",), ctypes.c_float), (("dt",), ctypes.c_int)) for n in names]


class AttentionGradients(ctypes.Structure):
    """lbi_attention_gradients."""

    _fields_ = [(n, t) for names, t in (
        (("dq",), ctypes.c_void_p), (("ld_dq",), ctypes.c_int64),
        (("dk",), ctypes.c_void_p), (("ld_dk",), ctypes.c_int64),
        (("dv",), ctypes.c_void_p), (("ld_dv",), ctypes.c_int64),
        (("dlog_decay", "dstate_in"), ctypes.c_void_p)) for n in names]


_lib = None


def load() -> ctypes.CDLL:
    """The HIP library with these entry points declared (raises RuntimeError when not built)."""
    global _lib
    if _lib is not None:
        return _lib
    lib = block.load()
    vp, i64, i32, sz, f32 = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_size_t,
                             ctypes.c_float)
    en = ctypes.c_int
    inputs, grads = ctypes.POINTER(AttentionInputs), ctypes.POINTER(AttentionGradients)
    for name, args, res in (
            ("lbi_layer_norm", [vp, i64, vp, i64, vp, vp, vp, i64, vp, i64, i64, i32, f32, en, en,
                                vp], en),
            ("lbi_layer_norm_backward_workspace_bytes", [i64, i32], sz),
            ("lbi_layer_norm_backward", [vp, i64, vp, i64, vp, vp, i64, vp, i64, vp, vp, i64, i32,
                                         f32, en, en, vp, sz, vp], en),
            ("lbi_projection_workspace_bytes", [i64, i32, i32, en], sz),
            ("lbi_projection", [vp, i64, vp, i64, vp, vp, i64, vp, i64, vp, i64, i64, i32, i32, en,
                                en, en, vp, sz, vp], en),
            ("lbi_projection_backward_workspace_bytes", [i64, i32, i32, en, en, en], sz),
            ("lbi_projection_backward", [vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp,
                                         i64, i32, i32, en, en, en, vp, sz, vp], en),
            ("lbi_linear_attention_workspace_bytes", [i64, i64, i32, i32, i32, i32, i32, en], sz),
            ("lbi_linear_attention", [inputs, vp, i64, vp, vp, i32, vp, sz, vp], en),
            ("lbi_linear_attention_backward_workspace_bytes", [i64, i64, i32, i32, i32, i32, i32,
                                                               en], sz),
            ("lbi_linear_attention_backward", [inputs, vp, i64, vp, grads, vp, sz, vp], en),
            ("lbi_linear_attention_step", [inputs, vp, i64, vp, vp, i32, vp], en)):
        fn = getattr(lib, name)
        fn.argtypes, fn.restype = args, res
    _lib = lib
    return lib


# ---- layer norm --------------------------------------------------------------

def lbi_layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None,
                   bias: Optional[torch.Tensor] = None,
                   residual: Optional[torch.Tensor] = None, eps: float = 1e-5,
                   out: Optional[torch.Tensor] = None,
                   residual_out: Optional[torch.Tensor] = None, stream=None):
    """(out, residual_out): the layer norm of s = x + residual, and s (None without a residual).
    residual_out may be residual itself."""
    if stream is not None:
        return _aside(lbi_layer_norm, stream, x, weight, bias, residual, eps, out=out,
                      residual_out=residual_out)
    shape, D, T, dtype, dev, ld_x, w, ld_r, ld_o, rdt, residual_out = _norm_inputs(
        x, weight, residual, residual_out)
    if out is None:
        out = x.new_empty(shape)
    _run(dev, load().lbi_layer_norm,
         x.data_ptr(), ld_x, _ptr(residual), ld_r, w, _vector("bias", bias, (D,), dev),
         out.data_ptr(), _rows("out", out, shape, dtype, dev), _ptr(residual_out), ld_o, T, D, eps,
         _DTYPES[dtype], rdt, _stream(dev))
    return out, residual_out


def lbi_layer_norm_backward_workspace_bytes(T: int, D: int) -> int:
    return int(load().lbi_layer_norm_backward_workspace_bytes(int(T), int(D)))


def lbi_layer_norm_backward(dout: torch.Tensor, s: torch.Tensor,
                            weight: Optional[torch.Tensor] = None,
                            dresidual: Optional[torch.Tensor] = None, eps: float = 1e-5,
                            ds: Optional[torch.Tensor] = None,
                            dweight: Optional[torch.Tensor] = None,
                            dbias: Optional[torch.Tensor] = None,
                            workspace: Optional[torch.Tensor] = None, stream=None):
    """(ds, dweight, dbias): the gradient of what was normalised (of x and of residual alike), with
    ``dresidual`` added, and of the weight and the bias.  ds may be dresidual itself."""
    if stream is not None:
        return _aside(lbi_layer_norm_backward, stream, dout, s, weight, dresidual, eps, ds=ds,
                      dweight=dweight, dbias=dbias, workspace=workspace)
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
        dweight = s.new_empty((D,), dtype=torch.float32)
    if dbias is None:
        dbias = s.new_empty((D,), dtype=torch.float32)
    workspace, ws, wb = _scratch(load().lbi_layer_norm_backward_workspace_bytes(T, D), workspace,
                                 dev)
    _run(dev, load().lbi_layer_norm_backward,
         dout.data_ptr(), ld_dout, s.data_ptr(), ld_s, w, _ptr(dresidual), ld_r, ds.data_ptr(),
         _rows("ds", ds, shape, st, dev), _vector("dweight", dweight, (D,), dev),
         _vector("dbias", dbias, (D,), dev), T, D, eps, _DTYPES[dtype], _DTYPES[st], ws, wb,
         _stream(dev))
    return ds, dweight, dbias


# ---- projection --------------------------------------------------------------

def _matrix(name: str, t: torch.Tensor, shape, dtype, dev: int) -> int:
    """Checks a matrix and returns its row stride."""
    if t.dim() != 2:
        raise ValueError(f"{name} must be a matrix")
    return _rows(name, t, shape, dtype, dev)


def _act(act) -> int:
    if act not in (LBI_ACT_NONE, LBI_ACT_SILU, LBI_ACT_GELU):
        raise ValueError(f"act must be LBI_ACT_NONE, LBI_ACT_SILU or LBI_ACT_GELU, got {act}")
    return int(act)


def lbi_projection_workspace_bytes(T: int, K: int, N: int, dtype: torch.dtype) -> int:
    return int(load().lbi_projection_workspace_bytes(int(T), int(K), int(N), _DTYPES[dtype]))


def lbi_projection(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None,
                   act: int = LBI_ACT_NONE, residual: Optional[torch.Tensor] = None,
                   out: Optional[torch.Tensor] = None, pre: Optional[torch.Tensor] = None,
                   workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """act(x weight^T + bias) + residual for weight [N, K] and a float32 bias [N].  ``out`` has
    the residual's type (without one, its own or x's) and may be the residual itself; ``pre``: a
    tensor to write act's argument to."""
    if stream is not None:
        return _aside(lbi_projection, stream, x, weight, bias, act, residual, out=out, pre=pre,
                      workspace=workspace)
    shape, T, dtype, dev, ld_x = _tokens("x", x)
    K = shape[-1]
    if weight.dim() != 2:
        raise ValueError("weight must be [N, K]")
    N = _int32("N", weight.shape[0])
    ld_w = _matrix("weight", weight, (N, K), dtype, dev)
    to = (*shape[:-1], N)
    ot = residual.dtype if residual is not None else out.dtype if out is not None else dtype
    if ot not in _DTYPES:
        raise TypeError(f"residual and out must be float32 or bfloat16, got {ot}")
    ld_r = 0 if residual is None else _rows("residual", residual, to, ot, dev)
    if out is None:
        out = x.new_empty(to, dtype=ot)
    ld_p = 0 if pre is None else _rows("pre", pre, to, dtype, dev)
    lib, dt = load(), _DTYPES[dtype]
    workspace, ws, wb = _scratch(lib.lbi_projection_workspace_bytes(T, K, N, dt), workspace, dev)
    _run(dev, lib.lbi_projection,
         x.data_ptr(), ld_x, weight.data_ptr(), ld_w, _vector("bias", bias, (N,), dev),
         _ptr(residual), ld_r, out.data_ptr(), _rows("out", out, to, ot, dev), _ptr(pre), ld_p, T,
         K, N, _act(act), dt, _DTYPES[ot], ws, wb, _stream(dev))
    return out


def lbi_projection_backward_workspace_bytes(T: int, K: int, N: int, act: int, dtype: torch.dtype,
                                            out_dtype: torch.dtype) -> int:
    return int(load().lbi_projection_backward_workspace_bytes(
        int(T), int(K), int(N), int(act), _DTYPES[dtype], _DTYPES[out_dtype]))


def lbi_projection_backward(x: torch.Tensor, weight: torch.Tensor, dout: torch.Tensor,
                            act: int = LBI_ACT_NONE, pre: Optional[torch.Tensor] = None,
                            dx: Optional[torch.Tensor] = None,
                            dweight: Optional[torch.Tensor] = None,
                            dbias: Optional[torch.Tensor] = None,
                            workspace: Optional[torch.Tensor] = None, stream=None):
    """(dx, dweight, dbias); ``pre``: what the forward call wrote there, required with an
    activation.  The residual's gradient is dout itself."""
    if stream is not None:
        return _aside(lbi_projection_backward, stream, x, weight, dout, act, pre, dx=dx,
                      dweight=dweight, dbias=dbias, workspace=workspace)
    shape, T, dtype, dev, ld_x = _tokens("x", x)
    K = shape[-1]
    if weight.dim() != 2:
        raise ValueError("weight must be [N, K]")
    N = _int32("N", weight.shape[0])
    ld_w = _matrix("weight", weight, (N, K), dtype, dev)
    to, ot = (*shape[:-1], N), dout.dtype
    if ot not in _DTYPES:
        raise TypeError(f"dout must be float32 or bfloat16, got {ot}")
    ld_d = _rows("dout", dout, to, ot, dev)
    ld_p = 0 if pre is None else _rows("pre", pre, to, dtype, dev)
    if dx is None:
        dx = x.new_empty(shape)
    if dweight is None:
        dweight = weight.new_empty((N, K))
    if dbias is None:
        dbias = x.new_empty((N,), dtype=torch.float32)
    lib, dt = load(), _DTYPES[dtype]
    need = lib.lbi_projection_backward_workspace_bytes(T, K, N, _act(act), dt, _DTYPES[ot])
    workspace, ws, wb = _scratch(need, workspace, dev)
    _run(dev, lib.lbi_projection_backward,
         x.data_ptr(), ld_x, weight.data_ptr(), ld_w, dout.data_ptr(), ld_d, _ptr(pre), ld_p,
         dx.data_ptr(), _rows("dx", dx, shape, dtype, dev), dweight.data_ptr(),
         _matrix("dweight", dweight, (N, K), dtype, dev), _vector("dbias", dbias, (N,), dev), T, K,
         N, int(act), dt, _DTYPES[ot], ws, wb, _stream(dev))
    return dx, dweight, dbias


# ---- linear attention --------------------------------------------------------

def _heads(name: str, t: torch.Tensor, lead, dtype, dev: int):
    """(row stride, heads, values of one) of queries, keys or values: [..., heads, values]."""
    shape, stride, k = t.shape, t.stride(), len(lead)
    if t.dtype is not dtype or t.get_device() != dev or shape[:k] != lead or len(shape) != k + 2:
        raise ValueError(f"{name} must be a {dtype} {(*lead, 'heads', 'values')} tensor on "
                         f"cuda:{dev}, got {t.dtype} {tuple(shape)} on {t.device}")
    H, D = shape[-2], shape[-1]
    if (stride[-1] != 1 and D > 1) or (stride[-2] != D and H > 1):
        raise ValueError(f"{name}: a token's values must lie side by side")
    if (H | D) >> 31:  # the library takes them in 32 bits
        raise ValueError(f"{name}'s heads or values are out of range: {H}, {D}")
    if k == 1:
        return (stride[0] if lead[0] > 1 else H * D), H, D
    return _row_stride(name, (*lead, H * D), (*stride[:k], 1)), H, D


def _attention_inputs(q, k, v, log_decay, scale, offsets, sequences):
    """(the struct without states, shape before the heads, dtype, device index)."""
    if q.dtype not in _DTYPES:
        raise TypeError(f"q must be float32 or bfloat16, got {q.dtype}")
    if q.dim() not in (3, 4) or not q.is_cuda:
        raise ValueError("q must be a [T, H, DK] or [B, L, H, DK] GPU tensor")
    lead, dtype, dev = q.shape[:-2], q.dtype, q.get_device()
    ld_q, H, DK = _heads("q", q, lead, dtype, dev)
    ld_k, KH, DK2 = _heads("k", k, lead, dtype, dev)
    ld_v, KH2, DV = _heads("v", v, lead, dtype, dev)
    if DK2 != DK or KH2 != KH:
        raise ValueError("k must have q's values a head, and v k's heads")
    n = _batch((*lead, 1), offsets, sequences, dev)
    T = lead[0] if len(lead) == 1 else lead[0] * lead[1]
    return AttentionInputs(
        q.data_ptr(), ld_q, k.data_ptr(), ld_k, v.data_ptr(), ld_v,
        _vector("log_decay", log_decay, (H,), dev), None, _ptr(offsets), T, n, H, KH, DK, DV,
        max(DK, 1) ** -0.5 if scale is None else float(scale), _DTYPES[dtype]), lead, dtype, dev


def _output(name, out, like, shape, dtype, dev: int):
    """(the tensor, its row stride), allocated when not given."""
    if out is None:
        out = like.new_empty(shape)
    stride, H, D = _heads(name, out, shape[:-2], dtype, dev)
    if (H, D) != tuple(shape[-2:]):
        raise ValueError(f"{name} must be {tuple(shape)}")
    return out, stride


def lbi_linear_attention_workspace_bytes(T: int, sequences: int, H: int, KH: int, DK: int, DV: int,
                                         ragged: bool, dtype: torch.dtype) -> int:
    return int(load().lbi_linear_attention_workspace_bytes(
        int(T), int(sequences), int(H), int(KH), int(DK), int(DV), int(ragged), _DTYPES[dtype]))


def lbi_linear_attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                         log_decay: torch.Tensor, scale: Optional[float] = None,
                         offsets: Optional[torch.Tensor] = None, sequences: Optional[int] = None,
                         state_in: Optional[torch.Tensor] = None,
                         state_out: Optional[torch.Tensor] = None,
                         slots: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                         workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Causal linear attention of q [..., H, DK] to k [..., KH, DK] and v [..., KH, DV], heads
    h H/KH .. sharing keys and values, whose weights fade by exp(log_decay[h]) a token; scale:
    DK^-1/2 unless given.  state_in, state_out [B, H, DK, DV] float32: the states before and after
    each sequence; they may be the same tensor."""
    if stream is not None:
        return _aside(lbi_linear_attention, stream, q, k, v, log_decay, scale, offsets, sequences,
                      state_in, state_out=state_out, slots=slots, out=out, workspace=workspace)
    a, lead, dtype, dev = _attention_inputs(q, k, v, log_decay, scale, offsets, sequences)
    a.state_in, so, sp, ns = _states(state_in, state_out, slots, a.sequences, (a.H, a.DK, a.DV),
                                     torch.float32, dev)
    out, ld_o = _output("out", out, q, (*lead, a.H, a.DV), dtype, dev)
    lib = load()
    need = lib.lbi_linear_attention_workspace_bytes(a.T, a.sequences, a.H, a.KH, a.DK, a.DV,
                                                    int(offsets is not None), a.dt)
    workspace, w, wb = _scratch(need, workspace, dev)
    _run(dev, lib.lbi_linear_attention, ctypes.byref(a), out.data_ptr(), ld_o, so, sp, ns, w, wb,
         _stream(dev))
    return out


def lbi_linear_attention_backward_workspace_bytes(T: int, sequences: int, H: int, KH: int, DK: int,
                                                  DV: int, ragged: bool,
                                                  dtype: torch.dtype) -> int:
    return int(load().lbi_linear_attention_backward_workspace_bytes(
        int(T), int(sequences), int(H), int(KH), int(DK), int(DV), int(ragged), _DTYPES[dtype]))


def lbi_linear_attention_backward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                                  log_decay: torch.Tensor, dout: torch.Tensor,
                                  scale: Optional[float] = None,
                                  offsets: Optional[torch.Tensor] = None,
                                  sequences: Optional[int] = None,
                                  state_in: Optional[torch.Tensor] = None,
                                  dstate_out: Optional[torch.Tensor] = None,
                                  outputs: Optional[dict] = None,
                                  workspace: Optional[torch.Tensor] = None, stream=None) -> dict:
    """The gradients by input: "q", "k", "v", "log_decay" and "state_in" (None without one).
    ``outputs``: tensors to write some of them to."""
    if stream is not None:
        return _aside(lbi_linear_attention_backward, stream, q, k, v, log_decay, dout, scale, offsets,
                      sequences, state_in, dstate_out, outputs=outputs, workspace=workspace)
    a, lead, dtype, dev = _attention_inputs(q, k, v, log_decay, scale, offsets, sequences)
    a.state_in, so, _, _ = _states(state_in, dstate_out, None, a.sequences, (a.H, a.DK, a.DV),
                                   torch.float32, dev, ("state_in", "dstate_out"))
    ld_dout, H, DV = _heads("dout", dout, lead, dtype, dev)
    if (H, DV) != (a.H, a.DV):
        raise ValueError(f"dout must be {(*lead, a.H, a.DV)}")
    g = {} if outputs is None else dict(outputs)
    names = ("q", "k", "v", "log_decay", "state_in")
    if not g.keys() <= set(names):
        raise ValueError(f"outputs go by the inputs' names, got {sorted(g.keys() - set(names))}")
    if state_in is None and g.get("state_in") is not None:
        raise ValueError("outputs['state_in']: there is no such input")
    ld = {}
    for name, t in (("q", q), ("k", k), ("v", v)):
        g[name], ld[name] = _output(f"outputs['{name}']", g.get(name), t, t.shape, dtype, dev)
    if g.get("log_decay") is None:
        g["log_decay"] = log_decay.new_empty((a.H,))
    if g.get("state_in") is None:
        g["state_in"] = None if state_in is None else torch.empty_like(state_in)
    ag = AttentionGradients(
        g["q"].data_ptr(), ld["q"], g["k"].data_ptr(), ld["k"], g["v"].data_ptr(), ld["v"],
        _vector("outputs['log_decay']", g["log_decay"], (a.H,), dev),
        _vector("outputs['state_in']", g["state_in"], (a.sequences, a.H, a.DK, a.DV), dev))
    lib = load()
    need = lib.lbi_linear_attention_backward_workspace_bytes(
        a.T, a.sequences, a.H, a.KH, a.DK, a.DV, int(offsets is not None), a.dt)
    workspace, w, wb = _scratch(need, workspace, dev)
    _run(dev, lib.lbi_linear_attention_backward, ctypes.byref(a), dout.data_ptr(), ld_dout, so,
         ctypes.byref(ag), w, wb, _stream(dev))
    return g


def lbi_linear_attention_step(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                              log_decay: torch.Tensor, state_in: torch.Tensor,
                              state_out: torch.Tensor, scale: Optional[float] = None,
                              slots: Optional[torch.Tensor] = None,
                              out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """One token for each of n sequences, q [n, H, DK]; state_out may be state_in."""
    if stream is not None:
        return _aside(lbi_linear_attention_step, stream, q, k, v, log_decay, state_in, state_out,
                      scale, slots, out=out)
    if q.dim() != 3:
        raise ValueError("q must be [n, H, DK]")
    a, lead, dtype, dev = _attention_inputs(q, k, v, log_decay, scale, None, q.shape[0])
    a.state_in, so, sp, ns = _states(state_in, state_out, slots, a.sequences, (a.H, a.DK, a.DV),
                                     torch.float32, dev)
    out, ld_o = _output("out", out, q, (*lead, a.H, a.DV), dtype, dev)
    _run(dev, load().lbi_linear_attention_step, ctypes.byref(a), out.data_ptr(), ld_o, so, sp, ns,
         _stream(dev))
    return out
