"""The operators of a region block with linear attention from their definitions, in float64 on the
CPU.

Test infrastructure: the attention as a loop over sequences and tokens in torch float64 (stored
values widen exactly), gradients by automatic differentiation of the forward.  ``lengths`` are the
tokens of each packed sequence.
"""
from __future__ import annotations

import math

import torch


def _wide(t):
    return None if t is None else t.detach().cpu().double()


def layer_norm(x, weight=None, bias=None, residual=None, eps=1e-5):
    """(out, s)."""
    x, residual = _wide(x), _wide(residual)
    s = x if residual is None else x + residual
    return _layer_norm(s, _wide(weight), _wide(bias), eps), s


def _layer_norm(s, weight, bias, eps):
    d = s - s.mean(-1, keepdim=True)
    out = d / torch.sqrt((d * d).mean(-1, keepdim=True) + eps)
    if weight is not None:
        out = out * weight
    return out if bias is None else out + bias


def layer_norm_backward(dout, s, weight=None, dresidual=None, eps=1e-5):
    """(ds, dweight, dbias)."""
    s = _wide(s).requires_grad_()
    w = torch.ones(s.shape[-1], dtype=torch.float64) if weight is None else _wide(weight)
    w.requires_grad_()
    b = torch.zeros_like(w, requires_grad=True)
    ds, dw, db = torch.autograd.grad(_layer_norm(s, w, b, eps), [s, w, b], _wide(dout))
    return (ds if dresidual is None else ds + _wide(dresidual)), dw, db


def activation(act, z):
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z * (1 + torch.erf(z / math.sqrt(2))) / 2 if act == "gelu" else z


def projection(x, weight, bias=None, act="none", residual=None):
    """(out, pre)."""
    z = _wide(x) @ _wide(weight).T
    if bias is not None:
        z = z + _wide(bias)
    out = activation(act, z)
    return (out if residual is None else out + _wide(residual)), z


def slope(act, pre):
    z = _wide(pre).requires_grad_()
    return torch.autograd.grad(activation(act, z).sum(), z)[0]


def projection_backward(x, weight, dout, act="none", pre=None):
    """(dx, dweight, dbias, dz)."""
    dz = _wide(dout)
    if act != "none":
        dz = dz * slope(act, pre)
    return dz @ _wide(weight), dz.T @ _wide(x), dz.sum(0), dz


def _attention(q, k, v, log_decay, scale, lengths, state):
    """q [T, H, DK], k [T, KH, DK], v [T, KH, DV] in float64."""
    H, share = q.shape[1], q.shape[1] // k.shape[1]
    k, v = k.repeat_interleave(share, 1), v.repeat_interleave(share, 1)
    a = torch.exp(log_decay)[:, None, None]
    out, new, at = [q.new_zeros(0, H, v.shape[2])], [], 0
    for i, n in enumerate(lengths):
        S = state[i] if state is not None else q.new_zeros(H, q.shape[2], v.shape[2])
        for t in range(at, at + n):
            S = a * S + k[t, :, :, None] * v[t, :, None, :]
            out.append((scale * (q[t, :, :, None] * S).sum(1))[None])
        new.append(S)
        at += n
    new = torch.stack(new) if new else q.new_zeros(0, H, q.shape[2], v.shape[2])
    return torch.cat(out), new


def attention(q, k, v, log_decay, scale, lengths, state=None):
    """(out, states after the sequences)."""
    return _attention(_wide(q), _wide(k), _wide(v), _wide(log_decay), scale, lengths, _wide(state))


def attention_backward(q, k, v, log_decay, scale, lengths, dout, state=None, dstate=None):
    """The gradients by input."""
    ins = {"q": q, "k": k, "v": v, "log_decay": log_decay}
    ins = {n: _wide(t).requires_grad_() for n, t in ins.items()}
    if state is not None:
        ins["state_in"] = _wide(state).requires_grad_()
    out, new = _attention(*list(ins.values())[:4], scale, lengths, ins.get("state_in"))
    of, by = [out], [_wide(dout)]
    if dstate is not None:
        of.append(new)
        by.append(_wide(dstate))
    got = torch.autograd.grad(of, list(ins.values()), by, allow_unused=True)
    return {n: torch.zeros_like(t) if g is None else g for (n, t), g in zip(ins.items(), got)}


def attention_terms(q, k, v, log_decay, scale, lengths, dout=None):
    """Root sums of squares of what meets inside the products over pairs of tokens: for each value of
    out, of the terms p_ij v_j; with ``dout``, of those of dq, dk and dv as well (shared heads'
    together).  An operand's rounding enters each of them by itself."""
    q, k, v, dout = _wide(q), _wide(k), _wide(v), _wide(dout)
    H, KH = q.shape[1], k.shape[1]
    r = {"out": torch.zeros(q.shape[0], H, v.shape[2], dtype=torch.float64)}
    if dout is not None:
        r |= {"q": torch.zeros_like(q), "k": torch.zeros_like(k), "v": torch.zeros_like(v)}
    at = 0
    for n in lengths:
        rows = slice(at, at + n)
        at += n
        i = torch.arange(n, dtype=torch.float64)
        lag = i[:, None] - i
        for h in range(H):
            kh = h * KH // H
            fade = torch.where(lag >= 0, torch.exp(lag.clamp(min=0) * log_decay[h].item()), 0.0)
            fade = torch.where(lag == 0, 1.0, fade) * scale  # for a decay of -infinity
            a, b, c = q[rows, h], k[rows, kh], v[rows, kh]
            p = (a @ b.T * fade) ** 2
            r["out"][rows, h] = p @ c ** 2
            if dout is not None:
                d = dout[rows, h]
                e = (d @ c.T * fade) ** 2
                r["q"][rows, h] = e @ b ** 2
                r["k"][rows, kh] += e.T @ a ** 2
                r["v"][rows, kh] += p.T @ d ** 2
    return {name: t.sqrt() for name, t in r.items()}
