"""The operators of a state-space region block from their definitions, in float64 on the CPU.

Test infrastructure: the forward of each operator as a plain loop over sequences and tokens in
torch float64 (stored values widen exactly), and gradients by automatic differentiation of that
forward.  ``lengths`` are the tokens of each packed sequence.
"""
from __future__ import annotations

import torch

Q8_TOP = {"e4m3": 448.0, "int8": 127.0}


def _wide(t):
    return None if t is None else t.detach().cpu().double()


def rms_norm(x, weight, residual=None, eps=1e-5):
    """(out, s)."""
    x, weight, residual = _wide(x), _wide(weight), _wide(residual)
    s = x if residual is None else x + residual
    return s / torch.sqrt((s * s).mean(-1, keepdim=True) + eps) * weight, s


def q8_scales(out, group, fmt):
    """The scale of each group of features of ``out`` (0: the row)."""
    D = out.shape[-1]
    group = group or D
    top = torch.stack([out[..., i:i + group].abs().amax(-1) for i in range(0, D, group)], -1)
    scale = top / Q8_TOP[fmt]
    return torch.where(scale > 0, scale, 1.0)


def rms_norm_backward(dout, s, weight, dresidual=None, eps=1e-5):
    """(ds, dweight)."""
    s, weight = _wide(s).requires_grad_(), _wide(weight).requires_grad_()
    out = s / torch.sqrt((s * s).mean(-1, keepdim=True) + eps) * weight
    ds, dw = torch.autograd.grad(out, [s, weight], _wide(dout))
    return (ds if dresidual is None else ds + _wide(dresidual)), dw


def _conv(x, weight, bias, state, lengths, silu):
    D, W = weight.shape
    out, new, at = [x[:0]], [], 0
    for i, n in enumerate(lengths):
        old = state[i] if state is not None else x.new_zeros(W - 1, D)
        rows = torch.cat([old, x[at:at + n]])
        for t in range(n):
            v = (rows[t:t + W] * weight.T).sum(0)
            if bias is not None:
                v = v + bias
            out.append((v * torch.sigmoid(v) if silu else v)[None])
        new.append(rows[n:])
        at += n
    return torch.cat(out), torch.stack(new) if new else x.new_zeros(0, W - 1, D)


def conv(x, weight, bias, state, lengths, silu=True):
    """(out, states after the sequences)."""
    return _conv(_wide(x), _wide(weight), _wide(bias), _wide(state), lengths, silu)


def conv_backward(x, weight, bias, state, lengths, dout, dstate=None, silu=True):
    """(dx, dweight, dbias, dstate_in); the last two None without the input."""
    v = [None if t is None else _wide(t).requires_grad_() for t in (x, weight, bias, state)]
    out, new = _conv(*v, lengths, silu)
    return _gradients(v, [(out, dout), (new, dstate)])


def _scan(u, delta, A, B, C, skip, z, delta_bias, state, lengths, softplus):
    D, N = A.shape
    G = B.shape[1]
    step = delta if delta_bias is None else delta + delta_bias
    if softplus:
        step = torch.nn.functional.softplus(step, threshold=200.0)
    B, C = B.repeat_interleave(D // G, 1), C.repeat_interleave(D // G, 1)
    out, new, at = [u[:0]], [], 0
    for i, n in enumerate(lengths):
        h = state[i] if state is not None else u.new_zeros(D, N)
        for t in range(at, at + n):
            h = torch.exp(step[t][:, None] * A) * h + (step[t] * u[t])[:, None] * B[t]
            out.append((h * C[t]).sum(1)[None])
        new.append(h)
        at += n
    y = torch.cat(out)
    if skip is not None:
        y = y + skip * u
    if z is not None:
        y = y * z * torch.sigmoid(z)
    return y, torch.stack(new) if new else u.new_zeros(0, D, N)


SCAN_INPUTS = ("u", "delta", "A", "B", "C", "skip", "z", "delta_bias", "state_in")


def scan(inputs, lengths, softplus=True):
    """(y, states after the sequences) from a dict of SCAN_INPUTS (any of skip, z, delta_bias and
    state_in may be None); B and C are [T, G, N]."""
    return _scan(*(_wide(inputs.get(k)) for k in SCAN_INPUTS), lengths, softplus)


def scan_backward(inputs, lengths, dout, dstate=None, softplus=True):
    """The gradients, by input."""
    v = [None if inputs.get(k) is None else _wide(inputs[k]).requires_grad_()
         for k in SCAN_INPUTS]
    y, new = _scan(*v, lengths, softplus)
    return dict(zip(SCAN_INPUTS, _gradients(v, [(y, dout), (new, dstate)])))


def _gradients(inputs, pairs):
    of = [(o, _wide(g)) for o, g in pairs if g is not None and o.requires_grad]
    wrt = [t for t in inputs if t is not None]
    if not of:
        return [None if t is None else torch.zeros_like(t) for t in inputs]
    got = iter(torch.autograd.grad([o for o, _ in of], wrt, [g for _, g in of],
                                   allow_unused=True))
    out = []
    for t in inputs:
        g = None if t is None else next(got)
        out.append(None if t is None else (torch.zeros_like(t) if g is None else g))
    return out
