"""A chain of K regions with linear attention, trained by the interface-adjoint scan and then served.

A region takes its tokens and the interface vector m [r] from the region before it, and hands one on:
the interface is decoded onto the tokens, the sum is normalised, projected to queries, keys and
values, attended, projected back onto the tokens, put through a two-layer map, normalised, and read
out into the next interface.

Training and serving are compared as in examples/region_block.py: the gradients by
lbi_scan_backward over the regions' interface Jacobians with the chain's own, and the outputs of
single tokens behind ragged prompts with those of whole sequences.

    python -m examples.attention_block
"""
from __future__ import annotations

import torch

from paper_2605_09204_amd import binding, linear


class Norm(torch.autograd.Function):
    """(layer norm of x + residual, x + residual)."""

    @staticmethod
    def forward(ctx, x, residual, weight, bias):
        out, s = linear.lbi_layer_norm(x, weight, bias, residual)
        ctx.save_for_backward(s, weight)
        return out, s

    @staticmethod
    def backward(ctx, dout, ds):
        s, weight = ctx.saved_tensors
        ds, dw, db = linear.lbi_layer_norm_backward(dout.contiguous(), s, weight, ds.contiguous())
        return ds, ds, dw, db


class Projection(torch.autograd.Function):
    """act(x weight^T + bias) + residual."""

    @staticmethod
    def forward(ctx, x, weight, bias, act, residual):
        pre = None
        if act != linear.LBI_ACT_NONE:
            pre = x.new_empty(*x.shape[:-1], weight.shape[0])
        ctx.act, ctx.residual = act, residual is not None
        ctx.save_for_backward(x, weight, pre)
        return linear.lbi_projection(x, weight, bias, act, residual, pre=pre)

    @staticmethod
    def backward(ctx, dout):
        x, weight, pre = ctx.saved_tensors
        dout = dout.contiguous()
        dx, dw, db = linear.lbi_projection_backward(x, weight, dout, ctx.act, pre)
        return dx, dw, db, None, dout if ctx.residual else None


class Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, log_decay):
        ctx.save_for_backward(q, k, v, log_decay)
        return linear.lbi_linear_attention(q, k, v, log_decay)

    @staticmethod
    def backward(ctx, dout):
        q, k, v, log_decay = ctx.saved_tensors
        g = linear.lbi_linear_attention_backward(q, k, v, log_decay, dout.contiguous())
        return g["q"], g["k"], g["v"], g["log_decay"]


def make_weights(D=96, H=4, KH=2, DK=16, DV=24, X=160, r=16, seed=0, device="cuda:0"):
    """The weights of one region; all regions of a chain share them."""
    g = torch.Generator()
    g.manual_seed(seed)

    def mat(o, i):
        return torch.randn(o, i, generator=g) / i ** 0.5
    w = {"decode": mat(D, r), "norm_in": torch.ones(D), "norm_in_b": torch.zeros(D),
         "qkv": mat(H * DK + KH * (DK + DV), D), "qkv_b": torch.zeros(H * DK + KH * (DK + DV)),
         "log_decay": -torch.exp(torch.linspace(-4.0, -0.5, H)),
         "out": mat(D, H * DV), "out_b": torch.zeros(D), "norm_mid": torch.ones(D),
         "norm_mid_b": torch.zeros(D), "up": mat(X, D), "up_b": torch.zeros(X), "down": mat(D, X),
         "down_b": torch.zeros(D), "norm_out": torch.ones(D), "norm_out_b": torch.zeros(D),
         "encode": mat(r, D)}
    return {k: v.to(device) for k, v in w.items()}, (H, KH, DK, DV)


def heads(qkv, sizes):
    """Queries, keys and values as slices of the projection's rows."""
    H, KH, DK, DV = sizes
    q, k, v = qkv.split((H * DK, KH * DK, KH * DV), -1)
    return q.unflatten(-1, (H, DK)), k.unflatten(-1, (KH, DK)), v.unflatten(-1, (KH, DV))


def region(w, sizes, tokens, m):
    """tokens [n, L, D] and m [n, r] -> the next interfaces [n, r]."""
    none, silu = linear.LBI_ACT_NONE, linear.LBI_ACT_SILU
    decoded = (m @ w["decode"].T).unsqueeze(1).expand(tokens.shape).contiguous()
    h, s = Norm.apply(decoded, tokens, w["norm_in"], w["norm_in_b"])
    q, k, v = heads(Projection.apply(h, w["qkv"], w["qkv_b"], none, None), sizes)
    y = Attention.apply(q, k, v, w["log_decay"]).flatten(-2)
    y = Projection.apply(y, w["out"], w["out_b"], none, None)
    h, s = Norm.apply(y, s, w["norm_mid"], w["norm_mid_b"])
    h = Projection.apply(h, w["up"], w["up_b"], silu, None)
    s = Projection.apply(h, w["down"], w["down_b"], none, s)
    h, _ = Norm.apply(s, torch.zeros_like(s), w["norm_out"], w["norm_out_b"])
    return 0.5 * m + h.mean(1) @ w["encode"].T


def chain_gradients(w, sizes, tokens, m0, target):
    """The loss |m_K - target|^2 / 2 and its gradients, backwards through the chain."""
    w = {k: v.clone().requires_grad_() for k, v in w.items()}
    m = m0
    for k in range(tokens.shape[0]):
        m = region(w, sizes, tokens[k:k + 1], m)
    loss = 0.5 * (m - target).square().sum()
    return loss.detach(), dict(zip(w, torch.autograd.grad(loss, list(w.values()))))


def scan_gradients(w, sizes, tokens, m0, target):
    """The same, all regions at once, by the scan over their interface Jacobians."""
    K, r = tokens.shape[0], m0.shape[1]
    with torch.no_grad():
        ms = [m0]
        for k in range(K):
            ms.append(region(w, sizes, tokens[k:k + 1], ms[-1]))
    m_in, m_end = torch.cat(ms[:-1]), ms[-1]
    m_each = m_in.repeat_interleave(r, 0).requires_grad_()
    units = torch.eye(r, device=m0.device).repeat(K, 1)
    out = region(w, sizes, tokens.repeat_interleave(r, 0), m_each)
    (rows,) = torch.autograd.grad(out, m_each, units)
    A = rows.view(1, K, r, r).transpose(-1, -2).contiguous()
    lam = binding.lbi_scan_backward(A, None, m_end - target)
    lam_out = torch.cat([lam[0, 1:K], m_end - target])
    w = {k: v.clone().requires_grad_() for k, v in w.items()}
    grads = torch.autograd.grad(region(w, sizes, tokens, m_in), list(w.values()), lam_out)
    return 0.5 * (m_end - target).square().sum(), dict(zip(w, grads))


def train(K=5, L=70, D=96, r=16, seed=0):
    """The largest relative difference between the two ways' gradients."""
    w, sizes = make_weights(D=D, r=r, seed=seed)
    g = torch.Generator()
    g.manual_seed(seed + 1)
    tokens, m0, target = (torch.randn(s, generator=g).cuda() for s in ((K, L, D), (1, r), (1, r)))
    loss, want = chain_gradients(w, sizes, tokens, m0, target)
    loss2, got = scan_gradients(w, sizes, tokens, m0, target)
    # the keys' bias only shifts all keys of a token, the norms' inputs' mean is taken off: some
    # gradients are sums that cancel, so differences are taken over all weights' size
    size = max(t.norm().item() for t in want.values())
    worst = max((got[k] - want[k]).norm().item() for k in want) / size
    return max(worst, abs(loss2.item() / loss.item() - 1))


class Server:
    """A region's weights in bf16 and the states of its slots."""

    def __init__(self, w, sizes, slots):
        self.w = {k: v.bfloat16() if v.dim() == 2 else v for k, v in w.items()}
        self.sizes = sizes
        H, _, DK, DV = sizes
        self.state = w["out"].new_zeros(slots, H, DK, DV)

    def run(self, x, slots, offsets=None):
        """x [T, D] bf16: prompts behind each other (offsets), or one token for each slot."""
        w, none, silu = self.w, linear.LBI_ACT_NONE, linear.LBI_ACT_SILU
        h, s = linear.lbi_layer_norm(x, w["norm_in"], w["norm_in_b"], x.new_zeros(x.shape, dtype=torch.float32))
        q, k, v = heads(linear.lbi_projection(h, w["qkv"], w["qkv_b"]), self.sizes)
        state = {"state_in": self.state, "state_out": self.state, "slots": slots}
        if offsets is None:
            y = linear.lbi_linear_attention_step(q, k, v, w["log_decay"], **state)
        else:
            y = linear.lbi_linear_attention(q, k, v, w["log_decay"], offsets=offsets, **state)
        s = linear.lbi_projection(y.flatten(-2), w["out"], w["out_b"], none, s, out=s)
        h, _ = linear.lbi_layer_norm(s.bfloat16(), w["norm_mid"], w["norm_mid_b"])
        h = linear.lbi_projection(h, w["up"], w["up_b"], silu)
        return linear.lbi_projection(h, w["down"], w["down_b"], none, s)


def serve(lengths=(37, 1, 130, 64), steps=5, D=96, seed=0):
    """The relative difference between the single tokens' outputs and the whole sequences'."""
    w, sizes = make_weights(D=D, seed=seed)
    n = len(lengths)
    g = torch.Generator()
    g.manual_seed(seed + 2)
    seqs = [torch.randn(k + steps, D, generator=g).bfloat16().cuda() for k in lengths]

    def offsets(ks):
        return torch.tensor([0, *ks]).cumsum(0).cuda()
    slots = torch.randperm(n + 3, generator=g)[:n].to(torch.int32).cuda()
    whole = Server(w, sizes, n + 3).run(torch.cat(seqs), slots, offsets([k + steps for k in lengths]))
    server = Server(w, sizes, n + 3)
    server.run(torch.cat([s[:k] for s, k in zip(seqs, lengths)]), slots, offsets(lengths))
    got = torch.stack([server.run(torch.stack([s[k + t] for s, k in zip(seqs, lengths)]), slots)
                       for t in range(steps)], 1)
    want = torch.stack([y[-steps:] for y in whole.split([k + steps for k in lengths])])
    return ((got - want).norm() / want.norm()).item()


if __name__ == "__main__":
    print(f"training: gradients by the interface scan and by the chain differ by {train():.2g}")
    print(f"serving: single tokens and whole sequences differ by {serve():.2g}")
