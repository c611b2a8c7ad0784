"""The projection's larger tiles, whole and with the sum cut, against its definition in float64,
element by element (needs a GPU; which tile each call takes is held by test_linear_plans.py).

Bounds for each element, u = eps / 2 of a type (bf16 2^-8, float32 2^-24):
  - a float32 sum of K products: (K + 8) 2^-24 of the sum of their magnitudes, in any order; float32
    operands as three bf16 values leave out 2^-22 of each product;
  - an activation: 2^-22 |z| (2 + |z|), its argument's error times its steepest slope, 1.13;
  - dz rounded to bf16 as an operand: errors of at most 2^-8 of each term, independent of each other, so
    with a deviation of at most 2^-8 / sqrt(3) of the terms' root sum of squares; seven deviations,
    4.1 of 2^-8, are passed once in 10^11;
  - the output's rounding, u of the element.
Rows in 16-byte pieces, the same as slices of wider rows whose other values are NaN, and rows at odd
places (through registers instead of straight into LDS) have to agree bit for bit.
"""
import pytest
import torch

from oracle import linear as ref
from paper_2605_09204_amd import linear
from test_gpu_linear import ACT, DTYPE, beside, gen_num, rand, say, wide_rows
from test_linear_plans import DWEIGHT, DX, FORWARD

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
SUM = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def within(got, want, bound, label):
    got64 = got.cpu().double()
    off = (got64 - want).abs() - bound - half_step(got.dtype) * want.abs()
    bad = ~(off <= 0)
    assert not bad.any(), (f"{label}: {int(bad.sum())} of {bad.numel()} elements, the first at "
                           f"{bad.nonzero()[0].tolist()}, by {off[bad].max().item():.3g}")


def products(a, b, K):
    """(a b^T in float64, what its float32 sums may be off by)."""
    return a @ b.T, ((K + 8) * SUM + 2.0 ** -22) * (a.abs() @ b.abs().T)


def pieces(t):
    """The same values as a slice of wider rows, in whole 16-byte pieces; the rest is NaN."""
    full = torch.full((t.shape[0], (t.shape[1] + 7) // 8 * 8 + 32), float("nan"), dtype=t.dtype,
                      device=t.device)
    view = full[:, 16:16 + t.shape[1]]
    view.copy_(t)
    return view


@pytest.mark.parametrize("T,K,N", [c[0] for c in FORWARD])
@pytest.mark.parametrize("dtype,stream", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"),
                                          ("bf16", "f32")])
def test_projection_tiles(T, K, N, dtype, stream):
    act = {"f32f32": "silu", "bf16bf16": "gelu", "f32bf16": "none", "bf16f32": "silu"}[dtype + stream]
    say(f"[projection] T={T} K={K} N={N} {dtype} {stream} {act}")
    g = gen_num(T + 3 * K + 7 * N)
    dt, st = DTYPE[dtype], DTYPE[stream]
    x, w = rand((T, K), g, dt), rand((N, K), g, dt, K ** -0.5)
    b, res = rand((N,), g, scale=0.3), rand((T, N), g, st)
    pre = torch.full((T, N), float("nan"), dtype=dt, device=DEV)
    out = linear.lbi_projection(x, w, b, ACT[act], res, pre=pre)
    b64 = b.cpu().double()
    z, off = products(x.cpu().double(), w.cpu().double(), K)
    z = z + b64
    off += 4 * SUM * (b64.abs() + z.abs())
    within(pre, z, off, "pre")
    y, r64 = ref.activation(act, z), res.cpu().double()
    if act != "none":
        off = 1.13 * off + 2.0 ** -22 * z.abs() * (2 + z.abs())
    within(out, y + r64, off + 2 * SUM * (y.abs() + r64.abs()), "out")
    for rows in (pieces, lambda t: wide_rows(t, 5)):
        rs, ps = rows(res), rows(torch.zeros_like(pre))
        linear.lbi_projection(rows(x), rows(w), b, ACT[act], rs, out=rs, pre=ps)  # in place
        assert torch.equal(rs, out) and torch.equal(ps, pre)
        assert torch.isnan(beside(rs)).all() and torch.isnan(beside(ps)).all()


@pytest.mark.parametrize("T,K,N", [c[0] for c in DX + DWEIGHT])
@pytest.mark.parametrize("dtype,stream", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"),
                                          ("bf16", "f32")])
def test_projection_backward_tiles(T, K, N, dtype, stream):
    act = {"f32f32": "gelu", "bf16bf16": "silu", "f32bf16": "silu", "bf16f32": "none"}[dtype + stream]
    say(f"[projection_backward] T={T} K={K} N={N} {dtype} {stream} {act}")
    g = gen_num(T + 5 * K + 11 * N)
    dt, st = DTYPE[dtype], DTYPE[stream]
    x, w = rand((T, K), g, dt), rand((N, K), g, dt, K ** -0.5)
    dout = rand((T, N), g, st)
    pre = None if act == "none" else rand((T, N), g, dt)
    dx, dw, db = linear.lbi_projection_backward(x, w, dout, ACT[act], pre)
    dz, x64, w64 = dout.cpu().double(), x.cpu().double(), w.cpu().double()
    off = torch.zeros_like(dz)  # of dz, in float32
    if pre is not None:
        z = pre.cpu().double()
        off = 2.0 ** -22 * dz.abs() * (2 + z.abs())
        dz = dz * ref.slope(act, pre)
    # operands that are dout's own bf16 values are not rounded
    rounding = 4.1 * 2.0 ** -8 if dt == torch.bfloat16 and (pre is not None or st != dt) else 0.0
    for got, a, b, n, e, label in ((dx, dz, w64.T, N, off, "dx"), (dw, dz.T, x64.T, T, off.T, "dweight")):
        want, bound = products(a, b, n)
        bound += (e + 2 * SUM * a.abs()) @ b.abs().T
        bound += rounding * ((a * a) @ (b * b).T).sqrt()
        within(got, want, bound, label)
    within(db, dz.sum(0), ((T + 8) * SUM * dz.abs() + off).sum(0), "dbias")
    for rows in (pieces, lambda t: wide_rows(t, 5)):
        xs, ws = rows(torch.zeros_like(x)), rows(torch.zeros_like(w))
        again = linear.lbi_projection_backward(rows(x), rows(w), rows(dout), ACT[act],
                                               None if pre is None else rows(pre), dx=xs, dweight=ws)
        assert torch.equal(xs, dx) and torch.equal(ws, dw) and torch.equal(again[2], db)
        assert torch.isnan(beside(xs)).all() and torch.isnan(beside(ws)).all()
