"""Layer norm of rows whose values are equal, lie close together far from zero, or are so large that
their squares pass float32's range (needs a GPU).

Where the values of a row are equal, the differences from their mean are exactly zero, so the output
is the bias to the last bit.  So it is where the sum of the squares is infinite: its reciprocal root
is zero, and nothing of a finite row is left; the gradient is then dresidual, the weight's zero.
Everything else has the tolerances of the operators' parity tests.
"""
import pytest
import torch

from oracle import linear as ref
from paper_2605_09204_amd import linear
from test_gpu_linear import DTYPE, check, gen_num, rand, say

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
WIDTHS = [3, 100, 300, 777, 1000, 1111, 2047, 3000, 5000, 9000, 16383]
TYPES = [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")]


def parameters(D, g):
    return 1.0 + rand((D,), g, scale=0.2), rand((D,), g)


def backward(dout, s, w, dres):
    """The gradient, in memory that held something else."""
    return linear.lbi_layer_norm_backward(dout, s, w, dres, ds=torch.full_like(s, float("nan")))


@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("dtype,stream", TYPES)
def test_equal_values(D, dtype, stream):
    """Rows of one value each, 2^-126 to 2^126."""
    say(f"[layer norm] equal values, D={D} {dtype} {stream}")
    g = gen_num(D)
    c = torch.rand(85, 1, generator=g) + 1.0
    c = torch.ldexp(c, torch.arange(-126, 127, 3)[:, None]) * (1 - 2 * (torch.arange(85) % 2))[:, None]
    w, b = parameters(D, g)
    x = c.to(DTYPE[dtype]).to(DEV).expand(85, D).contiguous()
    out, _ = linear.lbi_layer_norm(x, w, b)
    assert torch.equal(out, b.to(out.dtype).expand(85, D))
    res = (0.3 * c.flip(0)).to(DTYPE[stream]).to(DEV).expand(85, D).contiguous()
    total = (x.float() + res.float()).to(res.dtype)
    out, _ = linear.lbi_layer_norm(x, w, b, res, residual_out=res)
    assert torch.equal(out, b.to(out.dtype).expand(85, D)) and torch.equal(res, total)
    dout, dres = rand((85, D), g, DTYPE[dtype]), rand((85, D), g, DTYPE[stream])
    ds, dw, db = backward(dout, total, w, dres)
    want, _, want_b = ref.layer_norm_backward(dout, total, w, dres)
    check(ds, want, "ds", floor=1e-5 ** -0.5 * dout.float().norm().item())
    check(db, want_b, "dbias", floor=dout.float().norm().item())
    assert (dw == 0).all()


@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("base", [3.5, 1e8, -9.42e17, 1e24])
def test_neighbouring_values(D, base):
    """Rows of a float32 value and the next one: squares of their distance stay in range."""
    say(f"[layer norm] neighbours of {base:g}, D={D}")
    g = gen_num(D + 1)
    c = torch.full((9, D), base)
    up = torch.nextafter(c, 2 * c)
    pick = torch.rand(9, D, generator=g) < torch.tensor(
        [0.5, 0.5, 0.5, 0.1, 0.1, 0.9, 0.9, 0.0, 1.0])[:, None]
    pick[:, 0], pick[:, 1] = True, False
    pick[7, 1:], pick[8, 1:], pick[8, 0] = False, True, False  # the first one apart from the others
    x = torch.where(pick, up, c).to(DEV)
    w, b = parameters(D, g)
    size = float(9 * D) ** 0.5
    out, _ = linear.lbi_layer_norm(x, w, b)
    check(out, ref.layer_norm(x, w, b)[0], "out", floor=size)
    dout, dres = rand((9, D), g), rand((9, D), g)
    ds, dw, _ = backward(dout, x, w, None)
    want, want_w, _ = ref.layer_norm_backward(dout, x, w)
    d = x.double().cpu() - x.double().cpu().mean(-1, keepdim=True)
    root = torch.sqrt((d * d).mean(-1, keepdim=True) + 1e-5)
    check(ds, want, "ds", floor=(dout.double().cpu() / root).norm().item())
    check(dw, want_w, "dweight", floor=dout.norm().item())


@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("scale", [1e15, 1e22, 1e28, 1e34, 1e37])
@pytest.mark.parametrize("mean", [0.0, 8.0])
def test_large_values(D, dtype, stream, scale, mean):
    """Normal values times 10^15, whose squares are in range, to 10^37, alone and about a mean that the
    sum of the row passes the range with."""
    say(f"[layer norm] D={D} {dtype} {stream} {scale:g} ({mean:g} + normal)")
    g = gen_num(D + 2)
    scale /= 1.0 + mean
    x = ((mean + torch.randn(5, D, generator=g)) * scale).to(DTYPE[dtype]).to(DEV)
    w, b = parameters(D, g)
    dout, dres = rand((5, D), g, DTYPE[dtype]), rand((5, D), g, DTYPE[stream])
    res = torch.zeros(5, D, dtype=DTYPE[stream], device=DEV)
    out, s = linear.lbi_layer_norm(x, w, b, res)
    s = s.clone()
    ds, dw, db = backward(dout, s, w, dres)
    check(db, ref.layer_norm_backward(dout, s, w)[2], "dbias", floor=dout.float().norm().item())
    if scale < 1e16:
        check(out, ref.layer_norm(x, w, b)[0], "out")
        want, want_w, _ = ref.layer_norm_backward(dout, s, w, dres)
        check(ds, want, "ds")
        check(dw, want_w, "dweight", floor=dout.float().norm().item())
    else:
        assert torch.equal(out, b.to(out.dtype).expand(5, D))
        assert torch.equal(ds, dres) and (dw == 0).all()


def test_differences_at_the_range_s_end():
    """The largest values of both signs give the bias; a difference from the mean that float32 does
    not hold makes its row NaN, and no other."""
    x, b = torch.randn(6, 300, device=DEV), torch.randn(300, device=DEV)
    good, _ = linear.lbi_layer_norm(x, None, b)
    x[1, 0::2], x[1, 1::2] = 3.4e38, -3.4e38
    x[2, 5], x[2, 200] = -3.4e38, 3.4e38
    x[4], x[4, 7] = -3.4e38, 3.4e38
    out, _ = linear.lbi_layer_norm(x, None, b)
    assert torch.equal(out[1], b) and torch.equal(out[2], b) and torch.isnan(out[4]).all()
    keep = [0, 3, 5]
    assert torch.equal(out[keep], good[keep])
    dout = torch.randn(6, 300, device=DEV)
    ds, _, _ = linear.lbi_layer_norm_backward(dout, x)
    assert (ds[1:3] == 0).all() and torch.isnan(ds[4]).all()
    assert torch.isfinite(ds[keep]).all()
