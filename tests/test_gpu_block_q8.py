"""The 8-bit norm value by value (needs a GPU).

A quotient that lies in the middle between two 8-bit values is decided by the last bits of what it
was computed from, so no tolerance helps there: the library adds a row's squares in one stated order
and rounds after each operation, and its bytes, scales and sums are then those of the same formula in
float32 tensor operations, bit for bit.  (That holds for 8 rows and more and up to 2^24 values; for
fewer rows the tensor operations use other orders, for more values another 1 / D.)
"""
import pytest
import torch

from oracle import block as ref
from paper_2605_09204_amd import block

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
FORMAT = {"e4m3": block.LBI_Q8_E4M3, "int8": block.LBI_Q8_INT8}
EPS = 1e-5


def inputs(T, D, dtype, stream, residual, seed=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(T * 101 + D + seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV)
    size = torch.exp(0.5 * normal(D))
    x = (normal(T, D) * size).to(DTYPE[dtype])
    r = (normal(T, D) * size).to(DTYPE[stream]) if residual else None
    return x, 1.0 + 0.1 * normal(D), r


def formula(x, w, r, fmt, group):
    """(q, scales, s) in float32 tensor operations."""
    s = x.float() if r is None else x.float() + r.float()
    out = s * torch.rsqrt((s * s).mean(1, keepdim=True) + EPS) * w
    T, D = out.shape
    width = group or D
    n = -(-D // width)
    padded = torch.zeros(T, n * width, device=DEV)
    padded[:, :D] = out
    scales = padded.view(T, n, width).abs().amax(2) / (448.0 if fmt == "e4m3" else 127.0)
    v = out / scales.repeat_interleave(width, 1)[:, :D]
    q = v.to(torch.float8_e4m3fn) if fmt == "e4m3" else torch.round(v).to(torch.int8)
    return q, scales, s


SHAPES = [(4099, 2048), (3001, 768), (777, 4096), (5003, 128), (700, 1111), (2003, 130), (64, 8000),
          (9, 16), (40, 17), (33, 63), (301, 64), (200, 100), (64, 127), (51, 129), (45, 131),
          (31, 1024), (30, 1025), (23, 2047), (20, 4100), (12, 8127), (6747, 176), (301, 132),
          (700, 143), (90, 200), (512, 255), (100, 256), (64, 257), (9, 252), (8, 8128), (300, 8129),
          (40, 8192), (17, 8195), (9, 12345), (33, 16384), (8, 16383)]


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("T,D", SHAPES)
def test_bytes_are_those_of_the_formula(T, D, fmt):
    types = [("bf16", "bf16", True), ("f32", "f32", False), ("bf16", "f32", True),
             ("f32", "bf16", True)]
    for i, (dtype, stream, residual) in enumerate(types):
        group = (128, 0, 32, 64)[(i + D) % 4]
        print(f"[q8 formula] T={T} D={D} {fmt} {dtype} {stream} group={group}", flush=True)
        x, w, r = inputs(T, D, dtype, stream, residual)
        q, scales, s = block.lbi_rms_norm_q8(x, w, r, EPS, FORMAT[fmt], group)
        want, want_scales, total = formula(x, w, r, fmt, group)
        assert torch.equal(scales, want_scales)
        different = (q.view(torch.uint8) != want.view(torch.uint8)).sum().item()
        assert different == 0, f"{different} of {q.numel()} values"
        assert s is None or torch.equal(s, total.to(s.dtype))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype,stream", [("f32", "f32"), ("bf16", "f32"), ("f32", "bf16"),
                                          ("bf16", "bf16")])
@pytest.mark.parametrize("T,D", [(1, 40), (5, 300), (2, 1500), (3, 9000)])
def test_values_against_64_bits(T, D, dtype, stream, fmt):
    """Half a step of the 8-bit type, at any shape and pair of types; rows of q at a stride of their
    own, with nothing written beside them."""
    print(f"[q8 values] T={T} D={D} {fmt} {dtype} {stream}", flush=True)
    x, w, r = inputs(T, D, dtype, stream, True, seed=7)
    for group in (0, 32, 64, 128):
        wide = torch.full((T, D + 11), 0x55, dtype=torch.uint8, device=DEV)
        kind = torch.float8_e4m3fn if fmt == "e4m3" else torch.int8
        q, scales, _ = block.lbi_rms_norm_q8(x, w, r, EPS, FORMAT[fmt], group,
                                             q=wide.view(kind)[:, 5:5 + D])
        assert (wide[:, :5] == 0x55).all() and (wide[:, 5 + D:] == 0x55).all()
        want, _ = ref.rms_norm(x, w, r)
        assert torch.allclose(scales.cpu().double(), ref.q8_scales(want, group, fmt), rtol=1e-5, atol=0)
        sc = scales.cpu().double().repeat_interleave(group or D, -1)[..., :D]
        err = (q.cpu().float().double() * sc - want).abs()
        if fmt == "e4m3":  # half a step is 2^-4 of the value, or of the smallest normal one, 2^-6
            bound = torch.maximum(want.abs(), sc * 2.0 ** -6) * 2.0 ** -4
        else:
            bound = sc * 0.5
        assert (err <= bound * (1 + 1e-4) + 1e-30).all(), (err / bound).max()


def test_a_group_that_32_bits_do_not_hold_is_refused():
    x, w = torch.zeros(6, 256, device=DEV), torch.ones(256, device=DEV)
    for group in (1 << 32, (1 << 32) + 128, -(1 << 32) + 32):
        with pytest.raises(ValueError):
            block.lbi_rms_norm_q8(x, w, group=group)
    torch.cuda.synchronize()
