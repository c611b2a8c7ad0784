"""Calls of include/lbi_linear.h that the other tests do not make (needs a GPU): outputs left out at
the C interface, activations far from zero.

Activations: float32 rounds erf and 1 / (1 + e^-z) by 2^-23 and less of 1, which z multiplies as far as
they are not 0 or 1 to that precision (|z| < 8 for GELU; for SiLU the exponent's rounding is |z| 2^-24
of e^-z, and |z|^2 e^-|z| is below 1): 2^-20 absolutely, 2^-22 of the value, and the output's rounding.
"""
import ctypes

import pytest
import torch

from oracle import linear as ref
from paper_2605_09204_amd import linear
from test_gpu_linear import ACT, DTYPE, args_of, attention_inputs, gen_num, packing, rand, say

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
TAG = {torch.float32: 0, torch.bfloat16: 1}


def stream():
    return torch.cuda.current_stream().cuda_stream


def workspace(need):
    return torch.empty(max(need, 1), dtype=torch.uint8, device=DEV)


def subsets(names):
    for mask in range(1 << len(names)):
        yield [n for i, n in enumerate(names) if mask >> i & 1]


@pytest.mark.parametrize("T,D", [(70, 100), (300, 768), (9, 9000)])
def test_layer_norm_gradients_left_out(T, D):
    g = gen_num(D)
    dout, s, w = rand((T, D), g, torch.bfloat16), rand((T, D), g), rand((D,), g)
    want = dict(zip(("ds", "dw", "db"), linear.lbi_layer_norm_backward(dout, s, w)))
    need = linear.lbi_layer_norm_backward_workspace_bytes(T, D)
    for names in subsets(["dw", "db"]):
        got = {n: torch.full_like(want[n], float("nan")) for n in ["ds", *names]}
        p = {n: t.data_ptr() for n, t in got.items()}
        ws = workspace(need if names else 0)
        st = linear.load().lbi_layer_norm_backward(
            dout.data_ptr(), D, s.data_ptr(), D, w.data_ptr(), None, 0, p["ds"], D, p.get("dw"),
            p.get("db"), T, D, 1e-5, 1, 0, ws.data_ptr() if names else None, need if names else 0,
            stream())
        assert st == 0 and all(torch.equal(t, want[n]) for n, t in got.items()), names


@pytest.mark.parametrize("act", sorted(ACT))
@pytest.mark.parametrize("dtype,stream_dtype", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("T,K,N", [(300, 96, 200), (1300, 64, 72), (0, 8, 8)])
def test_projection_gradients_left_out(T, K, N, dtype, stream_dtype, act):
    g = gen_num(T + K)
    dt, st = DTYPE[dtype], DTYPE[stream_dtype]
    x, w = rand((T, K), g, dt), rand((N, K), g, dt)
    dout, pre = rand((T, N), g, st), rand((T, N), g, dt)
    pre = None if act == "none" else pre
    want = dict(zip(("dx", "dw", "db"), linear.lbi_projection_backward(x, w, dout, ACT[act], pre)))
    need = linear.lbi_projection_backward_workspace_bytes(T, K, N, ACT[act], dt, st)
    for names in subsets(["dx", "dw", "db"]):
        got = {n: torch.full_like(want[n], float("nan")) for n in names}
        p = {n: t.data_ptr() for n, t in got.items()}
        ws = workspace(need)
        status = linear.load().lbi_projection_backward(
            x.data_ptr() if "dw" in names else None, K, w.data_ptr() if "dx" in names else None, K,
            dout.data_ptr(), N, None if pre is None else pre.data_ptr(), N, p.get("dx"), K,
            p.get("dw"), K, p.get("db"), T, K, N, ACT[act], TAG[dt], TAG[st],
            ws.data_ptr() if need else None, need, stream())
        assert status == 0 and all(torch.equal(t, want[n]) for n, t in got.items()), names


@pytest.mark.parametrize("lengths", [[70, 0, 130], [64, 64], [2000]], ids=str)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_gradients_left_out(lengths, dtype):
    H, KH, DK, DV = 4, 2, 32, 48
    s, g = attention_inputs(lengths, H, KH, DK, DV, dtype, 3)
    T, B = sum(lengths), len(lengths)
    dout, scale = rand((T, H, DV), g, DTYPE[dtype]), 0.3
    want = linear.lbi_linear_attention_backward(*args_of(s), dout, scale, state_in=s["state"],
                                                **packing(lengths))
    off = packing(lengths).get("offsets")
    need = linear.lbi_linear_attention_backward_workspace_bytes(T, B, H, KH, DK, DV, off is not None,
                                                                DTYPE[dtype])
    a = linear.AttentionInputs(
        s["q"].data_ptr(), H * DK, s["k"].data_ptr(), KH * DK, s["v"].data_ptr(), KH * DV,
        s["log_decay"].data_ptr(), s["state"].data_ptr(), None if off is None else off.data_ptr(), T,
        B, H, KH, DK, DV, scale, TAG[DTYPE[dtype]])
    for names in subsets(["log_decay", "state_in"]):
        got = {n: torch.full_like(want[n], float("nan")) for n in ["q", "k", "v", *names]}
        p = {n: t.data_ptr() for n, t in got.items()}
        grads = linear.AttentionGradients(p["q"], H * DK, p["k"], KH * DK, p["v"], KH * DV,
                                          p.get("log_decay"), p.get("state_in"))
        ws = workspace(need)
        status = linear.load().lbi_linear_attention_backward(
            ctypes.byref(a), dout.data_ptr(), H * DV, None, ctypes.byref(grads), ws.data_ptr(), need,
            stream())
        assert status == 0 and all(torch.equal(t, want[n]) for n, t in got.items()), names


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_activations_far_from_zero(act, dtype):
    say(f"[activations] {act} {dtype}")
    z = torch.cat([torch.linspace(-40, 40, 1601), torch.tensor([0.0, 88.0, 89.0, 104.0, 1e4, 1e19, 1e30]),
                   -torch.tensor([0.0, 88.0, 89.0, 104.0, 1e4, 1e19, 1e30])]).to(DTYPE[dtype])
    z64 = z.double()
    half = torch.finfo(z.dtype).eps / 2
    x, one = z[:, None].to(DEV), torch.ones(1, 1, dtype=z.dtype, device=DEV)
    out = linear.lbi_projection(x, one, act=ACT[act])[:, 0].cpu().double()
    # beyond 100 the functions are z or 0 to more digits than there are
    want = torch.where(z64 > 100, z64, torch.where(z64 < -100, 0.0, ref.activation(act, z64.clamp(-100, 100))))
    assert ((out - want).abs() <= 2.0 ** -20 + (2.0 ** -22 + half) * want.abs()).all()
    want = torch.where(z64 > 100, 1.0, torch.where(z64 < -100, 0.0, ref.slope(act, z64.clamp(-100, 100))))
    dx, _, db = linear.lbi_projection_backward(x, one, torch.ones_like(x), ACT[act], x)
    # dz is rounded as an operand, then dx
    assert ((dx[:, 0].cpu().double() - want).abs() <= 2.0 ** -20 + (2.0 ** -22 + 2 * half) * want.abs()).all()
    assert abs(db.item() - want.sum().item()) <= z.numel() * (2.0 ** -20 + 2.0 ** -24 * want.abs().sum().item())
