"""Forms of the region block's operators that test_gpu_block.py leaves out, against the float64
definitions and with its tolerances (needs a GPU): the scan's gradient without softplus, the norm's
gradient with float32 tokens on a bf16 stream, what lies beside strided outputs, and bf16 scans of
many ranges."""
import pytest
import torch

from oracle import block as ref
from paper_2605_09204_amd import block
from test_gpu_block import (DEV, DTYPE, LENGTHS, NORM_SHAPES, call_scan, check, gen_num, packing, rand,
                            scan_inputs, wide_rows)

pytestmark = pytest.mark.gpu


def say(msg):
    print(msg, flush=True)


def untouched(view):
    """The rest of a wide_rows() tensor is NaN still."""
    full, D = view._base, view.shape[-1]
    begin = view.storage_offset()
    return torch.isnan(full[..., :begin]).all() and torch.isnan(full[..., begin + D:]).all()


@pytest.mark.parametrize("T,D", NORM_SHAPES)
def test_norm_backward_of_float32_tokens_on_a_bf16_stream(T, D):
    say(f"[norm_backward] T={T} D={D} f32 bf16")
    g = gen_num(T * 43 + D)
    dout, s = rand((T, D), g), rand((T, D), g, torch.bfloat16, 1.5)
    w, dr = 1.0 + rand((D,), g, scale=0.2), rand((T, D), g, torch.bfloat16)
    ds, dw = block.lbi_rms_norm_backward(dout, s, w, dr)
    want, want_w = ref.rms_norm_backward(dout, s, w, dr)
    check(ds, want, "ds")
    check(dw, want_w, "dweight")


@pytest.mark.parametrize("lengths", ["short", "ragged", "long", "wide"])
@pytest.mark.parametrize("D,N,G", [(5, 3, 1), (130, 16, 2), (70, 64, 1)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scan_backward_without_softplus(lengths, D, N, G, dtype):
    say(f"[scan_backward] no softplus, {lengths} D={D} N={N} G={G} {dtype}")
    n = LENGTHS[lengths]
    s, g = scan_inputs(n, D, N, G, dtype, D * 17 + N)
    s["delta"] = (0.05 * s["delta"].float().abs()).to(DTYPE[dtype])
    s["delta_bias"] = 0.02 * s["delta_bias"].abs()
    dout, dnew = rand((sum(n), D), g, DTYPE[dtype]), rand((len(n), D, N), g)
    opt = {k: s[k] for k in ("skip", "z", "delta_bias", "state_in")}
    a = [s[k] for k in ("u", "delta", "A", "B", "C")]
    got = block.lbi_ssm_scan_backward(*a, dout, softplus=False, dstate_out=dnew, **opt, **packing(n))
    want = ref.scan_backward(s, n, dout, dnew, softplus=False)
    for k, e in want.items():
        check(got[k], e, k, want["delta"].norm().item() if k == "delta_bias" else None)


@pytest.mark.parametrize("lengths", ["one", "ragged", "long"])
@pytest.mark.parametrize("D", [1, 7, 64, 131])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nothing_is_written_beside_strided_outputs(lengths, D, dtype):
    say(f"[borders] {lengths} D={D} {dtype}")
    n, N, W, dt = LENGTHS[lengths], 6, 4, DTYPE[dtype]
    T = sum(n)
    s, g = scan_inputs(n, D, N, 1, dtype, D * 19)
    x, dout = rand((T, D), g, dt), rand((T, D), g, dt)
    w, b = rand((D, W), g, scale=0.6), rand((D,), g, scale=0.2)

    def out(cols=D):
        return wide_rows(torch.zeros(T, cols, dtype=dt, device=DEV), 9, g)
    o = out()
    assert torch.equal(block.lbi_ssm_conv(x, w, b, out=o, **packing(n)),
                       block.lbi_ssm_conv(x, w, b, **packing(n))) and untouched(o)
    o = out()
    assert torch.equal(block.lbi_ssm_conv_backward(x, w, dout, b, dx=o, **packing(n))[0],
                       block.lbi_ssm_conv_backward(x, w, dout, b, **packing(n))[0]) and untouched(o)
    o = out()
    assert torch.equal(call_scan(s, n, out=o), call_scan(s, n)) and untouched(o)
    o = {k: out(N if k in "BC" else D) for k in ("u", "delta", "z", "B", "C")}
    got = block.lbi_ssm_scan_backward(dout=dout, outputs=o, **s, **packing(n))
    want = block.lbi_ssm_scan_backward(dout=dout, **s, **packing(n))
    for k, t in o.items():
        assert torch.equal(got[k].reshape(-1), want[k].reshape(-1)) and untouched(t), k
    m = min(T, 5)
    o = out()[:m]
    state, last = rand((m, W - 1, D), g, dt), torch.empty(m, W - 1, D, dtype=dt, device=DEV)
    assert torch.equal(block.lbi_ssm_conv_step(x[:m], w, state, last, b, out=o),
                       block.lbi_ssm_conv_step(x[:m], w, state, last, b)) and untouched(o)
    o = out()[:m]
    one = [s[k] if k == "A" else s[k][:m] for k in ("u", "delta", "A", "B", "C")]
    state, last = rand((m, D, N), g), torch.empty(m, D, N, device=DEV)
    assert torch.equal(block.lbi_ssm_scan_step(*one, state, last, out=o),
                       block.lbi_ssm_scan_step(*one, state, last)) and untouched(o)


@pytest.mark.parametrize("lengths", [[3900], [1300, 0, 1, 2600, 77]], ids=str)
@pytest.mark.parametrize("D,N,G", [(6, 16, 2), (20, 40, 1)])
def test_bf16_scan_over_many_ranges(lengths, D, N, G):
    say(f"[many ranges] {lengths} D={D} N={N} bf16")
    s, g = scan_inputs(lengths, D, N, G, "bf16", sum(lengths) + N)
    T, S = sum(lengths), len(lengths)
    assert block.lbi_ssm_scan_workspace_bytes(T, S, D, N, G, "offsets" in packing(lengths)) \
        > 33 * 8 * D * N, "more ranges than one batch of the carry"
    new = torch.full((S, D, N), float("nan"), device=DEV)
    y = call_scan(s, lengths, state_out=new)
    want, want_new = ref.scan(s, lengths)
    check(y, want, "y")
    check(new, want_new, "state_out")
    dout, dnew = rand((T, D), g, torch.bfloat16), rand((S, D, N), g)
    got = block.lbi_ssm_scan_backward(dout=dout, dstate_out=dnew, **s, **packing(lengths))
    want = ref.scan_backward(s, lengths, dout, dnew)
    for k, e in want.items():
        check(got[k], e, k, want["delta"].norm().item() if k == "delta_bias" else None)
