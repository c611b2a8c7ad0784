"""Region block calls of more than 2^24 workgroups, whose work items a single launch cannot number
(needs a GPU, and up to 80 GB of its memory)."""
import pytest
import torch

from paper_2605_09204_amd import block

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def say(msg):
    print(msg, flush=True)


def halves(T, cut):
    return slice(0, cut), slice(cut, T)


@pytest.fixture(autouse=True)
def memory():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def test_scan_of_many_single_tokens():
    """Each sequence takes a workgroup; two calls of half as many stay below the limit."""
    T = (1 << 24) + 77
    g = torch.Generator(device=DEV)
    g.manual_seed(31)

    def r(*shape):
        return torch.randn(shape, generator=g, device=DEV)
    s = {"u": r(T, 1), "delta": r(T, 1), "B": r(T, 1), "C": r(T, 1), "z": r(T, 1),
         "state_in": r(T, 1, 1)}
    p = {"A": -torch.ones(1, 1, device=DEV), "skip": torch.ones(1, device=DEV)}
    dout, dlast = r(T, 1), r(T, 1, 1)
    last = torch.full((T, 1, 1), float("nan"), device=DEV)
    say(f"[large] scan of {T} sequences")
    y = block.lbi_ssm_scan(**s, **p, sequences=T, state_out=last,
                           out=torch.full((T, 1), float("nan"), device=DEV))
    # h = exp(-softplus(delta)) h_0 + softplus(delta) u B
    d = torch.nn.functional.softplus(s["delta"].double())
    h = torch.exp(-d) * s["state_in"].double()[:, 0] + d * s["u"].double() * s["B"].double()
    assert (last[:, 0].double() - h).norm() <= 1e-6 * h.norm()
    want = (h * s["C"] + s["u"]) * s["z"].double() * torch.sigmoid(s["z"].double())
    assert (y.double() - want).norm() <= 1e-6 * want.norm()
    say("[large] its gradient")
    got = block.lbi_ssm_scan_backward(**s, **p, dout=dout, dstate_out=dlast, sequences=T)
    for part in halves(T, T // 2):
        few = {k: t[part] for k, t in s.items()}
        n = few["u"].shape[0]
        for k, t in block.lbi_ssm_scan_backward(**few, **p, dout=dout[part], dstate_out=dlast[part],
                                                sequences=n).items():
            if k in s:
                assert torch.equal(got[k][part], t), k
    torch.cuda.synchronize()


def test_sums_of_many_values_of_B():
    """2^32 values of dB and more, a thread each."""
    L, N = 64, 64
    S = (1 << 20) + 2
    T = S * L
    g = torch.Generator(device=DEV)
    g.manual_seed(32)

    def r(*shape):
        return torch.randn(shape, generator=g, device=DEV, dtype=torch.bfloat16)
    s = {"u": r(T, 1), "delta": r(T, 1), "B": r(T, N), "C": r(T, N)}
    A = -torch.arange(1, N + 1, device=DEV).float()[None]
    dout = r(T, 1)
    say(f"[large] {T * N} values of dB")
    got = block.lbi_ssm_scan_backward(**s, A=A, dout=dout, sequences=S)
    for part in (slice(0, 3 * L), slice(S // 2 * L, (S // 2 + 3) * L), slice(T - 3 * L, T)):
        few = block.lbi_ssm_scan_backward(**{k: t[part] for k, t in s.items()}, A=A, dout=dout[part],
                                          sequences=3)
        for k in s:
            assert torch.equal(got[k][part], few[k]), k
    torch.cuda.synchronize()


@pytest.mark.parametrize("in_place", [False, True])
def test_states_of_many_empty_sequences(in_place):
    """The convolution hands them on, four sequences and 128 channels a workgroup."""
    B, D, W = (1 << 22) + 5, 2048, 2
    old = torch.empty(B, 1, D, dtype=torch.int16, device=DEV)
    flat = old.view(-1)
    for at in range(0, flat.numel(), 1 << 28):
        n = min(1 << 28, flat.numel() - at)
        flat[at:at + n] = torch.arange(at, at + n, device=DEV).remainder_(30011).to(torch.int16)
    x = torch.empty(0, D, dtype=torch.bfloat16, device=DEV)
    off = torch.zeros(B + 1, dtype=torch.int64, device=DEV)
    w = torch.ones(D, W, device=DEV)
    new = old.clone() if in_place else torch.zeros_like(old)
    as_bf16 = old.view(torch.bfloat16)
    say(f"[large] states of {B} sequences, in place: {in_place}")
    block.lbi_ssm_conv(x, w, offsets=off, state_in=new.view(torch.bfloat16) if in_place else as_bf16,
                       state_out=new.view(torch.bfloat16))
    assert torch.equal(new, old)
    if not in_place:
        del new
        got = block.lbi_ssm_conv_backward(x, w, x, offsets=off, state_in=as_bf16, dstate_out=as_bf16)
        assert torch.equal(got[3].view(torch.int16), old)
    torch.cuda.synchronize()


def test_conv_step_of_many_tokens():
    """A workgroup takes 256 vectors of eight channels: one vector a token here."""
    n = (1 << 32) + 300
    x = torch.empty(n, 1, dtype=torch.bfloat16, device=DEV)
    x[:] = 1.0
    x[-300:] = 2.0
    w = torch.tensor([[3.0, 5.0]], device=DEV)
    state = torch.ones(n, 1, 1, dtype=torch.bfloat16, device=DEV)
    say(f"[large] step of {n} tokens")
    y = block.lbi_ssm_conv_step(x, w, state, state, silu=False)
    assert (y[:-300] == 8.0).all() and (y[-300:] == 13.0).all()
    assert (state[:-300] == 1.0).all() and (state[-300:] == 2.0).all()
    torch.cuda.synchronize()
