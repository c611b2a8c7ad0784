"""Channels whose states grow (A > 0), or forget everything at each token (A = -inf), in scans that
are cut into ranges (needs a GPU).

Tolerances as in test_gpu_block.py: 1e-5 of the result's norm, each channel by itself here.
"""
import pytest
import torch

from oracle import block as ref
from paper_2605_09204_amd import block

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TOL = 1e-5


def close(got, want, label, dims):
    """Relative error over ``dims``, channel by channel."""
    got = got.detach().cpu().double().reshape(want.shape)
    assert torch.isfinite(got).all(), f"{label}: not finite"
    off = (got - want).square().sum(dims).sqrt()
    size = want.square().sum(dims).sqrt()
    assert (off <= TOL * size).all(), f"{label}: {(off / size).max():.3g}"


@pytest.mark.parametrize("T,step", [(2000, 0.2), (9000, 0.1), (700, 0.3), (1500, 3.0)])
@pytest.mark.parametrize("ragged", [False, True])
def test_states_that_grow(T, step, ragged):
    """exp(sum D_t A) over all tokens passes float32's range by far; inputs that begin late keep
    every state within it, and for the gradients no inputs and cotangents that end early."""
    D, N = 3, 5
    g = torch.Generator()
    g.manual_seed(T)

    def r(*shape):
        return torch.randn(shape, generator=g).to(DEV)
    A = torch.tensor([[1.0, 0.5, -1.0, 0.0, -3.0], [0.9, -0.1, 0.2, 1.0, 0.7],
                      [-1.0, -2.0, -3.0, -4.0, -5.0]]).to(DEV)
    delta = (step * (0.9 + 0.2 * torch.rand(T, D, generator=g))).to(DEV)
    live = int(30 / step)  # tokens that grow a state by e^30
    late, early = torch.arange(T) >= T - live, torch.arange(T) < live
    s = {"u": r(T, D) * late[:, None].to(DEV), "delta": delta, "A": A, "B": r(T, 1, N),
         "C": r(T, 1, N), "state_in": torch.zeros(1, D, N, device=DEV)}
    kw = {"offsets": torch.tensor([0, T], device=DEV)} if ragged else {"sequences": 1}
    assert block.lbi_ssm_scan_workspace_bytes(T, 1, D, N, 1, ragged) > 0, "not cut"
    print(f"[growth] T={T} step={step} ragged={ragged}", flush=True)
    last = torch.empty(1, D, N, device=DEV)
    y = block.lbi_ssm_scan(**s, softplus=False, state_out=last, **kw)
    want, want_last = ref.scan(s, [T], softplus=False)
    close(last, want_last, "state_out", (0, 2))
    close(y, want, "y", 0)
    if step > 1:
        return  # the gradient's ranges each stay below 2^127
    s["u"] = torch.zeros(T, D, device=DEV)
    dout = r(T, D) * early[:, None].to(DEV)
    got = block.lbi_ssm_scan_backward(**s, dout=dout, softplus=False, **kw)
    for k, t in got.items():
        assert t is None or torch.isfinite(t).all(), k
    s64 = {k: v[:live] if k not in ("A", "state_in") else v for k, v in s.items()}
    want = ref.scan_backward(s64, [live], dout[:live], softplus=False)  # later tokens have no part
    close(got["u"][:live], want["u"], "u", 0)
    assert (got["u"][live:] == 0).all()
    close(got["state_in"], want["state_in"], "state_in", (0, 2))

@pytest.mark.parametrize("n", [[3], [37, 5, 1, 8, 66], [1500]])
def test_states_that_forget(n):
    """A = -inf: h is the token's own part.  (Rows past a sequence's end change nothing.)"""
    D, N, T = 2, 3, sum(n)
    g = torch.Generator()
    g.manual_seed(T)

    def r(*shape):
        return torch.randn(shape, generator=g).to(DEV)
    A = torch.tensor([[-1.0, -float("inf"), -2.0], [-float("inf")] * 3]).to(DEV)
    s = {"u": r(T, D), "delta": r(T, D), "A": A, "B": r(T, 1, N), "C": r(T, 1, N),
         "state_in": r(len(n), D, N)}
    off = torch.tensor([0, *n]).cumsum(0).to(DEV)
    last = torch.empty(len(n), D, N, device=DEV)
    y = block.lbi_ssm_scan(**s, offsets=off, state_out=last)
    want, want_last = ref.scan(s, n)
    close(y, want, "y", 0)
    close(last, want_last, "state_out", (0, 2))
    step = torch.empty(len(n), D, N, device=DEV)
    one = {k: v[:len(n)] if k in ("u", "delta", "B", "C") else v for k, v in s.items() if k != "state_in"}
    y = block.lbi_ssm_scan_step(**one, state_in=s["state_in"], state_out=step)
    want, want_last = ref.scan({**one, "state_in": s["state_in"]}, [1] * len(n))
    close(y, want, "step y", 0)
    close(step, want_last, "step states", (0, 2))
