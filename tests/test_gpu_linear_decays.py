"""The gradients of linear attention's decays, head by head (needs a GPU).

A decay's gradient is a sum over pairs of tokens, and over states, of products of two inner products;
its error is held to the root sum of squares of that head's own terms, ``decay_terms``.  Each is off
by what an inner product of DK or DV float32 products is, 2^-24 sqrt(DK) and 2^-24 sqrt(DV) of it, by
its power of the decay, 8 2^-24 (the exponent, up to 10 where it is not negligible, is rounded before
the power is), and together they are added up along a lane, each addition rounding what is there by
2^-24, a random walk over as many as a range has tokens (times DK / 64).
"""
import pytest
import torch

from oracle import linear as ref
from paper_2605_09204_amd import linear
from test_gpu_linear import DTYPE, HEADS, LENGTHS, args_of, attention_inputs, packing, rand, say
from test_linear_plans import BF16, F32, attention_plan

pytestmark = pytest.mark.gpu


def decay_terms(s, scale, lengths, dout, dnew):
    """For each head the root sum of squares of its decay's gradient's terms, as values and as inner
    products of independent terms."""
    q, k, v, S, d, G = (t.detach().cpu().double()
                        for t in (s["q"], s["k"], s["v"], s["state"], dout, dnew))
    H, share = q.shape[1], q.shape[1] // k.shape[1]
    total = torch.zeros(H, dtype=torch.float64)
    at = 0
    for b, n in enumerate(lengths):
        rows = slice(at, at + n)
        at += n
        i = torch.arange(n, dtype=torch.float64)
        lag = (i[:, None] - i).clamp(min=0)
        for h in range(H):
            la = s["log_decay"][h].item()
            Q, K, V, D = q[rows, h], k[rows, h // share], v[rows, h // share], d[rows, h]
            first, last = S[b, h], G[b, h]
            w = (lag * torch.exp(lag * la) * scale) ** 2
            total[h] += (w * ((Q @ K.T) ** 2 * (D @ V.T) ** 2
                              + ((Q * Q) @ (K * K).T) * ((D * D) @ (V * V).T))).sum()
            w = ((i + 1) * torch.exp((i + 1) * la) * scale) ** 2
            total[h] += (w * ((Q @ first * D).sum(1) ** 2 + ((Q * Q) @ (first * first) * D * D).sum(1))).sum()
            w = ((n - 1 - i) * torch.exp((n - 1 - i) * la)) ** 2
            total[h] += (w * ((K @ last * V).sum(1) ** 2 + ((K * K) @ (last * last) * V * V).sum(1))).sum()
            w = n * torch.exp(torch.tensor(n * la, dtype=torch.float64))
            total[h] += w ** 2 * ((first * last).sum() ** 2 + (first * last).square().sum())
    return total.sqrt()


def check_decays(got, want, terms, DK, DV, tokens, label):
    steps = 8 + DK ** 0.5 + DV ** 0.5 + (tokens * max(DK, 64) / 64) ** 0.5
    err = (got.cpu().double() - want).abs()
    worst = (err / (terms + 1e-300)).max().item()
    say(f"{label}: decays off by up to {worst:.2g} of their terms (bound {steps * 2.0 ** -24:.2g})")
    assert (err <= steps * 2.0 ** -24 * terms).all(), (err / terms).tolist()


@pytest.mark.parametrize("lengths", sorted(LENGTHS))
@pytest.mark.parametrize("H,KH,DK,DV", HEADS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_decay_gradients_head_by_head(lengths, H, KH, DK, DV, dtype):
    label = f"[decays] {lengths} H={H} KH={KH} DK={DK} DV={DV} {dtype}"
    n = LENGTHS[lengths]
    s, g = attention_inputs(n, H, KH, DK, DV, dtype, DK * 17 + DV)
    dout, dnew = rand((sum(n), H, DV), g, DTYPE[dtype]), rand(s["state"].shape, g)
    scale = DK ** -0.5
    got = linear.lbi_linear_attention_backward(*args_of(s), dout, state_in=s["state"],
                                               dstate_out=dnew, **packing(n))
    want = ref.attention_backward(*args_of(s), scale, n, dout, s["state"], dnew)
    tokens = 64 * attention_plan(n, H, KH, DK, DV, BF16 if dtype == "bf16" else F32, True)[0]
    check_decays(got["log_decay"], want["log_decay"], decay_terms(s, scale, n, dout, dnew), DK, DV,
                 min(tokens, max(n)), label)
