"""Linear attention in calls of training size: ranges of several tiles that pass states on, against the
definition in float64 for some of the heads, and a NaN in the middle of one (needs a GPU; what the
calls are cut into is held by test_linear_plans.py).  Tolerances are those of the parity tests, for
each head by itself.
"""
import pytest
import torch

from oracle import linear as ref
from paper_2605_09204_amd import linear
from test_gpu_linear import DTYPE, args_of, attention_inputs, check, packing, rand, say
from test_gpu_linear_decays import check_decays, decay_terms
from test_linear_plans import BF16, F32, PACKED, RANGES, attention_plan

pytestmark = pytest.mark.gpu


def some_heads(s, dout, dnew, heads, keys):
    """The problem with these heads alone (and the keys that they share)."""
    t = {"q": s["q"][:, heads], "k": s["k"][:, keys], "v": s["v"][:, keys],
         "log_decay": s["log_decay"][heads], "state": s["state"][:, heads]}
    return t, dout[:, heads], dnew[:, heads]


@pytest.mark.parametrize("lengths,H,KH,DK,DV", RANGES, ids=str)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_of_training_size(lengths, H, KH, DK, DV, dtype):
    label = f"[ranges] {lengths} H={H} KH={KH} DK={DK} DV={DV} {dtype}"
    say(label)
    s, g = attention_inputs(lengths, H, KH, DK, DV, dtype, DK * 7 + DV)
    dout, dnew = rand((sum(lengths), H, DV), g, DTYPE[dtype]), rand(s["state"].shape, g)
    scale, bf16, share = DK ** -0.5, dtype == "bf16", H // KH
    state = s["state"].clone()
    out = linear.lbi_linear_attention(*args_of(s), state_in=state, state_out=state, **packing(lengths))
    grads = linear.lbi_linear_attention_backward(*args_of(s), dout, state_in=s["state"],
                                                 dstate_out=dnew, **packing(lengths))
    other = torch.empty_like(state)
    assert torch.equal(out, linear.lbi_linear_attention(*args_of(s), state_in=s["state"],
                                                        state_out=other, **packing(lengths)))
    assert torch.equal(state, other)
    bare = linear.lbi_linear_attention_backward(*args_of(s), dout, **packing(lengths))
    keys = [0, KH - 1]
    heads = [kh * share + i for kh in keys for i in range(share)]
    t, dt, gt = some_heads(s, dout, dnew, heads, keys)
    terms = ref.attention_terms(*args_of(t), scale, lengths, dt)
    want, want_new = ref.attention(*args_of(t), scale, lengths, t["state"])
    for j, h in enumerate(heads):
        check(out[:, h], want[:, j], f"out of head {h}", terms["out"][:, j] if bf16 else None,
              terms["out"][:, j].norm().item())
        check(state[:, h], want_new[:, j], f"state of head {h}")
    say("  forward")
    tokens = 64 * attention_plan(lengths, H, KH, DK, DV, BF16 if bf16 else F32, True)[0]
    for got, first, last in ((grads, t["state"], gt), (bare, None, None)):
        want = ref.attention_backward(*args_of(t), scale, lengths, dt, first, last)
        for k, of in (("q", heads), ("k", keys), ("v", keys)):
            for j, h in enumerate(of):
                check(got[k][:, h], want[k][:, j], f"{k} of head {h}", terms[k][:, j] if bf16 else None,
                      terms[k][:, j].norm().item())
        if first is not None:
            for j, h in enumerate(heads):
                check(got["state_in"][:, h], want["state_in"][:, j], f"state_in of head {h}",
                      floor=scale * dt[:, j].float().norm().item())
        zero = torch.zeros_like(t["state"])
        check_decays(got["log_decay"][heads], want["log_decay"],
                     decay_terms(dict(t, state=zero if first is None else first), scale, lengths, dt,
                                 zero if last is None else last), DK, DV, tokens, label)


@pytest.mark.parametrize("which", ["q", "k", "v", "dout"])
@pytest.mark.parametrize("H,DK,DV,dtype", [(66, 64, 64, "bf16"), (66, 64, 64, "f32"),
                                           (48, 48, 101, "bf16"), (24, 128, 128, "f32")])
def test_a_nan_between_ranges(H, DK, DV, dtype, which):
    """One NaN in a sequence that lasts over several ranges, in a tile that is not its range's first:
    other heads and sequences keep their bits, and what may not see it its values."""
    say(f"[ranges] NaN in {which}, H={H} DK={DK} DV={DV} {dtype}")
    tiles = attention_plan(PACKED, H, H, DK, DV, BF16 if dtype == "bf16" else F32, True)[0]
    assert tiles >= 3
    s, g = attention_inputs(PACKED, H, H, DK, DV, dtype, 6)
    x = dict(s, dout=rand((sum(PACKED), H, DV), g, DTYPE[dtype]))
    begin, end, h = 301, 1504, H - 1
    at = (700 // (64 * tiles) + 1) * 64 * tiles + 64 + 40  # in the second tile of a range

    def run(x):
        state = x["state"].clone()
        out = linear.lbi_linear_attention(*args_of(x), state_in=state, state_out=state, **packing(PACKED))
        return out, state, linear.lbi_linear_attention_backward(
            *args_of(x), x["dout"], state_in=x["state"], **packing(PACKED))
    out, state, grad = run(x)
    bad = dict(x, **{which: x[which].clone()})
    bad[which][at, h, 5] = float("nan")
    out2, state2, grad2 = run(bad)

    def same(a, b):
        assert torch.isfinite(b).all()
        a, b = a.float(), b.float()
        # taken token by token the sums are rounded elsewhere
        assert (a - b).norm() <= (2.0 ** -6 if dtype == "bf16" else 2e-5) * a.norm()
    assert torch.equal(state[:, :h], state2[:, :h]) and torch.equal(state[[0, 1, 2, 4]], state2[[0, 1, 2, 4]])
    for a, b in ((out, out2), *((grad[k], grad2[k]) for k in ("q", "k", "v"))):
        assert torch.equal(a[:, :h], b[:, :h])
        assert torch.equal(a[:begin], b[:begin]) and torch.equal(a[end:], b[end:])
    assert torch.equal(grad["log_decay"][:h], grad2["log_decay"][:h])
    before, behind = slice(begin, at), slice(at + 1, end)
    seen = torch.isnan(out2[:, h]).any(1)
    if which == "dout":
        assert torch.equal(out, out2) and torch.equal(state, state2)
        same(grad["q"][before, h], grad2["q"][before, h])
        assert torch.isnan(grad2["q"][at, h]).all()
        for k in ("q", "k", "v"):
            same(grad[k][behind, h], grad2[k][behind, h])
        for k in ("k", "v"):  # dout of a token reaches the tokens before it
            assert torch.isnan(grad2[k][before, h]).any(1).all()
        return
    same(out[before, h], out2[before, h])
    if which == "q":
        assert int(seen.sum()) == 1 and seen[at]
        same(out[behind, h], out2[behind, h])
        same(state[3, h], state2[3, h])
        same(grad["q"][before, h], grad2["q"][before, h])
        same(grad["q"][behind, h], grad2["q"][behind, h])
        for k in ("k", "v"):
            same(grad[k][behind, h], grad2[k][behind, h])
    else:
        assert seen[at:end].all() and torch.isnan(state2[3, h]).any()
        same(grad["q"][before, h], grad2["q"][before, h])
