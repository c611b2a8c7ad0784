"""Pins of the float64 definitions in oracle/linear.py that share nothing with them: closed forms,
sums over all pairs of tokens, and gradients against central differences (CPU)."""
import math

import pytest
import torch

from oracle import linear as ref

F64 = torch.float64


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def r(g, *shape):
    return torch.randn(shape, generator=g, dtype=F64)


def test_layer_norm_closed_forms():
    out, s = ref.layer_norm(torch.tensor([[1.0, 3.0]]), eps=0.0)
    assert torch.allclose(out, torch.tensor([[-1.0, 1.0]], dtype=F64))
    out, s = ref.layer_norm(torch.tensor([[1.0, 2.0, 6.0]]), torch.tensor([1.0, 2.0, 3.0]),
                            torch.tensor([0.5, 0.0, 0.0]), torch.tensor([[1.0, 2.0, 0.0]]), eps=2.0)
    root = math.sqrt(8.0 / 3 + 2)  # s = 2, 4, 6
    assert torch.allclose(out, torch.tensor([[-2 / root + 0.5, 0.0, 6 / root]], dtype=F64))
    assert torch.equal(s, torch.tensor([[2.0, 4.0, 6.0]], dtype=F64))


def test_activations():
    z = torch.tensor([-3.0, 0.0, 1.0], dtype=F64)
    assert torch.allclose(ref.activation("silu", z), torch.tensor(
        [-3 / (1 + math.e ** 3), 0.0, 1 / (1 + 1 / math.e)], dtype=F64))
    normal = [0.5 * math.erfc(-x / math.sqrt(2)) for x in z.tolist()]
    assert torch.allclose(ref.activation("gelu", z), z * torch.tensor(normal, dtype=F64))
    for act in ("silu", "gelu", "none"):
        d = (ref.activation(act, z + 1e-6) - ref.activation(act, z - 1e-6)) / 2e-6
        assert torch.allclose(ref.slope(act, z), d, atol=1e-8)


def test_projection_is_the_sum():
    g = gen(1)
    x, w, b, res = r(g, 2, 3), r(g, 4, 3), r(g, 4), r(g, 2, 4)
    out, pre = ref.projection(x, w, b, "silu", res)
    for t in range(2):
        for n in range(4):
            z = sum(x[t, k].item() * w[n, k].item() for k in range(3)) + b[n].item()
            assert math.isclose(pre[t, n].item(), z, rel_tol=1e-12)
            assert math.isclose(out[t, n].item(), z / (1 + math.exp(-z)) + res[t, n].item(),
                                rel_tol=1e-12)


def attention_case(g, n=(5, 0, 3), H=4, KH=2, DK=2, DV=3):
    T, B = sum(n), len(n)
    return {"q": r(g, T, H, DK), "k": r(g, T, KH, DK), "v": r(g, T, KH, DV),
            "log_decay": -torch.exp(r(g, H)), "scale": 0.7, "lengths": list(n),
            "state": r(g, B, H, DK, DV)}


def test_attention_is_the_sum_over_pairs():
    s = attention_case(gen(2))
    out, new = ref.attention(**s)
    begin = 0
    for b, n in enumerate(s["lengths"]):
        for h in range(4):
            a = math.exp(s["log_decay"][h])
            for i in range(n):
                want = s["scale"] * a ** (i + 1) * (s["q"][begin + i, h] @ s["state"][b, h])
                for j in range(i + 1):
                    p = s["q"][begin + i, h] @ s["k"][begin + j, h // 2]
                    want = want + s["scale"] * a ** (i - j) * p * s["v"][begin + j, h // 2]
                assert torch.allclose(out[begin + i, h], want)
            last = a ** n * s["state"][b, h]
            for j in range(n):
                last = last + a ** (n - 1 - j) * torch.outer(s["k"][begin + j, h // 2],
                                                             s["v"][begin + j, h // 2])
            assert torch.allclose(new[b, h], last)
        begin += n
    assert torch.equal(new[1], s["state"][1])


def test_attention_limits():
    s = attention_case(gen(3), n=(4,))
    s["log_decay"] = torch.tensor([0.0, -math.inf, 0.0, -math.inf], dtype=F64)
    out, new = ref.attention(**s)
    kv = torch.einsum("thd,the->hde", s["k"], s["v"])
    assert torch.allclose(new[0, 0], s["state"][0, 0] + kv[0])  # never fades
    own = (s["q"][3, 1] @ s["k"][3, 0]) * s["v"][3, 0] * s["scale"]
    assert torch.allclose(out[3, 1], own)  # sees itself only


@pytest.mark.parametrize("name", ["q", "k", "v", "log_decay", "state_in"])
def test_attention_gradients_against_differences(name):
    g = gen(4)
    s = attention_case(g)
    dout, dstate = r(g, 8, 4, 3), r(g, *s["state"].shape)
    want = ref.attention_backward(**s, dout=dout, dstate=dstate)[name]
    key = "state" if name == "state_in" else name
    d = r(g, *s[key].shape)

    def loss(e):
        out, new = ref.attention(**{**s, key: s[key] + e * d})
        return ((out * dout).sum() + (new * dstate).sum()).item()
    e = 1e-6
    assert math.isclose((loss(e) - loss(-e)) / (2 * e), (want * d).sum().item(), rel_tol=1e-6)


def test_terms_are_those_of_the_sums():
    g = gen(5)
    s = attention_case(g, n=(3,), H=1, KH=1)
    del s["state"]
    dout = r(g, 3, 1, 3)
    t = ref.attention_terms(**s, dout=dout)
    a, c = math.exp(s["log_decay"][0]), s["scale"]
    q, k, v, d = (x[:, 0] for x in (s["q"], s["k"], s["v"], dout))
    p = [[c * a ** (i - j) * (q[i] @ k[j]).item() if j <= i else 0.0 for j in range(3)]
         for i in range(3)]
    e = [[c * a ** (i - j) * (d[i] @ v[j]).item() if j <= i else 0.0 for j in range(3)]
         for i in range(3)]
    for i in range(3):
        assert torch.allclose(t["out"][i, 0], sum((p[i][j] * v[j]) ** 2 for j in range(3)).sqrt())
        assert torch.allclose(t["q"][i, 0], sum((e[i][j] * k[j]) ** 2 for j in range(3)).sqrt())
        assert torch.allclose(t["k"][i, 0], sum((e[j][i] * q[j]) ** 2 for j in range(3)).sqrt())
        assert torch.allclose(t["v"][i, 0], sum((p[j][i] * d[j]) ** 2 for j in range(3)).sqrt())
