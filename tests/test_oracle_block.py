"""Pins of the float64 definitions in oracle/block.py that share nothing with them: closed forms,
brute-force sums, and gradients against central differences (CPU)."""
import math

import pytest
import torch

from oracle import block as ref


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def test_norm_closed_forms():
    out, s = ref.rms_norm(torch.tensor([[3.0, 4.0]]), torch.ones(2), eps=0.0)
    assert torch.allclose(out, torch.tensor([[3.0, 4.0]]).double() / math.sqrt(12.5))
    out, s = ref.rms_norm(torch.tensor([[1.0, 1.0]]), torch.tensor([2.0, 0.5]),
                          torch.tensor([[6.0, 6.0]]), eps=0.0)
    assert torch.allclose(s, torch.full((1, 2), 7.0, dtype=torch.float64))
    assert torch.allclose(out, torch.tensor([[2.0, 0.5]], dtype=torch.float64))


def test_q8_scales():
    y = torch.tensor([[0.0, 0.0, 4.48, -8.96]], dtype=torch.float64)
    assert ref.q8_scales(y, 2, "e4m3").tolist() == [[1.0, pytest.approx(0.02)]]
    assert ref.q8_scales(y, 0, "int8").tolist() == [[pytest.approx(8.96 / 127)]]


def test_conv_is_the_direct_sum():
    g = gen(1)
    n = [4, 0, 1]
    x, w = torch.randn(5, 3, generator=g), torch.randn(3, 3, generator=g)
    old = torch.randn(3, 2, 3, generator=g)
    y, new = ref.conv(x, w, None, old, n, silu=False)
    tape = torch.cat([old[0], x[:4]]).double()
    want = [sum(w[:, k].double() * tape[t + k] for k in range(3)) for t in range(4)]
    assert torch.allclose(y[:4], torch.stack(want))
    assert torch.equal(new[0], x[2:4].double()) and torch.equal(new[1], old[1].double())
    assert torch.equal(new[2], torch.stack([old[2, 1], x[4]]).double())


def scan_case(g, n=(5, 0, 3), D=2, N=3, G=2):
    T, B = sum(n), len(n)
    r = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    return {"u": r(T, D), "delta": r(T, D), "A": -torch.exp(r(D, N)), "B": r(T, G, N),
            "C": r(T, G, N), "skip": r(D), "z": r(T, D), "delta_bias": r(D),
            "state_in": r(B, D, N)}


def test_scan_closed_form():
    """h_t as the sum over s <= t of the decays between, token by token of nothing kept."""
    s = scan_case(gen(2), n=(4,))
    y, new = ref.scan(s, [4])
    d = torch.log1p(torch.exp(s["delta"] + s["delta_bias"]))
    for ch in range(2):
        for t in range(4):
            total = 0.0
            for k in range(3):
                h = s["state_in"][0, ch, k] * math.exp(s["A"][ch, k] * d[:t + 1, ch].sum())
                for q in range(t + 1):
                    h = h + d[q, ch] * s["u"][q, ch] * s["B"][q, ch, k] * \
                        math.exp(s["A"][ch, k] * d[q + 1:t + 1, ch].sum())
                total = total + s["C"][t, ch, k] * h
                if t == 3:
                    assert abs(new[0, ch, k] - h) < 1e-12
            z = s["z"][t, ch]
            want = (total + s["skip"][ch] * s["u"][t, ch]) * z / (1 + math.exp(-z))
            assert abs(y[t, ch] - want) < 1e-12


def differences(f, inputs, grads, h=1e-6, tol=1e-7):
    """Central differences of the scalar f() in every entry of the inputs."""
    for k, t in inputs.items():
        flat, want = t.view(-1), grads[k].reshape(-1)
        for i in range(flat.numel()):
            keep = flat[i].item()
            flat[i] = keep + h
            up = f()
            flat[i] = keep - h
            down = f()
            flat[i] = keep
            assert abs((up - down) / (2 * h) - want[i]) < tol * (1 + abs(want[i])), (k, i)


def test_gradients_against_differences():
    g = gen(3)
    n = [5, 0, 3]
    s = scan_case(g, n)
    dy, dn = torch.randn(8, 2, generator=g).double(), torch.randn(3, 2, 3, generator=g).double()

    def loss():
        y, new = ref.scan(s, n)
        return ((y * dy).sum() + (new * dn).sum()).item()
    differences(loss, s, ref.scan_backward(s, n, dy, dn))

    v = {"x": torch.randn(8, 2, generator=g).double(), "w": torch.randn(2, 3, generator=g).double(),
         "b": torch.randn(2, generator=g).double(), "old": torch.randn(3, 2, 2, generator=g).double()}
    dn = torch.randn(3, 2, 2, generator=g).double()

    def conv_loss():
        y, new = ref.conv(v["x"], v["w"], v["b"], v["old"], n)
        return ((y * dy).sum() + (new * dn).sum()).item()
    got = ref.conv_backward(v["x"], v["w"], v["b"], v["old"], n, dy, dn)
    differences(conv_loss, v, dict(zip(("x", "w", "b", "old"), got)))

    v = {"s": torch.randn(3, 5, generator=g).double(), "w": torch.randn(5, generator=g).double()}
    do = torch.randn(3, 5, generator=g).double()
    got = ref.rms_norm_backward(do, v["s"], v["w"])
    differences(lambda: (ref.rms_norm(v["s"], v["w"])[0] * do).sum().item(), v,
                {"s": got[0], "w": got[1]})


@pytest.mark.parametrize("mistake", ["state dropped", "one token late", "no skip"])
def test_planted_mistakes_are_seen(mistake):
    """The closed form tells the definition from forms that are wrong by one thing."""
    s = scan_case(gen(4), n=(4,))
    y, _ = ref.scan(s, [4])
    wrong = dict(s)
    if mistake == "state dropped":
        wrong["state_in"] = torch.zeros_like(s["state_in"])
    elif mistake == "one token late":
        wrong["B"] = s["B"].roll(1, 0)
    else:
        wrong["skip"] = None
    assert (ref.scan(wrong, [4])[0] - y).abs().max() > 1e-3
