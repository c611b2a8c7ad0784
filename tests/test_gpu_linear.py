"""Parity of the operators in include/lbi_linear.h with their definitions in float64
(oracle/linear.py), through the C-ABI (needs a GPU).

Tolerances, from the arithmetic: relative Frobenius error.  Sums and states are float32: 1e-5 bounds
what their roundings of 2^-24 come to, as for the library's other float32 results; with bf16 tokens a
state, or its gradient, enters the products as two bf16 values that leave at most 2^-16 of it, a
rounding that is random over the 16 and more values of a head, so 1e-5 holds there too.  A bf16 output adds one rounding of at most 2^-8
relative to each element.  Where float32 values are rounded to bf16 as operands of a product (p_ij,
e_ij, dz), each term of its sums has an independent error of at most 2^-8 of itself: together at
most 2^-8 times the root sum of the terms' squares, which ``terms`` gives.
"""
import sys

import pytest
import torch

from oracle import linear as ref
from paper_2605_09204_amd import linear

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
ACT = {"none": linear.LBI_ACT_NONE, "silu": linear.LBI_ACT_SILU, "gelu": linear.LBI_ACT_GELU}
F32_TOL = 1e-5
HALF_STEP = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}


def say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def check(got, want, label, terms=None, floor=0.0):
    """``terms``: root sums of squares of what was rounded to bf16 inside; ``floor``: the norm of
    what was summed, where that cancels."""
    assert got is not None, label
    got64 = got.detach().cpu().double().reshape(want.shape)
    if want.numel() == 0:
        return
    assert torch.isfinite(got64).all(), f"{label}: not finite"
    size = want.norm().item()
    bound = F32_TOL * max(size, floor) + HALF_STEP[got.dtype] * size
    if terms is not None:
        bound += 2.0 ** -8 * terms.norm().item() + F32_TOL * terms.norm().item()
    err = (got64 - want).norm().item()
    assert err <= bound, f"{label}: error {err:.3g} above {bound:.3g} (norm {size:.3g})"


def rand(shape, gen, dtype=torch.float32, scale=1.0):
    return (scale * torch.randn(shape, generator=gen)).to(dtype).to(DEV)


def gen_num(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def wide_rows(t, extra):
    """The same values as a slice of wider rows, from an odd element on; the rest is NaN."""
    flat = t.flatten(1) if t.dim() > 2 else t
    full = torch.full((flat.shape[0], flat.shape[1] + extra), float("nan"), dtype=t.dtype,
                      device=t.device)
    view = full[:, extra // 2:extra // 2 + flat.shape[1]]
    view.copy_(flat)
    return view.unflatten(1, t.shape[1:]) if t.dim() > 2 else view


def beside(view):
    """What lies beside the slice in its rows."""
    base = view._base if view._base is not None else view
    while base._base is not None:
        base = base._base
    at, width = view.storage_offset(), view[0].numel()
    return torch.cat([base[:, :at].flatten(), base[:, at + width:].flatten()])


# ---- layer norm --------------------------------------------------------------

NORM_SHAPES = [(1, 1), (3, 7), (5, 64), (130, 100), (17, 129), (9, 768), (1100, 520), (1030, 1111),
               (4, 1000), (1, 2048), (1025, 2040), (7, 4100), (3, 8192), (2, 8200), (5, 16383)]


@pytest.mark.parametrize("T,D", NORM_SHAPES)
@pytest.mark.parametrize("dtype,stream", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"),
                                          ("f32", "bf16")])
def test_layer_norm(T, D, dtype, stream):
    say(f"[layer_norm] T={T} D={D} {dtype} {stream}")
    g = gen_num(T * 31 + D)
    x = rand((T, D), g, DTYPE[dtype])
    w, b = 1.0 + rand((D,), g, scale=0.2), rand((D,), g)
    res = rand((T, D), g, DTYPE[stream], 2.0)
    out, total = linear.lbi_layer_norm(x, w, b, res)
    want, s = ref.layer_norm(x, w, b, res)
    check(out, want, "out")
    check(total, s, "residual_out")
    out, total = linear.lbi_layer_norm(x)
    assert total is None
    check(out, ref.layer_norm(x)[0], "out, bare", floor=T ** 0.5)
    check(linear.lbi_layer_norm(x, bias=b)[0], ref.layer_norm(x, bias=b)[0], "bias alone")
    # strided rows, in place on the residual
    xs, rs = wide_rows(x, 5), wide_rows(res, 3)
    outs = wide_rows(torch.zeros_like(x), 9)
    linear.lbi_layer_norm(xs, w, b, rs, out=outs, residual_out=rs)
    check(outs, want, "strided out")
    check(rs, s, "residual in place")
    assert torch.isnan(beside(outs)).all() and torch.isnan(beside(rs)).all()


@pytest.mark.parametrize("T,D", NORM_SHAPES + [(0, 33), (3000, 16), (2500, 768)])
@pytest.mark.parametrize("dtype,stream", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"),
                                          ("f32", "bf16")])
def test_layer_norm_backward(T, D, dtype, stream):
    say(f"[layer_norm_backward] T={T} D={D} {dtype} {stream}")
    g = gen_num(T * 41 + D)
    s = rand((T, D), g, DTYPE[stream], 2.0)
    w = 1.0 + rand((D,), g, scale=0.2)
    dout = rand((T, D), g, DTYPE[dtype])
    dres = rand((T, D), g, DTYPE[stream])
    for weight, extra in ((w, dres), (None, None)):
        ds, dw, db = linear.lbi_layer_norm_backward(dout, s, weight, extra)
        want, want_w, want_b = ref.layer_norm_backward(dout, s, weight, extra)
        # the terms of ds are as large as dout over the row's deviation (one feature: 1 / sqrt(eps))
        d = s.double().cpu()
        root = torch.sqrt((d - d.mean(-1, keepdim=True)).square().mean(-1, keepdim=True) + 1e-5)
        check(ds, want, "ds", floor=(dout.double().cpu() / root).norm().item())
        check(dw, want_w, "dweight", floor=dout.float().norm().item())
        check(db, want_b, "dbias", floor=dout.float().norm().item())
    outs, drs = wide_rows(torch.zeros_like(s), 5), wide_rows(dres, 7)
    if T > 0:
        linear.lbi_layer_norm_backward(wide_rows(dout, 3), wide_rows(s, 9), w, drs, ds=outs)
        a = linear.lbi_layer_norm_backward(dout, s, w, dres)
        assert torch.equal(outs, a[0]) and torch.isnan(beside(outs)).all()
        again = linear.lbi_layer_norm_backward(dout, s, w, drs, ds=drs)  # in place
        assert all(torch.equal(p, q) for p, q in zip(a, again))


def test_layer_norm_far_from_zero():
    """A mean 1000 times the deviation: what its rounding leaves is taken off again."""
    g = gen_num(3)
    x = 1000.0 + rand((64, 777), g)
    out, _ = linear.lbi_layer_norm(x)
    check(out, ref.layer_norm(x)[0], "out")
    dout = rand((64, 777), g)
    ds, dw, _ = linear.lbi_layer_norm_backward(dout, x)
    want, want_w, _ = ref.layer_norm_backward(dout, x)
    check(ds, want, "ds")
    check(dw, want_w, "dweight")


def test_layer_norm_odd_rows():
    """Equal values give the bias; a NaN or an infinity stays in its row."""
    x = torch.randn(6, 300, device=DEV)
    x[1] = 3.5
    x[3, 7] = float("nan")
    x[4, 299] = float("inf")
    b = torch.randn(300, device=DEV)
    out, _ = linear.lbi_layer_norm(x, None, b)
    assert torch.allclose(out[1], b, atol=1e-4)
    assert torch.isnan(out[3]).all() and torch.isnan(out[4]).all()
    rows = [0, 1, 2, 5]
    check(out[rows], ref.layer_norm(x[rows], None, b)[0], "the others", floor=(4 * 300) ** 0.5)


# ---- projection --------------------------------------------------------------

PRODUCTS = [(1, 1, 1), (1, 768, 96), (3, 17, 5), (64, 64, 64), (65, 63, 129), (7, 2000, 40),
            (130, 100, 300), (257, 130, 72), (1000, 257, 136), (300, 1000, 513), (2100, 96, 1030)]


@pytest.mark.parametrize("T,K,N", PRODUCTS)
@pytest.mark.parametrize("dtype,stream", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"),
                                          ("f32", "bf16")])
@pytest.mark.parametrize("act", sorted(ACT))
def test_projection(T, K, N, dtype, stream, act):
    say(f"[projection] T={T} K={K} N={N} {dtype} {stream} {act}")
    g = gen_num(T + 3 * K + 7 * N)
    dt, st = DTYPE[dtype], DTYPE[stream]
    x, w = rand((T, K), g, dt), rand((N, K), g, dt, K ** -0.5)
    b, res = rand((N,), g, scale=0.3), rand((T, N), g, st)
    want, want_pre = ref.projection(x, w, b, act, res)
    pre = torch.empty(T, N, dtype=dt, device=DEV)
    out = linear.lbi_projection(x, w, b, ACT[act], res, pre=pre)
    terms = (x.double().cpu().square() @ w.double().cpu().square().T).sqrt().norm().item()
    check(out, want, "out", floor=terms)
    check(pre, want_pre, "pre", floor=terms)
    # strided, in place on the residual
    rs, ps = wide_rows(res, 5), wide_rows(pre, 3)
    again = linear.lbi_projection(wide_rows(x, 3), wide_rows(w, 7), b, ACT[act], rs, out=rs, pre=ps)
    assert torch.equal(again, out) and torch.equal(ps, pre)
    assert torch.isnan(beside(rs)).all() and torch.isnan(beside(ps)).all()
    bare = linear.lbi_projection(x, w, act=ACT[act], out=torch.empty(T, N, dtype=st, device=DEV))
    check(bare, ref.projection(x, w, None, act)[0], "bare", floor=terms)


@pytest.mark.parametrize("T,K,N", PRODUCTS + [(0, 20, 30)])
@pytest.mark.parametrize("dtype,stream", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"),
                                          ("f32", "bf16")])
@pytest.mark.parametrize("act", sorted(ACT))
def test_projection_backward(T, K, N, dtype, stream, act):
    say(f"[projection_backward] T={T} K={K} N={N} {dtype} {stream} {act}")
    g = gen_num(T + 5 * K + 11 * N)
    dt, st = DTYPE[dtype], DTYPE[stream]
    x, w = rand((T, K), g, dt), rand((N, K), g, dt, K ** -0.5)
    dout, pre = rand((T, N), g, st), rand((T, N), g, dt)
    pre = None if act == "none" else pre
    dx, dw, db = linear.lbi_projection_backward(x, w, dout, ACT[act], pre)
    want_x, want_w, want_b, dz = ref.projection_backward(x, w, dout, act, pre)
    tx = (dz.square() @ w.double().cpu().square()).sqrt()
    tw = (dz.square().T @ x.double().cpu().square()).sqrt()
    rounded = dtype == "bf16"
    check(dx, want_x, "dx", tx if rounded else None, tx.norm().item())
    check(dw, want_w, "dweight", tw if rounded else None, tw.norm().item())
    check(db, want_b, "dbias", floor=dz.norm().item())
    if T == 0:
        assert (dw == 0).all() and (db == 0).all()
        return
    outs, ows = wide_rows(torch.zeros_like(x), 5), wide_rows(torch.zeros_like(w), 3)
    again = linear.lbi_projection_backward(
        wide_rows(x, 3), wide_rows(w, 9), wide_rows(dout, 5), ACT[act],
        None if pre is None else wide_rows(pre, 3), dx=outs, dweight=ows)
    assert torch.equal(outs, dx) and torch.equal(ows, dw) and torch.equal(again[2], db)
    assert torch.isnan(beside(outs)).all() and torch.isnan(beside(ows)).all()


@pytest.mark.parametrize("T,K,N", [(64, 1536, 768), (1, 4096, 100), (200, 5000, 64), (16, 700, 33)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_projection_of_few_rows(T, K, N, dtype):
    """Long sums over few rows."""
    say(f"[projection] T={T} K={K} N={N} {dtype}")
    g = gen_num(K)
    x, w = rand((T, K), g, DTYPE[dtype]), rand((N, K), g, DTYPE[dtype], K ** -0.5)
    b, res = rand((N,), g), rand((T, N), g)
    out = linear.lbi_projection(x, w, b, ACT["silu"], res)
    assert out.dtype == torch.float32
    check(out, ref.projection(x, w, b, "silu", res)[0], "out", floor=(T * N) ** 0.5)
    assert torch.equal(linear.lbi_projection(x, w, b, ACT["silu"], res), out)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_projection_nan_stays_in_its_row(dtype):
    g = gen_num(9)
    x, w = rand((140, 200), g, DTYPE[dtype]), rand((150, 200), g, DTYPE[dtype])
    good = linear.lbi_projection(x, w)
    x[5, 199], w[149, 3] = float("nan"), float("inf")
    out = linear.lbi_projection(x, w)
    assert torch.isnan(out[5]).all() and not torch.isfinite(out[:, 149]).any()
    keep = [t for t in range(140) if t != 5]
    assert torch.equal(out[keep][:, :149], good[keep][:, :149])


# ---- linear attention --------------------------------------------------------

LENGTHS = {"one": [1], "tile": [64], "tile + 1": [65], "mixed": [3, 0, 1, 64, 130], "equal": [70] * 3,
           "singles": [1] * 70, "late": [0, 0, 5], "long": [700, 300, 37], "even": [256] * 2}
HEADS = [(1, 1, 1, 1), (2, 2, 16, 16), (3, 1, 64, 64), (4, 2, 48, 101), (2, 1, 128, 128),
         (2, 2, 33, 64), (1, 1, 64, 128), (2, 1, 128, 17), (2, 1, 128, 64)]


def packing(n):
    """Equal lengths as such, others by offsets."""
    if len(set(n)) == 1:
        return {"sequences": len(n)}
    return {"offsets": torch.tensor([0, *n]).cumsum(0).to(DEV)}


def attention_inputs(n, H, KH, DK, DV, dtype, seed):
    T, B = sum(n), len(n)
    g = gen_num(seed)
    dt = DTYPE[dtype]
    decay = -torch.exp(torch.empty(H).uniform_(-7.0, -0.3, generator=g))
    return {"q": rand((T, H, DK), g, dt), "k": rand((T, KH, DK), g, dt),
            "v": rand((T, KH, DV), g, dt), "log_decay": decay.to(DEV),
            "state": rand((B, H, DK, DV), g, scale=3.0)}, g


def args_of(s):
    return s["q"], s["k"], s["v"], s["log_decay"]


@pytest.mark.parametrize("lengths", sorted(LENGTHS))
@pytest.mark.parametrize("H,KH,DK,DV", HEADS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention(lengths, H, KH, DK, DV, dtype):
    say(f"[attention] {lengths} H={H} KH={KH} DK={DK} DV={DV} {dtype}")
    n = LENGTHS[lengths]
    s, g = attention_inputs(n, H, KH, DK, DV, dtype, DK * 7 + DV)
    scale = DK ** -0.5
    terms = ref.attention_terms(*args_of(s), scale, n)["out"]
    inner = terms if dtype == "bf16" else None
    want, want_new = ref.attention(*args_of(s), scale, n, s["state"])
    new = torch.full_like(s["state"], float("nan"))
    out = linear.lbi_linear_attention(*args_of(s), state_in=s["state"], state_out=new, **packing(n))
    check(out, want, "out", inner, terms.norm().item())
    check(new, want_new, "state_out")
    bare = linear.lbi_linear_attention(*args_of(s), 0.3, **packing(n))
    check(bare, ref.attention(*args_of(s), 0.3, n)[0], "bare", inner, terms.norm().item())
    # in place, from slices of wider rows
    state = s["state"].clone()
    far = wide_rows(torch.zeros_like(out), 7)
    linear.lbi_linear_attention(*(wide_rows(t, 5) for t in args_of(s)[:3]), s["log_decay"],
                                state_in=state, state_out=state, out=far, **packing(n))
    assert torch.equal(far, out) and torch.equal(state, new)
    assert torch.isnan(beside(far)).all()


@pytest.mark.parametrize("lengths", sorted(LENGTHS))
@pytest.mark.parametrize("H,KH,DK,DV", HEADS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_backward(lengths, H, KH, DK, DV, dtype):
    say(f"[attention_backward] {lengths} H={H} KH={KH} DK={DK} DV={DV} {dtype}")
    n = LENGTHS[lengths]
    s, g = attention_inputs(n, H, KH, DK, DV, dtype, DK * 11 + DV)
    dout = rand((sum(n), H, DV), g, DTYPE[dtype])
    dnew = rand(s["state"].shape, g)
    scale = DK ** -0.5
    terms = ref.attention_terms(*args_of(s), scale, n, dout)
    for state, ds in ((s["state"], dnew), (s["state"], None), (None, None)):
        got = linear.lbi_linear_attention_backward(*args_of(s), dout, state_in=state, dstate_out=ds,
                                                   **packing(n))
        want = ref.attention_backward(*args_of(s), scale, n, dout, state, ds)
        assert (got["state_in"] is None) == (state is None)
        for k, e in want.items():
            if k == "log_decay":
                # a sum over all pairs: as exact as its terms, q . dq and k . dk over the memory
                floor = sum((s[x].double().cpu() * want[x]).norm().item() for x in ("q", "k"))
                floor *= (1.0 / (1.0 - torch.exp(s["log_decay"].double()))).max().item()
                if ds is not None:  # from the first state to the last one
                    floor += ds.norm().item() * s["state"].norm().item()
                check(got[k], e, k, floor=floor)
            else:
                inner = terms.get(k) if dtype == "bf16" else None
                floor = terms[k].norm().item() if k in terms else scale * dout.float().norm().item()
                check(got[k], e, k, inner, floor)
    again = linear.lbi_linear_attention_backward(*args_of(s), dout, state_in=state, dstate_out=ds,
                                                 **packing(n))
    for k, t in got.items():
        assert t is None or torch.equal(t, again[k]), k
    outs = {k: wide_rows(torch.zeros_like(s[k]), 5) for k in ("q", "k", "v")}
    linear.lbi_linear_attention_backward(*(wide_rows(t, 3) for t in args_of(s)[:3]), s["log_decay"],
                                         wide_rows(dout, 9), outputs=outs, **packing(n))
    for k, t in outs.items():
        assert torch.equal(t, got[k]) and torch.isnan(beside(t)).all(), k


@pytest.mark.parametrize("H,KH,DK,DV", HEADS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_steps_follow_the_prompt(H, KH, DK, DV, dtype):
    say(f"[attention_step] H={H} KH={KH} DK={DK} DV={DV} {dtype}")
    n, L = 5, 6
    s, g = attention_inputs([L] * n, H, KH, DK, DV, dtype, DK * 13 + DV)
    scale = DK ** -0.5
    want, want_new = ref.attention(*args_of(s), scale, [L] * n, s["state"])
    slots = torch.tensor([6, 0, 3, 4, 2], dtype=torch.int32, device=DEV)
    cache = rand((7, H, DK, DV), g)
    cache[slots.long()] = s["state"]
    before = cache.clone()
    rows = [t.view(n, L, *t.shape[1:]) for t in args_of(s)[:3]]

    def step(t, cache):
        return linear.lbi_linear_attention_step(*(x[:, t] for x in rows), s["log_decay"], cache,
                                                cache, slots=slots)
    y = torch.stack([step(t, cache) for t in range(L)], 1)
    check(y, want.view(n, L, H, DV), "steps", floor=want.norm().item())
    check(cache[slots.long()], want_new, "states")
    assert torch.equal(cache[[1, 5]], before[[1, 5]]), "other slots are left alone"
    # a slot out of range: zeros in, nothing written
    slots[1], slots[3] = -3, 7
    cache = before.clone()
    zeroed = s["state"].clone()
    zeroed[[1, 3]] = 0
    one = [x[:, 0] for x in rows]
    check(step(0, cache), ref.attention(*one, s["log_decay"], scale, [1] * n, zeroed)[0],
          "step without a slot", floor=want.norm().item() / L)
    assert torch.equal(cache[[0, 1, 4, 5]], before[[0, 1, 4, 5]])
    prompt = before.clone()
    y = linear.lbi_linear_attention(*args_of(s), sequences=n, state_in=prompt, state_out=prompt,
                                    slots=slots)
    want, want_new = ref.attention(*args_of(s), scale, [L] * n, zeroed)
    terms = ref.attention_terms(*args_of(s), scale, [L] * n)["out"]
    check(y, want, "prompt", terms if dtype == "bf16" else None, terms.norm().item())
    check(prompt[[6, 3, 2]], want_new[[0, 2, 4]], "prompt states")
    assert torch.equal(prompt[[0, 1, 4, 5]], before[[0, 1, 4, 5]])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_decays_at_their_ends(dtype):
    """Heads that never forget and that forget at once; above 0 and NaN there is no decay."""
    n, H = [150, 1, 90], 4
    s, g = attention_inputs(n, H, 4, 32, 48, dtype, 5)
    s["log_decay"] = torch.tensor([0.0, float("-inf"), -200.0, -1e-9], device=DEV)
    dout, scale = rand((sum(n), H, 48), g, DTYPE[dtype]), 32 ** -0.5
    terms = ref.attention_terms(*args_of(s), scale, n, dout)
    new = torch.empty_like(s["state"])
    out = linear.lbi_linear_attention(*args_of(s), state_in=s["state"], state_out=new, **packing(n))
    want, want_new = ref.attention(*args_of(s), scale, n, s["state"])
    bf16 = dtype == "bf16"
    check(out, want, "out", terms["out"] if bf16 else None)
    check(new, want_new, "state_out")
    finite = dict(s, log_decay=s["log_decay"].clamp(min=-1e4))  # the oracle differentiates e^x
    got = linear.lbi_linear_attention_backward(*args_of(s), dout, state_in=s["state"], **packing(n))
    want = ref.attention_backward(*args_of(finite), scale, n, dout, s["state"])
    for k in ("q", "k", "v"):
        check(got[k], want[k], k, terms[k] if bf16 else None)
    check(got["state_in"], want["state_in"], "state_in")
    assert got["log_decay"][1] == 0
    check(got["log_decay"][[0, 3]], want["log_decay"][[0, 3]], "log_decay",
          floor=150 * (s["q"].double().cpu() * want["q"]).norm().item())
    s["log_decay"][2], s["log_decay"][3] = 0.1, float("nan")
    out2 = linear.lbi_linear_attention(*args_of(s), state_in=s["state"], **packing(n))
    assert torch.isnan(out2[:, 2:]).all() and torch.equal(out2[:, :2], out[:, :2])
    state = s["state"].clone()
    one = [t[:3] for t in args_of(s)[:3]]
    y = linear.lbi_linear_attention_step(*one, s["log_decay"], state, state)
    assert torch.isnan(y[:, 2:]).all() and torch.isfinite(y[:, :2]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("which", ["q", "k", "v", "dout"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("D", [32, 64, 128])
def test_a_token_does_not_reach_what_it_may_not(dtype, which, value, D):
    """A NaN or an infinity in one token: outputs before it, gradients of what it does not see, other
    heads and other sequences keep their bits or their values."""
    n, H, at = [100, 90], 2, 37
    s, g = attention_inputs(n, H, 2, D, D, dtype, 6)
    x = dict(s, dout=rand((190, H, D), g, DTYPE[dtype]))
    off = packing(n)

    def run(x):
        out = linear.lbi_linear_attention(*args_of(x), state_in=x["state"], **off)
        return out, linear.lbi_linear_attention_backward(*args_of(x), x["dout"],
                                                         state_in=x["state"], **off)
    out, grad = run(x)
    bad = dict(x)
    bad[which] = x[which].clone()
    bad[which][at, 1, 5] = value
    out2, grad2 = run(bad)

    def same(a, b):
        assert torch.isfinite(b).all()
        a, b = a.float(), b.float()
        # taken token by token the sums are rounded elsewhere
        assert (a - b).norm() <= (2.0 ** -6 if dtype == "bf16" else 2 * F32_TOL) * a.norm()
    for a, b in ((out, out2), *((grad[k], grad2[k]) for k in ("q", "k", "v"))):
        assert torch.equal(a[:, 0], b[:, 0]) and torch.equal(a[100:], b[100:])
    if which == "dout":
        assert torch.equal(out, out2)
        same(grad["q"][:at, 1], grad2["q"][:at, 1])
        for k in ("q", "k", "v"):  # dout of a token reaches the tokens before it
            same(grad[k][at + 1:100, 1], grad2[k][at + 1:100, 1])
        assert not torch.isfinite(grad2["q"][at, 1]).all()
    else:
        same(out[:at, 1], out2[:at, 1])
        assert not torch.isfinite(out2[at, 1]).all()
    if which in ("k", "v"):
        same(grad["q"][:at, 1], grad2["q"][:at, 1])
    if which == "q":
        same(out[at + 1:100, 1], out2[at + 1:100, 1])
        same(grad["q"][:at, 1], grad2["q"][:at, 1])
        for k in ("k", "v"):
            same(grad[k][at + 1:100, 1], grad2[k][at + 1:100, 1])
