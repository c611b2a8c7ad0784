"""Parity of the region block's operators (include/lbi_block.h) with their definitions in float64
(oracle/block.py), through the C-ABI (needs a GPU).

Tolerances, from the arithmetic: relative Frobenius error.  Everything is held in float32, where
an element collects a few dozen roundings of 2^-24 that do not lean one way; a state collects
those of its memory, up to about 10^3 tokens at the slowest decays here, a random walk of 32
roundings' size: 1e-5 bounds all of them, as it does for the library's other float32 results.  A bf16
output adds one rounding of at most 2^-8 relative to each element (8 significant bits).  An 8-bit output adds half a
step: 2^-4 relative to an E4M3 value, half the scale to an INT8 one (both elementwise).
"""
import sys

import pytest
import torch

from oracle import block as ref
from paper_2605_09204_amd import block

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
F32_TOL = 1e-5
TOL = {torch.float32: F32_TOL, torch.bfloat16: 2.0 ** -8 + F32_TOL}


def say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def check(got, want, label, terms=None):
    """``terms``: the norm of what was summed over the tokens; a sum that cancels is as exact as
    those are, not as itself."""
    assert got is not None, label
    got64 = got.detach().cpu().double().reshape(want.shape)
    if want.numel() == 0:
        return
    assert torch.isfinite(got64).all(), f"{label}: not finite"
    norm = max(want.norm().item(), terms or 0.0)
    err = (got64 - want).norm().item() / (norm if norm > 0 else 1.0)
    assert err <= TOL[got.dtype], f"{label}: relative error {err:.3g}"


def rand(shape, gen, dtype=torch.float32, scale=1.0):
    return (scale * torch.randn(shape, generator=gen)).to(dtype).to(DEV)


def gen_of(*key):
    g = torch.Generator()
    g.manual_seed(hash(key) % (1 << 31))
    return g


def gen_num(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def wide_rows(t, extra, gen):
    """The same values as a slice of wider rows, from an odd element on; the rest is NaN."""
    lead, D = t.shape[:-1], t.shape[-1]
    full = torch.full((*lead, D + extra), float("nan"), dtype=t.dtype, device=t.device)
    view = full[..., extra // 2:extra // 2 + D]
    view.copy_(t)
    return view


# ---- norm --------------------------------------------------------------------

NORM_SHAPES = [(1, 1), (3, 7), (5, 64), (130, 100), (17, 129), (9, 768), (1100, 520), (1030, 1111),
               (4, 1000), (1, 2048), (1025, 2040), (7, 4100), (3, 8192), (2, 16383)]


@pytest.mark.parametrize("T,D", NORM_SHAPES)
@pytest.mark.parametrize("dtype,stream", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"),
                                          ("f32", "bf16")])
def test_norm(T, D, dtype, stream):
    say(f"[norm] T={T} D={D} {dtype} {stream}")
    g = gen_num(T * 31 + D)
    x = rand((T, D), g, DTYPE[dtype])
    w = 1.0 + rand((D,), g, scale=0.2)
    r = rand((T, D), g, DTYPE[stream], 2.0)
    out, total = block.lbi_rms_norm(x, w, r)
    want, s = ref.rms_norm(x, w, r)
    check(out, want, "out")
    check(total, s, "residual_out")
    out, total = block.lbi_rms_norm(x, w)
    assert total is None
    check(out, ref.rms_norm(x, w)[0], "out without a residual")
    # strided rows, in place on the residual
    xs, rs = wide_rows(x, 5, g), wide_rows(r, 3, g)
    outs = wide_rows(torch.zeros_like(x), 9, g)
    block.lbi_rms_norm(xs, w, rs, out=outs, residual_out=rs)
    check(outs, want, "strided out")
    check(rs, s, "residual in place")
    assert torch.isnan(outs._base[..., :4]).all() and torch.isnan(rs._base[..., -2:]).all()


@pytest.mark.parametrize("T,D", NORM_SHAPES)
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("group", [0, 32, 64, 128])
def test_norm_q8(T, D, fmt, group):
    say(f"[norm_q8] T={T} D={D} {fmt} group={group}")
    g = gen_num(T * 37 + D + group)
    x = rand((T, D), g, torch.bfloat16)
    x[T // 2] = 0  # a row of zeros
    w = 1.0 + rand((D,), g, scale=0.2)
    r = rand((T, D), g, torch.bfloat16) if T % 2 else None
    if r is not None:
        r[T // 2] = 0
    q, scales, total = block.lbi_rms_norm_q8(
        x, w, r, format=block.LBI_Q8_E4M3 if fmt == "e4m3" else block.LBI_Q8_INT8, group=group)
    want, s = ref.rms_norm(x, w, r)
    check(scales, ref.q8_scales(want, group, fmt), "scales")
    if r is not None:
        check(total, s, "residual_out")
    width = group or D
    sc = scales.cpu().double().repeat_interleave(width, -1)[..., :D]
    got = q.cpu().float().double() * sc
    err = (got - want).abs()
    if fmt == "e4m3":  # half a step is 2^-4 of the value, or of the smallest normal one, 2^-6
        bound = torch.maximum(want.abs(), sc * 2.0 ** -6) * 2.0 ** -4
    else:
        bound = sc * 0.5
    assert (err <= bound * (1 + 1e-4) + 1e-30).all(), (err / bound).max()
    assert (q[T // 2].float() == 0).all() and (scales[T // 2] == 1).all()


def test_norm_non_finite_rows():
    say("[norm] NaN, infinity, zero rows")
    g = gen_num(5)
    x = rand((6, 300), g)
    x[1, 7] = float("nan")
    x[3, 299] = float("inf")
    x[4] = 0
    w = torch.ones(300, device=DEV)
    out, _ = block.lbi_rms_norm(x, w)
    want = ref.rms_norm(x, w)[0]
    fine = [0, 2, 4, 5]
    check(out[fine], want[fine], "finite rows")
    assert torch.isnan(out[1]).all() and torch.isnan(out[3, 299])
    q, scales, _ = block.lbi_rms_norm_q8(x, w)
    assert torch.isnan(scales[[1, 3]]).all() and torch.isfinite(scales[fine]).all()
    assert scales[4] == 1


@pytest.mark.parametrize("T,D", NORM_SHAPES)
@pytest.mark.parametrize("dtype,stream", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
def test_norm_backward(T, D, dtype, stream):
    say(f"[norm_backward] T={T} D={D} {dtype} {stream}")
    g = gen_num(T * 41 + D)
    dout = rand((T, D), g, DTYPE[dtype])
    s = rand((T, D), g, DTYPE[stream], 1.5)
    w = 1.0 + rand((D,), g, scale=0.2)
    dr = rand((T, D), g, DTYPE[stream])
    for d in (None, dr):
        ds, dw = block.lbi_rms_norm_backward(dout, s, w, d)
        want, want_w = ref.rms_norm_backward(dout, s, w, d)
        if D > 1 or d is not None:  # D = 1: the norm is a sign, its gradient cancels
            check(ds, want, "ds")
        check(dw, want_w, "dweight")
    again, dw2 = block.lbi_rms_norm_backward(dout, s, w, dr)
    assert torch.equal(again, ds) and torch.equal(dw2, dw)
    block.lbi_rms_norm_backward(wide_rows(dout, 7, g), s, w, dr, ds=dr)
    assert torch.equal(dr, ds)


# ---- convolution -------------------------------------------------------------

LENGTHS = {"one": [1], "short": [1, 2, 3, 4, 5], "dense": [9, 9, 9], "ragged": [0, 17, 0, 0, 1, 40, 2, 0],
           "long": [700], "many": [3, 0, 5, 1] * 20, "empty": [0, 0, 0], "wide": [260, 31]}


def offsets_of(lengths):
    return torch.tensor([sum(lengths[:i]) for i in range(len(lengths) + 1)], dtype=torch.int64,
                        device=DEV)


def packing(lengths):
    """Keyword arguments for packed sequences: without offsets where all have one length."""
    if len(set(lengths)) == 1 and lengths[0] > 0:
        return {"sequences": len(lengths)}
    return {"offsets": offsets_of(lengths)}


@pytest.mark.parametrize("lengths", sorted(LENGTHS))
@pytest.mark.parametrize("D,W", [(1, 2), (7, 3), (64, 4), (130, 2), (777, 4), (1536, 3)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_conv(lengths, D, W, dtype):
    say(f"[conv] {lengths} D={D} W={W} {dtype}")
    n = LENGTHS[lengths]
    T, B = sum(n), len(n)
    g = gen_num(T * 3 + D + W)
    x = rand((T, D), g, DTYPE[dtype])
    w, b = rand((D, W), g, scale=0.6), rand((D,), g, scale=0.2)
    old = rand((B, W - 1, D), g, DTYPE[dtype])
    for silu, bias, state in ((True, b, old), (False, None, None)):
        new = torch.full_like(old, float("nan"))
        out = block.lbi_ssm_conv(x, w, bias, silu=silu, state_in=state, state_out=new,
                                 **packing(n))
        want, want_new = ref.conv(x, w, bias, state, n, silu)
        check(out, want, "out")
        assert torch.equal(new.cpu().double(), want_new), "the states are copies"
    # states in place, rows of wider tensors
    new = old.clone()
    out = block.lbi_ssm_conv(wide_rows(x, 3, g), w, b, state_in=new, state_out=new,
                             out=wide_rows(torch.zeros_like(x), 5, g), **packing(n))
    want, want_new = ref.conv(x, w, b, old, n, True)
    check(out, want, "strided out")
    assert torch.equal(new.cpu().double(), want_new)


@pytest.mark.parametrize("lengths", sorted(LENGTHS))
@pytest.mark.parametrize("D,W", [(1, 2), (7, 3), (64, 4), (130, 2), (777, 4)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_conv_backward(lengths, D, W, dtype):
    say(f"[conv_backward] {lengths} D={D} W={W} {dtype}")
    n = LENGTHS[lengths]
    T, B = sum(n), len(n)
    g = gen_num(T * 5 + D + W)
    x, dout = rand((T, D), g, DTYPE[dtype]), rand((T, D), g, DTYPE[dtype])
    w, b = rand((D, W), g, scale=0.6), rand((D,), g, scale=0.2)
    old, dnew = rand((B, W - 1, D), g, DTYPE[dtype]), rand((B, W - 1, D), g, DTYPE[dtype])
    for silu, bias, state, ds in ((True, b, old, dnew), (False, None, old, None),
                                  (True, b, None, dnew)):
        got = block.lbi_ssm_conv_backward(x, w, dout, bias, silu=silu, state_in=state,
                                          dstate_out=ds, **packing(n))
        want = ref.conv_backward(x, w, bias, state, n, dout, ds, silu)
        for name, a, e in zip(("dx", "dweight", "dbias", "dstate_in"), got, want):
            if e is None:
                assert a is None
            else:
                check(a, e, name)


@pytest.mark.parametrize("D,W", [(1, 2), (7, 3), (130, 4), (1536, 4)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_conv_steps_follow_the_prompt(D, W, dtype):
    say(f"[conv_step] D={D} W={W} {dtype}")
    g = gen_num(D + W)
    n, L = 5, 6
    x = rand((n, L, D), g, DTYPE[dtype])
    w, b = rand((D, W), g, scale=0.6), rand((D,), g, scale=0.2)
    old = rand((n, W - 1, D), g, DTYPE[dtype])
    want, want_new = ref.conv(x.reshape(n * L, D), w, b, old, [L] * n)
    # requests in slots 6, 0, 3, 4, 2 of a cache, stepped in place
    slots = torch.tensor([6, 0, 3, 4, 2], dtype=torch.int32, device=DEV)
    cache = rand((7, W - 1, D), g, DTYPE[dtype])
    cache[slots.long()] = old
    before = cache.clone()
    out = torch.stack([block.lbi_ssm_conv_step(x[:, t], w, cache, cache, b, slots=slots)
                       for t in range(L)], 1)
    check(out, want.view(n, L, D), "steps")
    assert torch.equal(cache[slots.long()].cpu().double(), want_new)
    assert torch.equal(cache[[1, 5]], before[[1, 5]]), "other slots are left alone"
    # a slot out of range: zeros in, nothing written
    slots[1] = -1
    slots[3] = 7
    cache = before.clone()
    out = block.lbi_ssm_conv_step(x[:, 0], w, cache, cache, b, slots=slots)
    zeroed = old.clone()
    zeroed[[1, 3]] = 0
    check(out, ref.conv(x[:, 0], w, b, zeroed, [1] * n)[0], "step without a slot")
    assert torch.equal(cache[[0, 1, 4, 5]], before[[0, 1, 4, 5]])
    prompt = before.clone()
    got = block.lbi_ssm_conv(x, w, b, state_in=prompt, state_out=prompt, slots=slots)
    check(got, ref.conv(x.reshape(n * L, D), w, b, zeroed, [L] * n)[0].view(n, L, D), "prompt")
    assert torch.equal(prompt[[0, 1, 4, 5]], before[[0, 1, 4, 5]])


# ---- scan --------------------------------------------------------------------

def scan_inputs(n, D, N, G, dtype, seed, full=True, slow=1e-3):
    T, B = sum(n), len(n)
    g = gen_num(seed)
    dt = DTYPE[dtype]
    step = torch.exp(torch.empty(D).uniform_(float(torch.log(torch.tensor(slow))), -2.3,
                                             generator=g))
    s = {"u": rand((T, D), g, dt), "delta": rand((T, D), g, dt, 0.5),
         "A": (-(torch.arange(N) + 1.0) * torch.exp(0.1 * torch.randn(D, N, generator=g))).to(DEV),
         "B": rand((T, G, N), g, dt), "C": rand((T, G, N), g, dt),
         "delta_bias": (step + torch.log(-torch.expm1(-step))).to(DEV)}
    if full:
        s |= {"skip": 1.0 + rand((D,), g, scale=0.1), "z": rand((T, D), g, dt),
              "state_in": rand((B, D, N), g)}
    return s, g


def call_scan(s, n, **kw):
    opt = {k: s.get(k) for k in ("skip", "z", "delta_bias", "state_in")}
    return block.lbi_ssm_scan(s["u"], s["delta"], s["A"], s["B"], s["C"], **opt, **packing(n), **kw)


SCAN_SIZES = [(1, 1, 1), (5, 3, 1), (64, 16, 1), (130, 16, 2), (100, 12, 4), (72, 8, 1), (48, 24, 2),
              (33, 33, 1), (70, 64, 1)]


@pytest.mark.parametrize("lengths", sorted(LENGTHS))
@pytest.mark.parametrize("D,N,G", SCAN_SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scan(lengths, D, N, G, dtype):
    say(f"[scan] {lengths} D={D} N={N} G={G} {dtype}")
    n = LENGTHS[lengths]
    s, g = scan_inputs(n, D, N, G, dtype, D * 7 + N)
    new = torch.full((len(n), D, N), float("nan"), device=DEV)
    y = call_scan(s, n, state_out=new)
    want, want_new = ref.scan(s, n)
    check(y, want, "y")
    check(new, want_new, "state_out")
    again = call_scan(s, n)
    assert torch.equal(again, y)
    # in place, from slices of wider rows
    w = dict(s)
    for k in ("u", "delta", "z"):
        w[k] = wide_rows(s[k], 3, g)
    both = wide_rows(torch.cat([s["B"], s["C"]], 1).flatten(1), 5, g)
    w["B"], w["C"] = (t.unflatten(1, (G, N)) for t in both.split(G * N, 1))
    w["state_in"] = s["state_in"].clone()
    y2 = call_scan(w, n, state_out=w["state_in"],
                   out=wide_rows(torch.zeros_like(s["u"]), 7, g))
    assert torch.equal(y2, y) and torch.equal(w["state_in"], new)
    # the bare recurrence
    bare, _ = scan_inputs(n, D, N, G, dtype, D * 7 + N, full=False)
    bare["delta"] = bare["delta"].abs()
    bare["delta_bias"] = None
    y = call_scan(bare, n, softplus=False)
    check(y, ref.scan(bare, n, softplus=False)[0], "bare y")


@pytest.mark.parametrize("lengths", sorted(LENGTHS))
@pytest.mark.parametrize("D,N,G", SCAN_SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scan_backward(lengths, D, N, G, dtype):
    say(f"[scan_backward] {lengths} D={D} N={N} G={G} {dtype}")
    n = LENGTHS[lengths]
    s, g = scan_inputs(n, D, N, G, dtype, D * 11 + N)
    dout = rand((sum(n), D), g, DTYPE[dtype])
    dnew = rand((len(n), D, N), g)
    bare, _ = scan_inputs(n, D, N, G, dtype, D * 11 + N, full=False)
    for case, ds in ((s, dnew), (s, None), (bare, None)):
        a = [case[k] for k in ("u", "delta", "A", "B", "C")]
        opt = {k: case.get(k) for k in ("skip", "z", "delta_bias", "state_in")}
        got = block.lbi_ssm_scan_backward(*a, dout, dstate_out=ds, **opt, **packing(n))
        want = ref.scan_backward(case, n, dout, ds)
        for k, e in want.items():
            if e is None:
                assert got[k] is None, k
            else:
                check(got[k], e, k,
                      want["delta"].norm().item() if k == "delta_bias" else None)
    again = block.lbi_ssm_scan_backward(*a, dout, dstate_out=ds, **opt, **packing(n))
    for k, t in got.items():
        assert t is None or torch.equal(t, again[k]), k


@pytest.mark.parametrize("D,N,G", SCAN_SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scan_steps_follow_the_prompt(D, N, G, dtype):
    say(f"[scan_step] D={D} N={N} G={G} {dtype}")
    n, L = 5, 6
    s, g = scan_inputs([L] * n, D, N, G, dtype, D * 13 + N)
    want, want_new = ref.scan(s, [L] * n)
    slots = torch.tensor([6, 0, 3, 4, 2], dtype=torch.int32, device=DEV)
    cache = rand((7, D, N), g)
    cache[slots.long()] = s["state_in"]
    before = cache.clone()
    rows = {k: s[k].view(n, L, *s[k].shape[1:]) for k in ("u", "delta", "B", "C", "z")}

    def step(t, cache):
        return block.lbi_ssm_scan_step(rows["u"][:, t], rows["delta"][:, t], s["A"],
                                       rows["B"][:, t], rows["C"][:, t], cache, cache, s["skip"],
                                       rows["z"][:, t], s["delta_bias"], slots=slots)
    y = torch.stack([step(t, cache) for t in range(L)], 1)
    check(y, want.view(n, L, D), "steps")
    check(cache[slots.long()], want_new, "states")
    assert torch.equal(cache[[1, 5]], before[[1, 5]])
    slots[1] = -3
    slots[3] = 7
    cache = before.clone()
    zeroed = dict(s, state_in=s["state_in"].clone())
    zeroed["state_in"][[1, 3]] = 0
    one = {k: (v[:, 0] if k in rows else zeroed[k]) for k, v in
           {**zeroed, **rows}.items()}
    check(step(0, cache), ref.scan(one, [1] * n)[0], "step without a slot")
    assert torch.equal(cache[[0, 1, 4, 5]], before[[0, 1, 4, 5]])
    prompt = before.clone()
    y = block.lbi_ssm_scan(s["u"], s["delta"], s["A"], s["B"], s["C"], s["skip"], s["z"],
                           s["delta_bias"], sequences=n, state_in=prompt, state_out=prompt,
                           slots=slots)
    want, want_new = ref.scan(zeroed, [L] * n)
    check(y, want, "prompt")
    check(prompt[[6, 3, 2]], want_new[[0, 2, 4]], "prompt states")
    assert torch.equal(prompt[[0, 1, 4, 5]], before[[0, 1, 4, 5]])
