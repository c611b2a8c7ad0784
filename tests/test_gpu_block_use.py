"""The region block's operators as a program uses them (needs a GPU): gradients against
differences of the operators' own outputs, addresses past 32 bits, other streams, replays in a
graph, results that do not change from run to run, refusals, and the example.

Differences: a central difference along one direction v, |v| = 1, with the steps 2^-3 and 2^-4
extrapolated.  What the extrapolation leaves is under 1e-5 of |gradient| for these sizes (held on
the CPU, in float64, by test_differences_are_exact_enough); the outputs' float32 errors, 1e-7 of
|cotangent| |outputs| with |outputs| under 20 |gradient|, divided by the step, add some 2e-5.
The bound is 1e-3 of |gradient|.
"""
import sys

import pytest
import torch

from oracle import block as ref
from paper_2605_09204_amd import binding, block

gpu = pytest.mark.gpu
DEV = "cuda:0"
DIFF_TOL = 1e-3


def say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def difference(f, inputs, dirs, h):
    def at(k):
        return f({n: t + k * dirs[n] for n, t in inputs.items()})
    return (at(h) - at(-h)) / (2 * h)


def extrapolated(f, inputs, dirs):
    return (4 * difference(f, inputs, dirs, 2.0 ** -4) - difference(f, inputs, dirs, 2.0 ** -3)) / 3


def directions(inputs, g, grads):
    """Half along the gradient and half anywhere, |v| = 1."""
    r = {n: torch.randn(t.shape, generator=g, dtype=torch.float64) for n, t in inputs.items()}
    a = sum(t.square().sum() for t in grads.values()).sqrt()
    b = sum(t.square().sum() for t in r.values()).sqrt()
    v = {n: grads[n] / a + r[n] / b for n in inputs}
    size = sum(t.square().sum() for t in v.values()).sqrt()
    return {n: t / size for n, t in v.items()}


def problem(kind, seed=5):
    """(inputs in float64, lengths, cotangents of the output and of the last state)."""
    g = gen(seed)
    n = [21, 0, 1, 18]
    T, S, D, N, G = sum(n), len(n), 6, 8, 2

    def r(*s):
        return torch.randn(s, generator=g).double()
    if kind == "norm":
        return {"s": r(T, 40), "w": r(40)}, n, r(T, 40), r(T, 40)
    if kind == "conv":
        return {"x": r(T, D), "w": r(D, 4), "b": r(D), "old": r(S, 3, D)}, n, r(T, D), r(S, 3, D)
    return {"u": r(T, D), "delta": r(T, D) - 1, "A": -torch.exp(0.5 * r(D, N)), "B": r(T, G, N),
            "C": r(T, G, N), "skip": r(D), "z": r(T, D), "delta_bias": r(D),
            "state_in": r(S, D, N)}, n, r(T, D), r(S, D, N)


def reference(kind, v, n, dy, dn):
    """(loss, gradients) in float64."""
    if kind == "norm":
        out, s = ref.rms_norm(v["s"], v["w"])
        ds, dw = ref.rms_norm_backward(dy, v["s"], v["w"])
        return (out * dy).sum() + (s * dn).sum(), {"s": ds + dn, "w": dw}
    if kind == "conv":
        y, new = ref.conv(v["x"], v["w"], v["b"], v["old"], n)
        g = ref.conv_backward(v["x"], v["w"], v["b"], v["old"], n, dy, dn)
        return (y * dy).sum() + (new * dn).sum(), dict(zip(("x", "w", "b", "old"), g))
    y, new = ref.scan(v, n)
    return (y * dy).sum() + (new * dn).sum(), ref.scan_backward(v, n, dy, dn)


def offsets_of(n):
    return torch.tensor([0, *n]).cumsum(0).to(DEV)


def on_gpu(kind, v, n, dy, dn, backward):
    """The same from the operators: the loss summed in float64, or the gradients."""
    v = {k: t.float().to(DEV) for k, t in v.items()}
    gy, gn, off = dy.float().to(DEV), dn.float().to(DEV), offsets_of(n)
    if kind == "norm":
        out, s = block.lbi_rms_norm(v["s"], v["w"], torch.zeros_like(v["s"]))
        grads = dict(zip("sw", block.lbi_rms_norm_backward(gy, s, v["w"], gn)))
        new = s
    elif kind == "conv":
        new = torch.empty_like(v["old"])
        out = block.lbi_ssm_conv(v["x"], v["w"], v["b"], offsets=off, state_in=v["old"],
                                 state_out=new)
        grads = dict(zip(("x", "w", "b", "old"), block.lbi_ssm_conv_backward(
            v["x"], v["w"], gy, v["b"], offsets=off, state_in=v["old"], dstate_out=gn)))
    else:
        new = torch.empty_like(v["state_in"])
        out = block.lbi_ssm_scan(**v, offsets=off, state_out=new)
        grads = block.lbi_ssm_scan_backward(dout=gy, **v, offsets=off, dstate_out=gn) \
            if backward else {}
    if backward:
        return {k: t.cpu().double() for k, t in grads.items()}
    return (out.cpu().double() * dy).sum() + (new.cpu().double() * dn).sum()


@pytest.mark.parametrize("kind", ["norm", "conv", "scan"])
def test_differences_are_exact_enough(kind):
    v, n, dy, dn = problem(kind)
    _, grads = reference(kind, v, n, dy, dn)
    size = sum(t.square().sum() for t in grads.values()).sqrt()
    dirs = directions(v, gen(6), grads)
    want = sum((grads[k] * dirs[k]).sum() for k in v)
    got = extrapolated(lambda w: reference(kind, w, n, dy, dn)[0], v, dirs)
    assert abs(got - want) <= 1e-5 * size
    assert abs(want) > 0.3 * size


@gpu
@pytest.mark.parametrize("kind", ["norm", "conv", "scan"])
def test_gradients_against_differences(kind):
    v, n, dy, dn = problem(kind)
    v = {k: t.float().double() for k, t in v.items()}
    grads = on_gpu(kind, v, n, dy, dn, True)
    size = sum(t.square().sum() for t in grads.values()).sqrt()
    dirs = directions(v, gen(6), grads)
    want = sum((grads[k] * dirs[k]).sum() for k in v)
    got = extrapolated(lambda w: on_gpu(kind, w, n, dy, dn, False), v, dirs)
    say(f"[differences] {kind}: {abs(got - want) / size:.2g} of |gradient|")
    assert abs(got - want) <= DIFF_TOL * size


# ---- many ranges ------------------------------------------------------------------

@gpu
@pytest.mark.parametrize("lengths", [[700, 1, 0, 1400, 33, 64, 2], [4100, 31, 2500, 0, 900, 1700],
                                     [9001], [3000, 3000]], ids=str)
def test_scan_over_many_ranges(lengths):
    """Few channels and many tokens are cut into tens to hundreds of ranges, with sequences that begin
    anywhere in them; tolerances as for the short ones."""
    from test_gpu_block import call_scan, check, packing, scan_inputs

    D, N, G = 6, 5, 2
    s, g = scan_inputs(lengths, D, N, G, "f32", sum(lengths))
    T, S = sum(lengths), len(lengths)
    assert block.lbi_ssm_scan_workspace_bytes(T, S, D, N, G, "offsets" in packing(lengths)) > 0
    new = torch.full((S, D, N), float("nan"), device=DEV)
    say(f"[many ranges] {lengths}")
    y = call_scan(s, lengths, state_out=new)
    want, want_new = ref.scan(s, lengths)
    check(y, want, "y")
    check(new, want_new, "state_out")
    dout, dnew = torch.randn(T, D, generator=g).to(DEV), torch.randn(S, D, N, generator=g).to(DEV)
    got = block.lbi_ssm_scan_backward(dout=dout, dstate_out=dnew, **s, **packing(lengths))
    want = ref.scan_backward(s, lengths, dout, dnew)
    for k, e in want.items():
        check(got[k], e, k, want["delta"].norm().item() if k == "delta_bias" else None)


# ---- addresses past 32 bits ------------------------------------------------------

FAR = 1 << 23  # elements from row to row: 600 rows span 2^32 elements and more


def far_rows(t):
    out = torch.empty(t.shape[0] * FAR, dtype=t.dtype, device=DEV)
    rows = out.as_strided(t.shape, (FAR, 1))
    rows.copy_(t)
    return rows


@gpu
def test_rows_past_32_bits():
    g = gen(8)
    T, D, N = 600, 80, 8
    x = torch.randn(T, D, generator=g).bfloat16().to(DEV)
    w, cw = torch.randn(D, generator=g).to(DEV), torch.randn(D, 4, generator=g).to(DEV)
    BC = torch.randn(T, 2 * N, generator=g).bfloat16().to(DEV)
    A = -torch.rand(D, N, generator=g).to(DEV)
    far = far_rows(x)
    out = far_rows(torch.zeros_like(x))
    say("[far rows] norm")
    want, s = block.lbi_rms_norm(x, w, x)
    assert torch.equal(block.lbi_rms_norm(far, w, far, out=out)[1], s) and torch.equal(out, want)
    out.zero_()
    for a, b in zip(block.lbi_rms_norm_backward(far, far, w, ds=out),
                    block.lbi_rms_norm_backward(x, x, w)):
        assert torch.equal(a, b)
    say("[far rows] conv")
    out.zero_()
    assert torch.equal(block.lbi_ssm_conv(far, cw, out=out), block.lbi_ssm_conv(x, cw))
    out.zero_()
    for a, b in zip(block.lbi_ssm_conv_backward(far, cw, far, dx=out)[:2],
                    block.lbi_ssm_conv_backward(x, cw, x)[:2]):
        assert torch.equal(a, b)
    say("[far rows] scan")
    fBC = far_rows(BC)
    near, distant = (x, x, A, BC[:, :N], BC[:, N:]), (far, far, A, fBC[:, :N], fBC[:, N:])
    out.zero_()
    assert torch.equal(block.lbi_ssm_scan(*distant, out=out), block.lbi_ssm_scan(*near))
    out.zero_()
    a = block.lbi_ssm_scan_backward(*distant, far, outputs={"u": out})
    b = block.lbi_ssm_scan_backward(*near, x)
    for k in ("u", "delta", "A", "B", "C"):
        assert torch.equal(a[k], b[k]), k
    say("[far rows] single tokens")
    st = torch.randn(T, D, N, generator=g).to(DEV)
    sa, sb = torch.empty_like(st), torch.empty_like(st)
    out.zero_()
    assert torch.equal(block.lbi_ssm_scan_step(*distant, st, sa, out=out),
                       block.lbi_ssm_scan_step(*near, st, sb)) and torch.equal(sa, sb)


@gpu
def test_slots_past_32_bits():
    """States whose rows begin past 2^32 bytes and past 2^32 elements."""
    g = gen(9)
    D, N, rows = 4096, 64, 16500
    state = torch.empty(rows, D, N, device=DEV)
    slots = torch.tensor([rows - 1, 3, 4100, 16390], dtype=torch.int32, device=DEV)
    first = torch.randn(4, D, N, generator=g).to(DEV)
    state[slots.long()] = first
    x = torch.randn(4, D, generator=g).bfloat16().to(DEV)
    BC = torch.randn(4, 2 * N, generator=g).bfloat16().to(DEV)
    A = -torch.rand(D, N, generator=g).to(DEV)
    args = (x, x, A, BC[:, :N], BC[:, N:])
    last = torch.empty_like(first)
    want = block.lbi_ssm_scan_step(*args, first, last)
    assert torch.equal(block.lbi_ssm_scan_step(*args, state, state, slots=slots), want)
    assert torch.equal(state[slots.long()], last)
    state[slots.long()] = first
    want = block.lbi_ssm_scan(*args, sequences=4, state_in=first, state_out=last)
    assert torch.equal(block.lbi_ssm_scan(*args, sequences=4, state_in=state, state_out=state,
                                          slots=slots), want)
    assert torch.equal(state[slots.long()], last)


# ---- streams, graphs, repetition ----------------------------------------------------

def all_calls(seed=11):
    """Every operator once, on tensors of its own: a list of () -> outputs."""
    g = gen(seed)
    n = [700, 0, 3, 261]
    T, S, D, N = sum(n), len(n), 200, 16

    def r(*s, dtype=torch.bfloat16):
        return torch.randn(s, generator=g).to(dtype).to(DEV)
    f32, off = torch.float32, offsets_of(n)
    x, dy, w, cw, cb = r(T, D), r(T, D), r(D, dtype=f32), r(D, 4, dtype=f32), r(D, dtype=f32)
    args = (x, r(T, D), -torch.rand(D, N, generator=g).to(DEV), r(T, 2, N), r(T, 2, N))
    rest = {"skip": w, "z": r(T, D), "delta_bias": cb, "offsets": off, "state_in": r(S, D, N, dtype=f32)}
    one = tuple(t if t.shape[0] == D else t[:S] for t in args)
    cs, c_new, s_new, s_one = r(S, 3, D), r(S, 3, D), r(S, D, N, dtype=f32), r(S, D, N, dtype=f32)
    return [
        ("norm", lambda: block.lbi_rms_norm(x, w, dy)),
        ("norm q8", lambda: block.lbi_rms_norm_q8(x, w, group=64)[:2]),
        ("norm backward", lambda: block.lbi_rms_norm_backward(dy, x, w)),
        ("conv", lambda: (block.lbi_ssm_conv(x, cw, cb, offsets=off, state_in=cs, state_out=c_new),
                          c_new)),
        ("conv backward", lambda: block.lbi_ssm_conv_backward(x, cw, dy, cb, offsets=off,
                                                              state_in=cs)),
        ("conv step", lambda: (block.lbi_ssm_conv_step(x[:S], cw, cs, c_new, cb), c_new)),
        ("scan", lambda: (block.lbi_ssm_scan(*args, **rest, state_out=s_new), s_new)),
        ("scan backward", lambda: tuple(block.lbi_ssm_scan_backward(*args, dy, **rest).values())),
        ("scan step", lambda: (block.lbi_ssm_scan_step(*one, rest["state_in"], s_one), s_one)),
    ]


def kept(outputs):
    return [t.view(torch.uint8).clone() if t.element_size() == 1 else t.clone()
            for t in outputs if t is not None]


def equal(outputs, want):
    got = kept(outputs)
    return len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))


@gpu
def test_results_do_not_change_and_other_streams():
    calls = all_calls()
    want = [kept(f()) for _, f in calls]
    torch.cuda.synchronize()
    for (name, f), w in zip(calls, want):
        for _ in range(3):
            assert equal(f(), w), name
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = [kept(f()) for _, f in calls]
    side.synchronize()
    for (name, _), a, w in zip(calls, again, want):
        assert all(torch.equal(p, q) for p, q in zip(a, w)), name
    # a stream given by name: the call sees what that stream's earlier work left
    x = torch.zeros(1 << 24, device=DEV).view(4096, 4096)
    w1, zeros = torch.ones(4096, device=DEV), torch.zeros_like(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(50):
            x.add_(1.0)
    out, s = torch.empty_like(x), torch.empty_like(x)
    block.lbi_rms_norm(x, w1, zeros, out=out, residual_out=s, stream=side)
    side.synchronize()
    assert (s == 50).all()


@gpu
def test_calls_replay_in_a_graph():
    calls = all_calls()
    want = [kept(f()) for _, f in calls]
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph):
            outs = [f() for _, f in calls]
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    other = all_calls(seed=12)
    for rep in range(3):
        for o in outs:
            for t in o:
                if t is not None:
                    t.view(torch.uint8).fill_(255)
        for _, f in other:  # eager work between the replays
            f()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        # calls that share a tensor for the last states are compared by their first outputs
        for (name, _), o, w in zip(calls, outs, want):
            if name == "conv":
                o, w = o[:1], w[:1]
            assert equal(o, w), f"replay {rep}: {name}"
        say(f"[graph] replay {rep}: {len(calls)} calls equal to the eager results")


# ---- refusals and the example ---------------------------------------------------------

@gpu
def test_binding_refusals():
    x = torch.zeros(6, 8, device=DEV)
    w, cw, A = torch.ones(8, device=DEV), torch.ones(8, 4, device=DEV), -torch.ones(8, 2, device=DEV)
    B = torch.zeros(6, 2, device=DEV)
    wrong = [
        lambda: block.lbi_rms_norm(x, w[:4]), lambda: block.lbi_rms_norm(x, w.double()),
        lambda: block.lbi_rms_norm(x, w, out=x.bfloat16()),
        lambda: block.lbi_rms_norm(x, w, residual_out=x.clone()),
        lambda: block.lbi_rms_norm(x.t(), torch.ones(6, device=DEV)),
        lambda: block.lbi_rms_norm_q8(x, w, format=7),
        lambda: block.lbi_ssm_conv(x, cw, offsets=torch.zeros(0, dtype=torch.int64, device=DEV)),
        lambda: block.lbi_ssm_conv(x, cw, offsets=torch.tensor([0, 6])),
        lambda: block.lbi_ssm_conv(x, cw, offsets=torch.tensor([0, 6], dtype=torch.int32).to(DEV)),
        lambda: block.lbi_ssm_conv(x, cw, state_in=torch.zeros(1, 4, 8, device=DEV)),
        lambda: block.lbi_ssm_conv(x.view(2, 3, 8), cw, sequences=3),
        lambda: block.lbi_ssm_conv_step(x.view(2, 3, 8), cw, x, x),
        lambda: block.lbi_ssm_scan(x, x, A, B, B[:5]),
        lambda: block.lbi_ssm_scan(x, x, A, B, B.view(6, 1, 2).expand(6, 2, 2)),
        lambda: block.lbi_ssm_scan(x, x, A, B.bfloat16(), B),
        lambda: block.lbi_ssm_scan(x, x, A, B, B, z=x[:5]),
        lambda: block.lbi_ssm_scan(x, x, A, B, B, state_in=torch.zeros(1, 8, 3, device=DEV)),
        lambda: block.lbi_ssm_scan_backward(x, x, A, B, B, x, outputs={"skip": w}),
    ]
    for i, call in enumerate(wrong):
        with pytest.raises((ValueError, TypeError)):
            call()
            pytest.fail(f"case {i} was taken")
    with pytest.raises(TypeError):
        block.lbi_rms_norm(x.half(), w)
    refused = [
        lambda: block.lbi_rms_norm(x, w, out=x),
        lambda: block.lbi_rms_norm(x, w, eps=-1.0),
        lambda: block.lbi_rms_norm_q8(x, w, group=24),
        lambda: block.lbi_ssm_conv(x, cw[:, :1].contiguous()),
        lambda: block.lbi_ssm_conv(x, cw, sequences=4),
        lambda: block.lbi_ssm_conv(x[:1].expand(6, 8), cw),
        lambda: block.lbi_ssm_scan(x, x, A, B, B, out=x),
    ]
    for i, call in enumerate(refused):
        with pytest.raises(binding.LbiError):
            call()
            pytest.fail(f"case {i} was taken")
    torch.cuda.synchronize()


@gpu
def test_example():
    """The interface scan's gradients and the chain's take the operators' float32 results, 1e-5
    each, through six operators of six regions: 4e-4.  Served tokens differ by bf16 roundings
    of the products' sums and what they turn over in 8 bits: 2e-2, the block's bound elsewhere."""
    from examples import region_block

    diff = region_block.train()
    say(f"[example] training: {diff:.2g}")
    assert diff <= 4e-4
    diff = region_block.serve()
    say(f"[example] serving: {diff:.2g}")
    assert diff <= 2e-2
