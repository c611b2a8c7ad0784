"""The operators of include/lbi_linear.h as a program uses them (needs a GPU): gradients against
differences of the operators' own outputs, many ranges, addresses past 32 bits, other streams, replays
in graphs, shared workspaces, many sequences, refusals, and the example.

Differences: a central difference along one direction v, |v| = 1, with the steps 2^-3 and 2^-4
extrapolated.  What the extrapolation leaves is under 1e-5 of |gradient| for these sizes (held on
the CPU, in float64, by test_differences_are_exact_enough); the outputs' float32 errors, 1e-7 of
|cotangent| |outputs| with |outputs| under 20 |gradient|, divided by the step, add some 2e-5.
The bound is 1e-3 of |gradient|.
"""
import sys

import pytest
import torch

from oracle import linear as ref
from paper_2605_09204_amd import binding, linear

gpu = pytest.mark.gpu
DEV = "cuda:0"
DIFF_TOL = 1e-3
SILU = linear.LBI_ACT_SILU


def say(msg):
    print(msg, flush=True)
    sys.stdout.flush()


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def offsets_of(n):
    return torch.tensor([0, *n]).cumsum(0).to(DEV)


# ---- differences -----------------------------------------------------------------

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
    n = [21, 0, 1, 68]
    T, S, H, KH, DK, DV = sum(n), len(n), 4, 2, 6, 5

    def r(*s):
        return torch.randn(s, generator=g).double()
    if kind == "norm":
        return {"s": r(T, 40), "w": r(40), "b": r(40)}, n, r(T, 40), r(T, 40)
    if kind == "projection":
        return {"x": r(T, 12), "w": r(9, 12), "b": r(9)}, n, r(T, 9), None
    return {"q": r(T, H, DK), "k": r(T, KH, DK), "v": r(T, KH, DV), "log_decay": -0.2 - r(H).abs(),
            "state_in": r(S, H, DK, DV)}, n, r(T, H, DV), r(S, H, DK, DV)


def reference(kind, v, n, dy, dn):
    """(loss, gradients) in float64."""
    if kind == "norm":
        out, s = ref.layer_norm(v["s"], v["w"], v["b"])
        ds, dw, db = ref.layer_norm_backward(dy, v["s"], v["w"])
        return (out * dy).sum() + (s * dn).sum(), {"s": ds + dn, "w": dw, "b": db}
    if kind == "projection":
        out, pre = ref.projection(v["x"], v["w"], v["b"], "silu")
        dx, dw, db, _ = ref.projection_backward(v["x"], v["w"], dy, "silu", pre)
        return (out * dy).sum(), {"x": dx, "w": dw, "b": db}
    a = (v["q"], v["k"], v["v"], v["log_decay"], 0.4, n)
    y, new = ref.attention(*a, v["state_in"])
    return (y * dy).sum() + (new * dn).sum(), ref.attention_backward(*a, dy, v["state_in"], dn)


def on_gpu(kind, v, n, dy, dn, backward):
    """The same from the operators: the loss summed in float64, or the gradients."""
    v = {k: t.float().to(DEV) for k, t in v.items()}
    gy, gn = dy.float().to(DEV), None if dn is None else dn.float().to(DEV)
    new = None
    if kind == "norm":
        out, new = linear.lbi_layer_norm(v["s"], v["w"], v["b"], torch.zeros_like(v["s"]))
        grads = dict(zip("swb", linear.lbi_layer_norm_backward(gy, new, v["w"], gn)))
    elif kind == "projection":
        pre = torch.empty_like(gy)
        out = linear.lbi_projection(v["x"], v["w"], v["b"], SILU, pre=pre)
        grads = dict(zip("xwb", linear.lbi_projection_backward(v["x"], v["w"], gy, SILU, pre)))
    else:
        a, kw = (v["q"], v["k"], v["v"], v["log_decay"]), {"offsets": offsets_of(n),
                                                          "state_in": v["state_in"]}
        new = torch.empty_like(v["state_in"])
        out = linear.lbi_linear_attention(*a, 0.4, state_out=new, **kw)
        grads = linear.lbi_linear_attention_backward(*a, gy, 0.4, dstate_out=gn, **kw)
    if backward:
        return {k: t.cpu().double() for k, t in grads.items()}
    loss = (out.cpu().double() * dy).sum()
    return loss if dn is None else loss + (new.cpu().double() * dn).sum()


@pytest.mark.parametrize("kind", ["norm", "projection", "attention"])
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
@pytest.mark.parametrize("kind", ["norm", "projection", "attention"])
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
@pytest.mark.parametrize("lengths", [[700, 1, 0, 1400, 33, 64, 2], [4100, 31, 1500, 0, 900],
                                     [5001], [3000, 3000], [64] * 40], ids=str)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention_over_many_ranges(lengths, dtype):
    """One head and many tokens are cut into tens of ranges, with sequences that begin anywhere in them;
    tolerances as for the short ones."""
    from test_gpu_linear import args_of, attention_inputs, check, packing

    H, DK, DV = 1, 12, 20
    s, g = attention_inputs(lengths, H, 1, DK, DV, dtype, sum(lengths))
    scale = DK ** -0.5
    say(f"[many ranges] {lengths} {dtype}")
    dout = torch.randn(sum(lengths), H, DV, generator=g).to(s["q"].dtype).to(DEV)
    dnew = torch.randn(s["state"].shape, generator=g).to(DEV)
    terms = ref.attention_terms(*args_of(s), scale, lengths, dout)
    bf16 = dtype == "bf16"
    want, want_new = ref.attention(*args_of(s), scale, lengths, s["state"])
    state = s["state"].clone()
    y = linear.lbi_linear_attention(*args_of(s), state_in=state, state_out=state, **packing(lengths))
    check(y, want, "out", terms["out"] if bf16 else None, terms["out"].norm().item())
    check(state, want_new, "state in place")
    got = linear.lbi_linear_attention_backward(*args_of(s), dout, state_in=s["state"],
                                               dstate_out=dnew, **packing(lengths))
    want = ref.attention_backward(*args_of(s), scale, lengths, dout, s["state"], dnew)
    for k in ("q", "k", "v"):
        check(got[k], want[k], k, terms[k] if bf16 else None, terms[k].norm().item())
    check(got["state_in"], want["state_in"], "state_in", floor=dout.float().norm().item())
    floor = (s["q"].double().cpu() * want["q"]).norm().item() \
        / (1 - torch.exp(s["log_decay"].double())).min().item() \
        + dnew.norm().item() * s["state"].norm().item()
    check(got["log_decay"], want["log_decay"], "log_decay", floor=floor)


# ---- addresses past 32 bits --------------------------------------------------------

FAR = 1 << 23  # elements from row to row: 600 rows span 2^32 elements and more


def far_rows(t):
    flat = t.flatten(1)
    out = torch.empty(t.shape[0] * FAR, dtype=t.dtype, device=DEV)
    rows = out.as_strided(flat.shape, (FAR, 1))
    rows.copy_(flat)
    return rows.unflatten(1, t.shape[1:]) if t.dim() > 2 else rows


@gpu
def test_rows_past_32_bits():
    g = gen(8)
    T, D, H, DK, DV = 600, 80, 2, 16, 24
    x = torch.randn(T, D, generator=g).bfloat16().to(DEV)
    w, b = torch.randn(D, generator=g).to(DEV), torch.randn(D, generator=g).to(DEV)
    far, out = far_rows(x), far_rows(torch.zeros_like(x))
    say("[far rows] layer norm")
    want = linear.lbi_layer_norm(x, w, b, x)
    got = linear.lbi_layer_norm(far, w, b, far, out=out)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for p, q in zip(linear.lbi_layer_norm_backward(far, far, w, ds=out),
                    linear.lbi_layer_norm_backward(x, x, w)):
        assert torch.equal(p, q)
    say("[far rows] projection")
    m = torch.randn(D, D, generator=g).bfloat16().to(DEV)
    pre, fpre = torch.empty_like(x), far_rows(torch.zeros_like(x))
    want = linear.lbi_projection(x, m, b, SILU, x, pre=pre)
    # rows this far apart go through registers, the dense ones straight into LDS: the same sums
    got = linear.lbi_projection(far, m, b, SILU, far, out=out, pre=fpre)
    assert torch.equal(got, want) and torch.equal(fpre, pre)
    for p, q in zip(linear.lbi_projection_backward(far, m, far, SILU, fpre, dx=out),
                    linear.lbi_projection_backward(x, m, x, SILU, pre)):
        assert torch.equal(p, q)
    say("[far rows] attention")
    q, k, v = (torch.randn(T, n, d, generator=g).bfloat16().to(DEV)
               for n, d in ((H, DK), (1, DK), (1, DV)))
    ld = -torch.rand(H, generator=g).to(DEV)
    dout = torch.randn(T, H, DV, generator=g).bfloat16().to(DEV)
    fq, fk, fv, fd = (far_rows(t) for t in (q, k, v, dout))
    fo = far_rows(torch.zeros_like(dout))
    assert torch.equal(linear.lbi_linear_attention(fq, fk, fv, ld, out=fo),
                       linear.lbi_linear_attention(q, k, v, ld))
    want = linear.lbi_linear_attention_backward(q, k, v, ld, dout)
    del out, far, fpre
    fg = far_rows(torch.zeros_like(q))
    got = linear.lbi_linear_attention_backward(fq, fk, fv, ld, fd, outputs={"q": fg})
    for n in ("q", "k", "v", "log_decay"):
        assert torch.equal(got[n], want[n]), n
    say("[far rows] single tokens")
    st = torch.randn(T, H, DK, DV, generator=g).to(DEV)
    sa, sb = torch.empty_like(st), torch.empty_like(st)
    assert torch.equal(linear.lbi_linear_attention_step(fq, fk, fv, ld, st, sa, out=fo),
                       linear.lbi_linear_attention_step(q, k, v, ld, st, sb))
    assert torch.equal(sa, sb)
    with pytest.raises(binding.LbiError):  # one element further is refused
        linear.lbi_linear_attention(torch.empty(FAR + 1 + H * DK, dtype=torch.bfloat16, device=DEV)
                                    .as_strided((2, H, DK), (FAR + 1, DK, 1)), k[:2], v[:2], ld)


@gpu
def test_slots_past_32_bits():
    """States whose rows begin past 2^32 bytes and past 2^32 elements."""
    g = gen(9)
    H, DK, DV, rows = 16, 128, 128, 16500
    state = torch.empty(rows, H, DK, DV, device=DEV)
    slots = torch.tensor([rows - 1, 3, 4100, 16390], dtype=torch.int32, device=DEV)
    first = torch.randn(4, H, DK, DV, generator=g).to(DEV)
    state[slots.long()] = first
    q, k, v = (torch.randn(4, n, 128, generator=g).bfloat16().to(DEV) for n in (H, 4, 4))
    ld = -torch.rand(H, generator=g).to(DEV)
    last = torch.empty_like(first)
    want = linear.lbi_linear_attention_step(q, k, v, ld, first, last)
    assert torch.equal(linear.lbi_linear_attention_step(q, k, v, ld, state, state, slots=slots), want)
    assert torch.equal(state[slots.long()], last)
    state[slots.long()] = first
    want = linear.lbi_linear_attention(q, k, v, ld, sequences=4, state_in=first, state_out=last)
    assert torch.equal(linear.lbi_linear_attention(q, k, v, ld, sequences=4, state_in=state,
                                                   state_out=state, slots=slots), want)
    assert torch.equal(state[slots.long()], last)


@gpu
def test_many_sequences():
    """70000 of one token, and 300000 of none between them."""
    g = gen(10)
    n, H, DK, DV = 70000, 1, 4, 8
    q, k, v = (torch.randn(n, H, d, generator=g).to(DEV) for d in (DK, DK, DV))
    ld = torch.full((H,), -0.1, device=DEV)
    y = linear.lbi_linear_attention(q, k, v, ld, 1.0, sequences=n)
    want = ((q * k).sum(-1, keepdim=True) * v)
    assert (y - want).norm() <= 1e-5 * want.norm()
    lengths = torch.zeros(370000, dtype=torch.int64)
    lengths[torch.randperm(370000, generator=g)[:n]] = 1
    off = torch.cat([torch.zeros(1, dtype=torch.int64), lengths.cumsum(0)]).to(DEV)
    old = torch.randn(370000, H, DK, DV, generator=g).to(DEV)
    new = torch.full_like(old, float("nan"))
    y = linear.lbi_linear_attention(q, k, v, ld, 1.0, offsets=off, state_in=old, state_out=new)
    one = (lengths == 1).to(DEV)
    assert torch.equal(new[~one], old[~one])
    s = torch.exp(ld)[0] * old[one] + k[..., None] * v[..., None, :]
    assert (new[one] - s).norm() <= 1e-5 * s.norm()
    want = (q[..., None] * s).sum(2)
    assert (y - want).norm() <= 1e-5 * want.norm()
    got = linear.lbi_linear_attention_backward(q, k, v, ld, v, 1.0, offsets=off, state_in=old,
                                               dstate_out=old)
    assert torch.equal(got["state_in"][~one], old[~one])
    G = old[one] + q[..., None] * v[..., None, :]
    assert (got["state_in"][one] - torch.exp(ld)[0] * G).norm() <= 1e-5 * G.norm()
    assert (got["k"] - (G * v[..., None, :]).sum(-1)).norm() <= 1e-5 * G.norm()


@gpu
def test_no_tokens():
    """Calls without tokens, and without sequences, leave states and zero gradients of parameters."""
    q, k, v = (torch.zeros(0, 2, d, device=DEV) for d in (8, 8, 4))
    ld, st = -torch.ones(2, device=DEV), torch.randn(3, 2, 8, 4, device=DEV)
    new = torch.full_like(st, float("nan"))
    for kw in ({"sequences": 3}, {"offsets": torch.zeros(4, dtype=torch.int64, device=DEV)}):
        y = linear.lbi_linear_attention(q, k, v, ld, state_in=st, state_out=new, **kw)
        assert y.shape == (0, 2, 4) and torch.equal(new, st)
        g = linear.lbi_linear_attention_backward(q, k, v, ld, y, state_in=st, dstate_out=st, **kw)
        assert torch.equal(g["state_in"], st) and (g["log_decay"] == 0).all()
    linear.lbi_linear_attention(q, k, v, ld, state_out=new, sequences=3)
    assert (new == 0).all()
    g = linear.lbi_linear_attention_backward(q, k, v, ld, y, sequences=0)
    assert (g["log_decay"] == 0).all()
    x = torch.zeros(0, 16, device=DEV)
    assert linear.lbi_layer_norm(x)[0].shape == (0, 16)
    assert all((t == 0).all() for t in linear.lbi_layer_norm_backward(x, x)[1:])
    assert linear.lbi_projection(x, torch.ones(4, 16, device=DEV)).shape == (0, 4)
    torch.cuda.synchronize()


# ---- streams, graphs, repetition -----------------------------------------------------

def all_calls(seed=11, lengths=(700, 0, 3, 261)):
    """Every operator, on tensors of its own: (name, call with keyword arguments -> outputs, workspace
    bytes)."""
    g = gen(seed)
    n = list(lengths)
    T, S, D, H, KH, DK, DV = sum(n), len(n), 200, 4, 2, 64, 32

    def r(*s, dtype=torch.bfloat16):
        return torch.randn(s, generator=g).to(dtype).to(DEV)
    f32, off = torch.float32, offsets_of(n)
    x, dy, w, b = r(T, D), r(T, D), r(D, dtype=f32), r(D, dtype=f32)
    m, long, wide = r(D, D), r(100, 8000), r(96, 8000)
    pre, pre_out = r(T, D), torch.empty(T, D, dtype=torch.bfloat16, device=DEV)
    a = (r(T, H, DK), r(T, KH, DK), r(T, KH, DV), -torch.rand(H, generator=g).to(DEV))
    dout, st, dst = r(T, H, DV), r(S, H, DK, DV, dtype=f32), r(S, H, DK, DV, dtype=f32)
    new, one = torch.empty_like(st), torch.empty_like(st)
    sizes = (T, S, H, KH, DK, DV, True, torch.bfloat16)
    bf = torch.bfloat16
    return [
        ("norm", lambda **k: linear.lbi_layer_norm(x, w, b, dy, **k), 0),
        ("norm backward", lambda **k: linear.lbi_layer_norm_backward(dy, x, w, **k),
         linear.lbi_layer_norm_backward_workspace_bytes(T, D)),
        ("projection", lambda **k: (linear.lbi_projection(x, m, b, SILU, dy, pre=pre_out, **k),
                                    pre_out), linear.lbi_projection_workspace_bytes(T, D, D, bf)),
        ("projection in parts", lambda **k: (linear.lbi_projection(long, wide, **k),),
         linear.lbi_projection_workspace_bytes(100, 8000, 96, bf)),
        ("projection backward", lambda **k: linear.lbi_projection_backward(x, m, dy, SILU, pre, **k),
         linear.lbi_projection_backward_workspace_bytes(T, D, D, SILU, bf, bf)),
        ("attention", lambda **k: (linear.lbi_linear_attention(*a, offsets=off, state_in=st,
                                                               state_out=new, **k), new),
         linear.lbi_linear_attention_workspace_bytes(*sizes)),
        ("attention backward", lambda **k: tuple(linear.lbi_linear_attention_backward(
            *a, dout, offsets=off, state_in=st, dstate_out=dst, **k).values()),
         linear.lbi_linear_attention_backward_workspace_bytes(*sizes)),
        ("attention step", lambda **k: (linear.lbi_linear_attention_step(
            *(t[:S] for t in a[:3]), a[3], st, one, **k), one), 0),
    ]


def kept(outputs):
    return [t.clone() for t in outputs if t is not None]


def equal(outputs, want):
    got = [t for t in outputs if t is not None]
    return len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))


@gpu
def test_results_do_not_change_and_other_streams():
    calls = all_calls()
    want = [kept(f()) for _, f, _ in calls]
    assert sum(need > 0 for _, _, need in calls) >= 5
    torch.cuda.synchronize()
    for (name, f, _), w in zip(calls, want):
        for _ in range(3):
            assert equal(f(), w), name
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = [kept(f()) for _, f, _ in calls]
    side.synchronize()
    for (name, _, _), a, w in zip(calls, again, want):
        assert all(torch.equal(p, q) for p, q in zip(a, w)), name
    # on a given stream: two calls at once, each with memory of its own stream
    for (name, f, _), w in zip(calls, want):
        here = f()
        there = f(stream=side) if name not in ("projection", "attention", "attention step") else here
        torch.cuda.synchronize()
        assert equal(here, w) and equal(there, w), name
    for name in ("projection", "attention", "attention step"):  # these share an output
        f, w = next((f, w) for (n, f, _), w in zip(calls, want) if n == name)
        got = f(stream=side.cuda_stream)
        torch.cuda.synchronize()
        assert equal(got, w), name


@gpu
def test_calls_replay_in_a_graph():
    calls = all_calls()
    want = [kept(f()) for _, f, _ in calls]
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph):
            outs = [f() for _, f, _ in calls]
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    other = all_calls(seed=12)
    for rep in range(3):
        for o in outs:
            for t in o:
                if t is not None:
                    t.view(torch.uint8).fill_(255)
        for _, f, _ in other:  # eager work between the replays
            f()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for (name, _, _), o, w in zip(calls, outs, want):
            assert equal(o, w), f"replay {rep}: {name}"
        say(f"[graph] replay {rep}: {len(calls)} calls equal to the eager results")


@gpu
def test_two_graphs_share_a_workspace():
    """Replays one after the other, in both orders: nothing is kept in a workspace between calls."""
    first, second = all_calls(seed=13), all_calls(seed=14, lengths=(5, 600, 1, 90))
    names = [n for n, _, need in first if need > 0]
    need = max(need for calls in (first, second) for _, _, need in calls)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    graphs = []
    for calls in (first, second):
        calls = [(n, f) for n, f, need in calls if n in names]
        want = [kept(f()) for _, f in calls]
        torch.cuda.synchronize()
        graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            with torch.cuda.graph(graph):
                outs = [f(workspace=ws) for _, f in calls]
        torch.cuda.synchronize()
        graphs.append((graph, outs, want))
    for order in ((0, 1), (1, 0), (0, 0), (1, 1)):
        ws.fill_(255)
        for i in order:
            graphs[i][0].replay()
            torch.cuda.synchronize()
            for name, o, w in zip(names, graphs[i][1], graphs[i][2]):
                assert equal(o, w), (order, name)


@gpu
@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two GPUs")
def test_tensors_on_another_device():
    x = torch.randn(6, 8)
    want = linear.lbi_layer_norm(x.to(DEV))[0].cpu()
    with torch.cuda.device(0):
        got = linear.lbi_layer_norm(x.to("cuda:1"))[0]
        assert torch.cuda.current_device() == 0
    assert got.device.index == 1 and torch.equal(got.cpu(), want)


# ---- refusals and the example -----------------------------------------------------------

@gpu
def test_binding_refusals():
    x, w = torch.zeros(6, 8, device=DEV), torch.ones(8, device=DEV)
    m = torch.ones(4, 8, device=DEV)
    q = torch.zeros(6, 2, 4, device=DEV)
    ld, st = -torch.ones(2, device=DEV), torch.zeros(1, 2, 4, 4, device=DEV)
    att, back = linear.lbi_linear_attention, linear.lbi_linear_attention_backward
    wrong = [
        lambda: linear.lbi_layer_norm(x, w[:4]), lambda: linear.lbi_layer_norm(x, w, w.double()),
        lambda: linear.lbi_layer_norm(x, out=x.bfloat16()),
        lambda: linear.lbi_layer_norm(x, residual_out=x.clone()),
        lambda: linear.lbi_projection(x, m.t()), lambda: linear.lbi_projection(x, m.bfloat16()),
        lambda: linear.lbi_projection(x, m[0]), lambda: linear.lbi_projection(x, m, w),
        lambda: linear.lbi_projection(x, m, act=5), lambda: linear.lbi_projection(x, m, residual=x),
        lambda: linear.lbi_projection(x, m, pre=torch.zeros(6, 4, device=DEV).bfloat16()),
        lambda: linear.lbi_projection_backward(x, m, x),
        lambda: linear.lbi_projection_backward(x, m, x[:, :4].contiguous(), dweight=m.double()),
        lambda: att(q, q, q, ld[:1]), lambda: att(q, q[:5], q, ld), lambda: att(q, q.bfloat16(), q, ld),
        lambda: att(q, q[..., :3].contiguous(), q, ld), lambda: att(q, q, q[:, :1], ld),
        lambda: att(q, q, q[..., :2], ld),  # the heads' values do not lie side by side
        lambda: att(q, q, q, ld, offsets=torch.tensor([0, 6])),
        lambda: att(q, q, q, ld, state_in=st[..., :3].contiguous()),
        lambda: att(q.view(2, 3, 2, 4), q.view(2, 3, 2, 4), q.view(2, 3, 2, 4), ld, sequences=3),
        lambda: back(q, q, q, ld, q, outputs={"dq": q}),
        lambda: back(q, q, q, ld, q, outputs={"state_in": st}),
        lambda: back(q, q, q, ld, q[..., :2].contiguous()),
        lambda: linear.lbi_linear_attention_step(q.view(2, 3, 2, 4), q, q, ld, st, st),
    ]
    for i, call in enumerate(wrong):
        with pytest.raises((ValueError, TypeError)):
            call()
            pytest.fail(f"case {i} was taken")
    refused = [
        lambda: linear.lbi_layer_norm(x, out=x), lambda: linear.lbi_layer_norm(x, eps=-1.0),
        lambda: linear.lbi_projection(x, torch.ones(8, 8, device=DEV), out=x),
        lambda: linear.lbi_projection(x[:1].expand(6, 8), m),
        lambda: linear.lbi_projection_backward(x, m, x[:, :4].contiguous(), linear.LBI_ACT_SILU),
        lambda: att(q, q, q, ld, sequences=4), lambda: att(q, q, q, ld, out=q),
        lambda: att(q, torch.cat([q, q], 1), torch.cat([q, q], 1), ld),  # more keys than queries
        lambda: att(*(torch.zeros(2, 1, 129, device=DEV) for _ in range(3)), ld[:1]),
    ]
    for i, call in enumerate(refused):
        with pytest.raises(binding.LbiError):
            call()
            pytest.fail(f"case {i} was taken")
    torch.cuda.synchronize()


@gpu
def test_example():
    """The interface scan's gradients and the chain's take the operators' float32 results, 1e-5 each,
    through eight operators of five regions: 4e-4.  Served tokens differ by bf16 roundings inside,
    five of them in a row, 2^-8 each: 2e-2, the block's bound elsewhere."""
    from examples import attention_block

    diff = attention_block.train()
    say(f"[example] training: {diff:.2g}")
    assert diff <= 4e-4
    diff = attention_block.serve()
    say(f"[example] serving: {diff:.2g}")
    assert diff <= 2e-2


@gpu
def test_heads_without_values_are_refused():
    q = torch.zeros(5, 1, 0, dtype=torch.bfloat16, device=DEV)
    v, decay = torch.zeros(5, 1, 4, dtype=torch.bfloat16, device=DEV), torch.zeros(1, device=DEV)
    with pytest.raises(binding.LbiError):
        linear.lbi_linear_attention(q, q, v, decay)
    with pytest.raises(binding.LbiError):
        linear.lbi_linear_attention_backward(q, q, v, decay, v)
