"""The calls of a state-space region block whose speed this library is held to.

A region transformation of the state-space kind is, between its projections,
three operators: the root-mean-square norm that joins the residual stream, the
short causal convolution along the tokens, and the selective scan, a diagonal
linear recurrence whose decay depends on the token:

    s = x + residual,  out = s / sqrt(mean(s^2) + eps) * weight
    out_t = silu(bias + sum_w weight_w x_{t - W + 1 + w})
    h_t = exp(D_t A) h_{t-1} + D_t u_t B_t,  y_t = (C_t . h_t + skip u_t) silu(z_t)

with D_t = softplus(delta_t + delta_bias).  Each case is one call as a training
step, a prompt pass or a single decoded token makes it.  Shapes follow the
block of this repository's Phase 1 workload (B = 8 sequences of L = 2048 tokens,
D = 768 features, the inner width twice that).
"""
import math

import torch

own = False

EPS = 1e-5
STORE = {"f32": torch.float32, "bf16": torch.bfloat16}
MAX_STATES = 8 * 2048 * 1536 * 16  # T D N of a drawn scan
MAX_WIDTH = 8 * 2048 * 1536  # T D of a drawn norm or convolution


def listed():
    return [
        # the norm at a block's entry in a training step, with the residual stream's addition
        {"name": "norm_tokens", "op": "norm", "dtype": "bf16", "stream": "bf16", "T": 16384,
         "D": 768, "residual": True},
        # a prompt's norm that feeds an 8-bit projection: an odd number of tokens, scales per 128
        {"name": "norm_q8_prompt", "op": "norm_q8", "dtype": "bf16", "stream": "bf16", "T": 4099,
         "D": 2048, "residual": True, "format": "e4m3", "group": 128},
        # the norm's gradient, joined with the gradient that comes along the residual stream
        {"name": "norm_backward", "op": "norm_backward", "dtype": "bf16", "stream": "bf16",
         "T": 16384, "D": 768, "residual": True},
        # the convolution over packed prompts of different lengths, each with its own past tokens
        {"name": "conv_prompts", "op": "conv", "dtype": "bf16", "B": 13, "T": 8201, "D": 1536,
         "W": 4, "ragged": True, "states": True},
        # the convolution's gradients in a training step
        {"name": "conv_backward", "op": "conv_backward", "dtype": "bf16", "B": 8, "T": 16384,
         "D": 1536, "W": 4, "ragged": False, "states": False},
        # one decoded token for each of 64 requests
        {"name": "conv_step", "op": "conv_step", "dtype": "bf16", "B": 64, "T": 64, "D": 1536,
         "W": 4},
        # the scan of a training step
        {"name": "scan_train", "op": "scan", "dtype": "bf16", "B": 8, "T": 16384, "D": 1536,
         "N": 16, "G": 1, "ragged": False, "states": False, "gated": True},
        # the scan over packed prompts of different lengths, from kept states to new ones
        {"name": "scan_prompts", "op": "scan", "dtype": "bf16", "B": 13, "T": 8201, "D": 1536,
         "N": 16, "G": 1, "ragged": True, "states": True, "gated": True},
        # one long sequence in float32: parallel only along the tokens
        {"name": "scan_long", "op": "scan", "dtype": "f32", "B": 1, "T": 32768, "D": 768,
         "N": 16, "G": 1, "ragged": False, "states": True, "gated": False},
        # the scan's gradients in a training step
        {"name": "scan_backward", "op": "scan_backward", "dtype": "bf16", "B": 8, "T": 16384,
         "D": 1536, "N": 16, "G": 1, "ragged": False, "states": False, "gated": True},
        # the gradients at odd sizes, float32, two groups, states passed from part to part
        {"name": "scan_backward_odd", "op": "scan_backward", "dtype": "f32", "B": 5, "T": 3885,
         "D": 202, "N": 12, "G": 2, "ragged": True, "states": True, "gated": True},
        # one decoded token for each of 64 requests
        {"name": "scan_step", "op": "scan_step", "dtype": "bf16", "B": 64, "T": 64, "D": 1536,
         "N": 16, "G": 1, "gated": True},
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)) - 1e-9)))))


def draw(rng):
    most = {k: max(work(c)[k] for c in listed()) for k in ("bytes", "flops")}
    while True:
        c = _draw(rng)
        if all(work(c)[k] <= most[k] for k in most):
            return c


def _draw(rng):
    op = rng.choice(["norm", "norm_q8", "norm_backward", "conv", "conv_backward", "conv_step",
                     "scan", "scan", "scan_backward", "scan_backward", "scan_step"])
    c = {"op": op, "dtype": rng.choice(["f32", "bf16", "bf16"])}
    if op.startswith("norm"):
        while True:
            c |= {"T": _log(rng, 1, 32768), "D": _log(rng, 16, 8192)}
            if rng.random() < 0.6:  # most widths are whole vectors
                c["D"] = max(16, c["D"] // 16 * 16)
            if c["T"] * c["D"] <= MAX_WIDTH // 2:
                break
        c |= {"stream": rng.choice([c["dtype"], "f32"]), "residual": rng.random() < 0.7}
        if op == "norm_q8":
            c |= {"format": rng.choice(["e4m3", "int8"]), "group": rng.choice([0, 32, 64, 128])}
        return c
    while True:
        c |= {"T": _log(rng, 1, 32768), "D": _log(rng, 16, 4096)}
        if rng.random() < 0.6:
            c["D"] = max(16, c["D"] // 16 * 16)
        if c["T"] * c["D"] <= MAX_WIDTH:
            break
    if op.endswith("step"):
        c["T"] = c["B"] = max(1, min(c["T"], 512))
    else:
        c["B"] = _log(rng, 1, min(64, c["T"]))
        c |= {"ragged": rng.random() < 0.5, "states": rng.random() < 0.5}
        if not c["ragged"]:
            c["T"] = c["T"] // c["B"] * c["B"]
    if op.startswith("conv"):
        return c | {"W": rng.randint(2, 4)}
    c |= {"N": rng.choice([1, 4, 8, 12, 16, 16, 16, 24, 32, 64]), "gated": rng.random() < 0.7}
    c["G"] = rng.choice([g for g in (1, 1, 2, 4) if c["D"] % g == 0])
    most = {"scan": MAX_STATES, "scan_backward": MAX_STATES // 2, "scan_step": MAX_STATES // 16}[op]
    if c["T"] * c["D"] * c["N"] > most:
        fits = max(1, most // (c["D"] * c["N"]))
        c["B"] = fits if op == "scan_step" else min(c["B"], fits)
        c["T"] = fits // c["B"] * c["B"]
    return c


# ---- inputs ------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1_000_003 + 29)
    return g


def _lengths(case, seed):
    """Tokens of each sequence: equal, or very different ones, some of none and one."""
    B, T = case["B"], case["T"]
    if not case.get("ragged"):
        return [T // B] * B
    g = torch.Generator()
    g.manual_seed(int(seed) * 7919 + 3)
    w = torch.exp(0.8 * torch.randn(B, generator=g, dtype=torch.float64))
    n = torch.floor(w / w.sum() * T).to(torch.int64).tolist()
    if B >= 4:
        n[1], n[2] = 0, min(1, n[2])
    n[0] += T - sum(n)
    return n


def prepare(case, seed):
    g = _gen(seed)
    dt = STORE[case["dtype"]]
    T, D, op = case["T"], case["D"], case["op"]

    def normal(*shape, dtype=dt, scale=1.0):
        return (scale * torch.randn(shape, generator=g, device="cuda")).to(dtype)

    if op.startswith("norm"):
        st = STORE[case["stream"]]
        s = {"case": case, "weight": 1.0 + 0.1 * normal(D, dtype=torch.float32)}
        # features differ in size, and a few stand far out, as activations do
        size = torch.exp(0.5 * normal(D, dtype=torch.float32))
        size[torch.randint(0, D, (1 + D // 256,), generator=g, device="cuda")] *= 10.0
        if op == "norm_backward":
            s["dout"] = normal(T, D)
            s["x"] = (normal(T, D, dtype=torch.float32) * size).to(st)
            if case["residual"]:
                s["dresidual"] = normal(T, D, dtype=st)
        else:
            s["x"] = (normal(T, D, dtype=torch.float32) * size).to(dt)
            if case["residual"]:
                s["residual"] = (normal(T, D, dtype=torch.float32) * size).to(st)
        return s
    B = case["B"]
    s = {"case": case}
    if "ragged" in case:
        s["lengths"] = _lengths(case, seed)
        if case["ragged"]:
            s["offsets"] = torch.tensor([sum(s["lengths"][:i]) for i in range(B + 1)],
                                        dtype=torch.int64).cuda()
    # the inner projection's output holds the convolution's input and the gate side by side
    xz = normal(T, 2 * D)
    if op.startswith("conv"):
        W = case["W"]
        s |= {"x": xz[:, :D], "weight": normal(D, W, dtype=torch.float32, scale=W ** -0.5),
              "bias": normal(D, dtype=torch.float32, scale=0.1)}
        if case.get("states") or op == "conv_step":
            s["state_in"] = normal(B, W - 1, D)
        if op == "conv_backward":
            s["dout"] = normal(T, D)
            if case["states"]:
                s["dstate_out"] = normal(B, W - 1, D)
        return s
    N, G = case["N"], case["G"]
    R = 16 * max(1, D // 512)  # the rank of delta's projection, beside B and C in one product
    dbc = normal(T, R + 2 * G * N)
    s |= {"u": torch.nn.functional.silu(normal(T, D, dtype=torch.float32)).to(dt),
          "delta": normal(T, D, scale=0.5), "B": dbc[:, R:R + G * N].unflatten(1, (G, N)),
          "C": dbc[:, R + G * N:].unflatten(1, (G, N)),
          "A": -torch.arange(1, N + 1, device="cuda") * torch.exp(normal(D, N, dtype=torch.float32,
                                                                      scale=0.1)),
          "skip": 1.0 + normal(D, dtype=torch.float32, scale=0.1)}
    step = torch.exp(math.log(1e-3) + math.log(100.0) * torch.rand(D, generator=g, device="cuda"))
    s["delta_bias"] = step + torch.log(-torch.expm1(-step))  # softplus(bias) = step
    if case["gated"]:
        s["z"] = xz[:, D:]
    if case.get("states") or op == "scan_step":
        s["state_in"] = normal(B, D, N, dtype=torch.float32)
    if op == "scan_backward":
        s["dout"] = normal(T, D)
        if case["states"]:
            s["dstate_out"] = normal(B, D, N, dtype=torch.float32)
    return s


# ---- the library's operators -------------------------------------------------

def _run_own(s):
    from paper_2605_09204_amd import block

    c = s["case"]
    op = c["op"]
    get = s.get
    if op == "norm":
        return block.lbi_rms_norm(s["x"], s["weight"], get("residual"), EPS)
    if op == "norm_q8":
        fmt = block.LBI_Q8_E4M3 if c["format"] == "e4m3" else block.LBI_Q8_INT8
        q, scales, total = block.lbi_rms_norm_q8(s["x"], s["weight"], get("residual"), EPS, fmt,
                                                 c["group"])
        return _stands_for(q, scales, c["group"]), scales, total
    if op == "norm_backward":
        return block.lbi_rms_norm_backward(s["dout"], s["x"], s["weight"], get("dresidual"), EPS)
    if op == "conv":
        new = torch.empty_like(s["state_in"]) if c["states"] else None
        return block.lbi_ssm_conv(s["x"], s["weight"], s["bias"], offsets=get("offsets"),
                                  sequences=c["B"], state_in=get("state_in"), state_out=new), new
    if op == "conv_backward":
        return block.lbi_ssm_conv_backward(s["x"], s["weight"], s["dout"], s["bias"],
                                           offsets=get("offsets"), sequences=c["B"],
                                           state_in=get("state_in"),
                                           dstate_out=get("dstate_out"))
    if op == "conv_step":
        new = torch.empty_like(s["state_in"])
        return block.lbi_ssm_conv_step(s["x"], s["weight"], s["state_in"], new, s["bias"]), new
    a = (s["u"], s["delta"], s["A"], s["B"], s["C"])
    kw = {"skip": s["skip"], "z": get("z"), "delta_bias": s["delta_bias"]}
    if op == "scan_step":
        new = torch.empty_like(s["state_in"])
        return block.lbi_ssm_scan_step(*a, s["state_in"], new, **kw), new
    kw |= {"offsets": get("offsets"), "sequences": c["B"], "state_in": get("state_in")}
    if op == "scan":
        new = torch.empty_like(s["state_in"]) if c["states"] else None
        return block.lbi_ssm_scan(*a, state_out=new, **kw), new
    return block.lbi_ssm_scan_backward(*a, s["dout"], dstate_out=get("dstate_out"), **kw)


def _stands_for(q, scales, group):
    """The values that the 8-bit ones and their scales stand for."""
    D = q.shape[1]
    return q.float() * (scales if not group else
                        scales.repeat_interleave(group, 1)[:, :D])


# ---- their plain forms, in float32 -------------------------------------------

def _f(t):
    return None if t is None else t.float()


def _plain_norm(s):
    c = s["case"]
    t = _f(s["x"])
    if c["residual"]:
        t = t + _f(s["residual"])
    y = t * torch.rsqrt((t * t).mean(1, keepdim=True) + EPS) * s["weight"]
    total = t.to(STORE[c["stream"]]) if c["residual"] else None
    if c["op"] == "norm":
        return y.to(STORE[c["dtype"]]), total
    T, D = y.shape
    group = c["group"] or D
    ng = -(-D // group)
    padded = torch.zeros(T, ng * group, device=y.device)
    padded[:, :D] = y
    scales = padded.view(T, ng, group).abs().amax(2) / (448.0 if c["format"] == "e4m3" else 127.0)
    scales = torch.where(scales > 0, scales, 1.0)
    v = y / scales.repeat_interleave(group, 1)[:, :D]
    q = v.to(torch.float8_e4m3fn) if c["format"] == "e4m3" else torch.round(v).to(torch.int8)
    return _stands_for(q, scales, c["group"]), scales, total


def _plain_norm_backward(s):
    t, dy = _f(s["x"]), _f(s["dout"])
    r = torch.rsqrt((t * t).mean(1, keepdim=True) + EPS)
    n = t * r
    gy = dy * s["weight"]
    dx = r * (gy - n * (gy * n).mean(1, keepdim=True))
    if s["case"]["residual"]:
        dx = dx + _f(s["dresidual"])
    return dx.to(s["x"].dtype), (dy * n).sum(0)


def _padded(s, t, before=None, fill=0.0):
    """The packed rows as [B, before + longest, ...] in float32, ``before`` rows of it the state."""
    c = s["case"]
    B, T = c["B"], c["T"]
    rows = t.float()
    if not c["ragged"]:
        out = rows.view((B, T // B) + rows.shape[1:])
    else:
        out = torch.cat([rows, rows.new_full((1,) + rows.shape[1:], fill)])[s["index"]]
    return out if before is None else torch.cat([before, out], 1)


def _plan(s):
    """Where each padded place finds its row, and each row its padded place."""
    c = s["case"]
    if c["ragged"] and "index" not in s:
        s = dict(s)
        B, T, off = c["B"], c["T"], s["offsets"]
        p = torch.arange(max(s["lengths"] + [1]), device="cuda")
        n = off[1:] - off[:-1]
        s["index"] = torch.where(p < n[:, None], off[:-1, None] + p, T)
        seq = torch.repeat_interleave(torch.arange(B, device="cuda"), n, output_size=T)
        s["seq"], s["pos"], s["n"] = seq, torch.arange(T, device="cuda") - off[seq], n
    return s


def _packed(s, t):
    c = s["case"]
    return t[s["seq"], s["pos"]] if c["ragged"] else t.reshape((c["T"],) + t.shape[2:])


def _silu_slope(v):
    g = torch.sigmoid(v)
    return g * (1.0 + v * (1.0 - g))


def _plain_conv(s):
    """Forward, or the gradients where ``dout`` is there."""
    c = s["case"]
    B, T, D, W = c["B"], c["T"], c["D"], c["W"]
    dt = s["x"].dtype
    old = _f(s.get("state_in"))
    past = old if old is not None else torch.zeros(B, W - 1, D, device="cuda")
    if c["op"] == "conv_step":
        x = torch.cat([past, _f(s["x"])[:, None]], 1)
        v = s["bias"] + (x * s["weight"].T).sum(1)
        return (v * torch.sigmoid(v)).to(dt), x[:, 1:].to(dt)
    s = _plan(s)
    x = _padded(s, s["x"], past)
    L = x.shape[1] - (W - 1)
    v = s["bias"] + sum(x[:, w:w + L] * s["weight"][:, w] for w in range(W))
    if c["op"] == "conv":
        y = _packed(s, v * torch.sigmoid(v)).to(dt)
        if not c["states"]:
            return y, None
        if c["ragged"]:
            last = s["n"][:, None] + torch.arange(W - 1, device="cuda")
            return y, x[torch.arange(B, device="cuda")[:, None], last].to(dt)
        return y, x[:, L:].to(dt)
    dv = _padded(s, s["dout"]) * _silu_slope(v)
    dx = torch.zeros_like(x)
    for w in range(W):
        dx[:, w:w + L] += dv * s["weight"][:, w]
    dw = torch.stack([(dv * x[:, w:w + L]).sum((0, 1)) for w in range(W)], 1)
    if c["states"]:
        if c["ragged"]:
            last = s["n"][:, None] + torch.arange(W - 1, device="cuda")
            at = torch.arange(B, device="cuda")[:, None]
            dx[at, last] = dx[at, last] + _f(s["dstate_out"])
        else:
            dx[:, L:] += _f(s["dstate_out"])
    return (_packed(s, dx[:, W - 1:]).to(dt), dw, dv.sum((0, 1)),
            dx[:, :W - 1].to(dt) if c["states"] else None)


def _softplus(v):
    return torch.where(v > 20.0, v, torch.log1p(torch.exp(torch.clamp(v, max=20.0))))


def _plain_scan(s):
    """Forward, or the gradients where ``dout`` is there: the tokens of a
    sequence in parts that step side by side, the parts joined by their ends."""
    c = s["case"]
    B, D, N, G = c["B"], c["D"], c["N"], c["G"]
    dt = s["u"].dtype
    A = s["A"].view(G, D // G, N)
    raw = _f(s["delta"]) + s["delta_bias"]
    if c["op"] == "scan_step":
        d, u = _softplus(raw).view(-1, G, D // G), _f(s["u"]).view(-1, G, D // G)
        h = torch.exp(d[..., None] * A) * s["state_in"].view(-1, G, D // G, N) \
            + (d * u)[..., None] * _f(s["B"])[:, :, None]
        y = (h * _f(s["C"])[:, :, None]).sum(-1).view(-1, D) + s["skip"] * _f(s["u"])
        if c["gated"]:
            z = _f(s["z"])
            y = y * z * torch.sigmoid(z)
        return y.to(dt), h.view(-1, D, N)
    s = _plan(s)
    L = max(s["lengths"] + [1]) if c["ragged"] else c["T"] // B
    K = max(1, 2 ** round(math.log2(max(1, L)) / 2))  # tokens of a part
    P = -(-L // K)

    def parts(t, width):  # [K][B, P, G, width]
        t = _padded(s, t)
        t = torch.cat([t, t.new_zeros((B, P * K - L) + t.shape[2:])], 1)
        return t.view(B, P, K, G, width).permute(2, 0, 1, 3, 4).contiguous()

    d, u = parts(_softplus(raw), D // G), parts(s["u"], D // G)  # 0 past a sequence's end
    Bm, Cm = parts(s["B"], N), parts(s["C"], N)
    x = d * u
    whole = torch.exp(d.sum(0)[..., None] * A)
    h = torch.zeros(B, P, G, D // G, N, device="cuda")

    def forward(h, k):
        return torch.exp(d[k][..., None] * A) * h + x[k][..., None] * Bm[k][..., None, :]

    for k in range(K if P > 1 else 0):
        h = forward(h, k)
    ends, h = h, torch.empty_like(h)
    cur = s["state_in"].view(B, G, D // G, N) if c["states"] else torch.zeros_like(h[:, 0])
    for p in range(P):
        h[:, p] = cur
        cur = whole[:, p] * cur + ends[:, p]
    backward = c["op"] == "scan_backward"
    y, hs = torch.empty_like(d), [h]
    for k in range(K):
        h = forward(h, k)
        y[k] = (h * Cm[k][..., None, :]).sum(-1)
        if backward:
            hs.append(h)

    def tokens(t):  # [K][B, P, G, width] back to packed rows
        t = t.permute(1, 2, 0, 3, 4).reshape(B, P * K, -1)[:, :L]
        return _packed(s, t)

    y = tokens(y) + s["skip"] * _f(s["u"])
    z = _f(s["z"]) if c["gated"] else None
    if not backward:
        if c["gated"]:
            y = y * z * torch.sigmoid(z)
        return y.to(dt), h[:, -1].reshape(B, D, N) if c["states"] else None
    dy, dz = _f(s["dout"]), None
    if c["gated"]:
        dz = (dy * y * _silu_slope(z)).to(dt)
        dy = dy * z * torch.sigmoid(z)
    e = parts(dy, D // G)
    g = torch.zeros_like(h)
    for k in reversed(range(K if P > 1 else 0)):
        g = (g + e[k][..., None] * Cm[k][..., None, :]) * torch.exp(d[k][..., None] * A)
    starts, g = g, torch.empty_like(g)
    cur = s["dstate_out"].view(B, G, D // G, N) if c["states"] else torch.zeros_like(g[:, 0])
    for p in reversed(range(P)):
        g[:, p] = cur
        cur = whole[:, p] * cur + starts[:, p]
    dx, dd = torch.empty_like(d), torch.empty_like(d)
    dB, dC = torch.empty_like(Bm), torch.empty_like(Cm)
    dA = torch.zeros_like(A)
    for k in reversed(range(K)):
        g = g + e[k][..., None] * Cm[k][..., None, :]
        dC[k] = (hs[k + 1] * e[k][..., None]).sum(3)
        dB[k] = (g * x[k][..., None]).sum(3)
        dx[k] = (g * Bm[k][..., None, :]).sum(-1)
        g = g * torch.exp(d[k][..., None] * A)
        q = g * hs[k]
        dd[k] = (q * A).sum(-1)
        dA += (q * d[k][..., None]).sum((0, 1))
    rows = _f(s["u"])
    dxr = tokens(dx)
    ddr = (tokens(dd) + dxr * rows) * torch.sigmoid(raw)
    return {"u": (dxr * _softplus(raw) + s["skip"] * dy).to(dt), "delta": ddr.to(dt),
            "A": dA.view(D, N), "B": tokens(dB).view(-1, G, N).to(dt),
            "C": tokens(dC).view(-1, G, N).to(dt), "skip": (dy * rows).sum(0), "z": dz,
            "delta_bias": ddr.sum(0),
            "state_in": g[:, 0].reshape(B, D, N) if c["states"] else None}


def run(state):
    if own:
        return _run_own(state)
    op = state["case"]["op"]
    if op == "norm_backward":
        return _plain_norm_backward(state)
    if op.startswith("norm"):
        return _plain_norm(state)
    return _plain_conv(state) if op.startswith("conv") else _plain_scan(state)


# ---- what a pass cannot do without -------------------------------------------

def work(case):
    """Each input read once, each output written once, and the operations of the
    formulas (an exponential counted as one)."""
    op, T, D = case["op"], case["T"], case["D"]
    e = 4 if case["dtype"] == "f32" else 2
    if op.startswith("norm"):
        f = 4 if case["stream"] == "f32" else 2
        extra = T * D * f if case["residual"] else 0
        if op == "norm_backward":  # dout, x, dresidual in; dx and dweight out
            return {"bytes": T * D * (e + 2 * f) + extra + 8 * D, "flops": 11 * T * D}
        out = T * D * e
        if op == "norm_q8":
            out = T * D + 4 * T * (-(-D // case["group"]) if case["group"] else 1)
        return {"bytes": T * D * e + 2 * extra + out + 4 * D, "flops": 6 * T * D}
    B = case["B"]
    if op.startswith("conv"):
        W = case["W"]
        state = B * (W - 1) * D * e if case.get("states") or op == "conv_step" else 0
        per = 4 * D * (W + 1)
        if op == "conv_backward":  # x, dout in; dx out; with states dstate_out and dstate_in too
            return {"bytes": 3 * T * D * e + 3 * state + 2 * per, "flops": (6 * W + 10) * T * D}
        return {"bytes": 2 * T * D * e + 2 * state + per, "flops": (2 * W + 5) * T * D}
    N, G = case["N"], case["G"]
    gate = 1 if case["gated"] else 0
    bc = 2 * T * G * N * e
    par = 4 * D * (N + 2)
    state = 4 * B * D * N if case.get("states") or op == "scan_step" else 0
    if op == "scan_backward":  # u, delta, dout, z in; their gradients out
        return {"bytes": T * D * e * (5 + 2 * gate) + 2 * bc + 2 * par + 3 * state,
                "flops": T * D * (20 * N + 20)}
    return {"bytes": T * D * e * (3 + gate) + bc + par + 2 * state, "flops": T * D * (7 * N + 12)}


# ---- the definitions in 64 bits ----------------------------------------------

def exact(case, seed):
    """What ``run`` returns, token by token in float64; gradients by torch's
    automatic differentiation of the forward."""
    s = prepare(case, seed)
    op, T, D = case["op"], case["T"], case["D"]
    keep = op.endswith("backward")
    v = {k: t.double().requires_grad_(keep) for k, t in s.items()
         if torch.is_tensor(t) and k not in ("offsets", "dout", "dresidual", "dstate_out")}
    if op.startswith("norm"):
        t = v["x"] + v["residual"] if "residual" in v else v["x"]
        y = v["weight"] * t / torch.sqrt(t.square().mean(1, keepdim=True) + EPS)
        if op == "norm":
            return y, t if case["residual"] else None
        if op == "norm_q8":  # the 8-bit values stand for y itself
            ends = list(range(0, D, case["group"] or D))
            top = torch.stack([y[:, i:i + (case["group"] or D)].abs().amax(1) for i in ends], 1)
            top = top / (448 if case["format"] == "e4m3" else 127)
            return y, torch.where(top > 0, top, 1.0), t if case["residual"] else None
        dx, dw = torch.autograd.grad(y, [v["x"], v["weight"]], s["dout"].double())
        return dx + s["dresidual"].double() if case["residual"] else dx, dw
    B = case["B"]
    n = s.get("lengths", [1] * B)
    begin = [sum(n[:i]) for i in range(B)]
    if op.startswith("conv"):
        W = case["W"]
        ys, news = [], []
        for b in range(B):
            old = v["state_in"][b] if "state_in" in v else torch.zeros(W - 1, D, dtype=torch.float64,
                                                                       device="cuda")
            x = torch.cat([old, v["x"][begin[b]:begin[b] + n[b]]])
            a = v["bias"].expand(n[b], D)
            for w in range(W):
                a = a + x[w:w + n[b]] * v["weight"][:, w]
            ys.append(a / (1 + torch.exp(-a)))
            news.append(x[n[b]:])
        y, new = torch.cat(ys), torch.stack(news)
        if not keep:
            return y, new if "state_in" in v else None
        wrt = [v[k] for k in ("x", "weight", "bias")] + ([v["state_in"]] if case["states"] else [])
        of = [y] + ([new] if case["states"] else [])
        by = [s["dout"].double()] + ([s["dstate_out"].double()] if case["states"] else [])
        got = torch.autograd.grad(of, wrt, by)
        return tuple(got) + (() if case["states"] else (None,))
    N, G = case["N"], case["G"]
    if max(n) * (4 if keep else 1) > 131072 or T * D * N * (6 if keep else 1) > 6e9:
        return None  # too many steps, or too much to keep
    # sequences by falling length: at each step those that still run are the first ones
    order = sorted(range(B), key=lambda b: -n[b])
    at = torch.tensor([begin[b] for b in order], device="cuda")
    d = torch.nn.functional.softplus(v["delta"] + v["delta_bias"], threshold=100.0)
    Br, Cr = (v[k].repeat_interleave(D // G, 1) for k in ("B", "C"))
    h = v["state_in"][order] if "state_in" in v else torch.zeros(B, D, N, dtype=torch.float64,
                                                                 device="cuda")
    rows, outs, done = [], [], []
    for t in range(max(n)):
        m = sum(1 for b in order if n[b] > t)
        if m < h.shape[0]:
            done.append(h[m:])
            h = h[:m]
        r = at[:m] + t
        h = torch.exp(d[r][..., None] * v["A"]) * h + (d[r] * v["u"][r])[..., None] * Br[r]
        outs.append((h * Cr[r]).sum(-1))
        rows.append(r)
    done.append(h)
    new = torch.cat(list(reversed(done)))[torch.argsort(torch.tensor(order)).cuda()]
    y = torch.cat(outs)[torch.argsort(torch.cat(rows))] + v["skip"] * v["u"]
    if case["gated"]:
        y = y * v["z"] / (1 + torch.exp(-v["z"]))
    if not keep:
        return y, new if "state_in" in v else None
    names = ["u", "delta", "A", "B", "C", "skip", "delta_bias"] + (["z"] if case["gated"] else []) \
        + (["state_in"] if case["states"] else [])
    of = [y] + ([new] if case["states"] else [])
    by = [s["dout"].double()] + ([s["dstate_out"].double()] if case["states"] else [])
    got = dict(zip(names, torch.autograd.grad(of, [v[k] for k in names], by)))
    return {k: got.get(k) for k in ("u", "delta", "A", "B", "C", "skip", "z", "delta_bias",
                                    "state_in")}
