"""The calls of a region block with linear attention whose speed this library is held to.

A region transformation of this kind is a layer norm that joins the residual
stream, projections with what follows them, and attention whose weights are the
plain products of queries and keys, fading with the distance, so that a state of
fixed size stands for all earlier tokens:

    s = x + residual,  out = (s - mean(s)) / sqrt(var(s) + eps) * weight + bias
    out = act(x W^T + bias) + residual
    S_t = exp(log_decay) S_{t-1} + k_t v_t^T,  o_t = scale q_t^T S_t

Each case is one call as a training step, a prompt pass or a single decoded token
makes it.  Shapes follow the block of this repository's Phase 1 workload (B = 8
sequences of L = 2048 tokens, D = 768 features) and of its state-space block (an
inner width of 1536).
"""
import math

import torch

own = False

EPS = 1e-5
STORE = {"f32": torch.float32, "bf16": torch.bfloat16}
CHUNK = 64  # tokens that the plain form of the attention takes at once


def listed():
    return [
        # the norm at a block's entry in a training step, with the residual stream's addition
        {"name": "norm_tokens", "op": "norm", "dtype": "bf16", "stream": "bf16", "T": 16384,
         "D": 768, "residual": True, "affine": True},
        # its gradient at an odd number of tokens on a float32 residual stream
        {"name": "norm_backward", "op": "norm_backward", "dtype": "bf16", "stream": "f32",
         "T": 12289, "D": 768, "residual": True, "affine": True},
        # a training step's projection into the block, which keeps what its activation was given
        {"name": "projection_in", "op": "projection", "dtype": "bf16", "stream": "bf16",
         "T": 16384, "K": 768, "N": 1536, "bias": True, "act": "silu", "residual": False,
         "pre": True},
        # packed prompts' projection back onto the residual stream, float32
        {"name": "projection_out", "op": "projection", "dtype": "f32", "stream": "f32",
         "T": 4099, "K": 1536, "N": 768, "bias": True, "act": "none", "residual": True,
         "pre": False},
        # one decoded token for each of 64 requests, back onto a float32 stream
        {"name": "projection_step", "op": "projection", "dtype": "bf16", "stream": "f32",
         "T": 64, "K": 1536, "N": 768, "bias": True, "act": "none", "residual": True,
         "pre": False},
        # the projection's gradients in a training step
        {"name": "projection_backward", "op": "projection_backward", "dtype": "bf16",
         "stream": "bf16", "T": 16384, "K": 768, "N": 1536, "bias": True, "act": "silu"},
        # the attention of a training step
        {"name": "attention_train", "op": "attention", "dtype": "bf16", "B": 8, "T": 16384,
         "H": 12, "KH": 12, "DK": 64, "DV": 64, "ragged": False, "states": False},
        # packed prompts of different lengths from kept states to new ones, keys shared by three
        # heads, the values twice as wide
        {"name": "attention_prompts", "op": "attention", "dtype": "bf16", "B": 13, "T": 8201,
         "H": 12, "KH": 4, "DK": 64, "DV": 128, "ragged": True, "states": True},
        # one long sequence in float32: parallel only along the tokens
        {"name": "attention_long", "op": "attention", "dtype": "f32", "B": 1, "T": 32768,
         "H": 12, "KH": 12, "DK": 64, "DV": 64, "ragged": False, "states": True},
        # the attention's gradients in a training step
        {"name": "attention_backward", "op": "attention_backward", "dtype": "bf16", "B": 8,
         "T": 16384, "H": 12, "KH": 12, "DK": 64, "DV": 64, "ragged": False, "states": False},
        # the gradients at odd sizes, float32, shared keys, states passed from part to part
        {"name": "attention_backward_odd", "op": "attention_backward", "dtype": "f32", "B": 5,
         "T": 3885, "H": 6, "KH": 2, "DK": 48, "DV": 101, "ragged": True, "states": True},
        # one decoded token for each of 64 requests
        {"name": "attention_step", "op": "attention_step", "dtype": "bf16", "B": 64, "T": 64,
         "H": 12, "KH": 12, "DK": 64, "DV": 128},
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)) - 1e-9)))))


def draw(rng):
    """One more call: any operator, sizes from one token to the training step's."""
    most = {}
    for c in listed():
        for k, v in work(c).items():
            at = (c["op"].split("_")[0], k)
            most[at] = max(most.get(at, 0), v)
    while True:
        c = _draw(rng)
        kind = c["op"].split("_")[0]
        if all(v <= most[kind, k] for k, v in work(c).items()):
            return c


def _draw(rng):
    op = rng.choice(["norm", "norm_backward", "projection", "projection", "projection_backward",
                     "attention", "attention", "attention_backward", "attention_backward",
                     "attention_step"])
    c = {"op": op, "dtype": rng.choice(["f32", "bf16", "bf16"])}
    if op.startswith("norm"):
        c |= {"T": _log(rng, 1, 32768), "D": _log(rng, 16, 8192)}
        if rng.random() < 0.6:  # most widths are whole vectors
            c["D"] = max(16, c["D"] // 16 * 16)
        return c | {"stream": rng.choice([c["dtype"], "f32"]), "residual": rng.random() < 0.7,
                    "affine": rng.random() < 0.8}
    if op.startswith("projection"):
        c |= {"T": _log(rng, 1, 32768), "K": _log(rng, 16, 4096), "N": _log(rng, 16, 4096)}
        if rng.random() < 0.6:
            c["K"] = max(16, c["K"] // 16 * 16)
            c["N"] = max(16, c["N"] // 16 * 16)
        c |= {"stream": rng.choice([c["dtype"], "f32"]), "bias": rng.random() < 0.7,
              "act": rng.choice(["none", "silu", "gelu"])}
        if op == "projection":
            c |= {"residual": rng.random() < 0.5,
                  "pre": c["act"] != "none" and rng.random() < 0.5}
        return c
    KH = rng.choice([1, 2, 3, 4, 6, 8, 12])
    c |= {"T": _log(rng, 1, 32768), "H": KH * rng.choice([1, 1, 2, 3]), "KH": KH,
          "DK": _log(rng, 16, 128), "DV": _log(rng, 16, 128)}
    if rng.random() < 0.6:
        c["DK"] = c["DK"] // 16 * 16
        c["DV"] = c["DV"] // 16 * 16
    if op == "attention_step":
        c["T"] = c["B"] = max(1, min(c["T"], 512))
        return c
    c["B"] = _log(rng, 1, min(64, c["T"]))
    c |= {"ragged": rng.random() < 0.5, "states": rng.random() < 0.5}
    if not c["ragged"]:
        c["T"] = c["T"] // c["B"] * c["B"]
    return c


# ---- inputs ------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1_000_003 + 53)
    return g


def _lengths(case, seed):
    """Tokens of each sequence: equal, or very different ones, some of none and one."""
    B, T = case["B"], case["T"]
    if not case.get("ragged"):
        return [T // B] * B
    g = torch.Generator()
    g.manual_seed(int(seed) * 7919 + 11)
    w = torch.exp(0.8 * torch.randn(B, generator=g, dtype=torch.float64))
    n = torch.floor(w / w.sum() * T).to(torch.int64).tolist()
    if B >= 4:
        n[1], n[2] = 0, min(1, n[2])
    n[0] += T - sum(n)
    return n


def prepare(case, seed):
    g = _gen(seed)
    dt = STORE[case["dtype"]]
    T, op = case["T"], case["op"]

    def normal(*shape, dtype=dt, scale=1.0):
        return (scale * torch.randn(shape, generator=g, device="cuda")).to(dtype)

    s = {"case": case}
    if op.startswith("norm"):
        st, D = STORE[case["stream"]], case["D"]
        # features differ in size and place, and a few stand far out, as activations do
        size = torch.exp(0.5 * normal(D, dtype=torch.float32))
        size[torch.randint(0, D, (1 + D // 256,), generator=g, device="cuda")] *= 10.0
        place = 0.5 + normal(D, dtype=torch.float32, scale=0.3)

        def activations(dtype):
            return ((normal(T, D, dtype=torch.float32) + place) * size).to(dtype)
        if case["affine"]:
            s |= {"weight": 1.0 + normal(D, dtype=torch.float32, scale=0.1),
                  "bias": normal(D, dtype=torch.float32, scale=0.1)}
        if op == "norm_backward":
            s |= {"dout": normal(T, D), "x": activations(st)}
            if case["residual"]:
                s["dresidual"] = normal(T, D, dtype=st)
        else:
            s["x"] = activations(dt)
            if case["residual"]:
                s["residual"] = activations(st)
        return s
    if op.startswith("projection"):
        st, K, N = STORE[case["stream"]], case["K"], case["N"]
        s |= {"x": normal(T, K), "weight": normal(N, K, scale=K ** -0.5)}
        if case["bias"]:
            s["bias"] = normal(N, dtype=torch.float32, scale=0.1)
        if op == "projection_backward":
            s["dout"] = normal(T, N, dtype=st)
            if case["act"] != "none":  # distributed as the forward pass leaves it
                s["pre"] = normal(T, N)
        elif case["residual"]:
            s["residual"] = normal(T, N, dtype=st)
        return s
    B, H, KH, DK, DV = (case[k] for k in ("B", "H", "KH", "DK", "DV"))
    # one projection's output holds queries, keys and values side by side
    qkv = normal(T, H * DK + KH * (DK + DV))
    s |= {"q": qkv[:, :H * DK].unflatten(1, (H, DK)),
          "k": qkv[:, H * DK:(H + KH) * DK].unflatten(1, (KH, DK)),
          "v": qkv[:, (H + KH) * DK:].unflatten(1, (KH, DV)), "scale": DK ** -0.5}
    # memories from one or two tokens to a thousand
    s["log_decay"] = -torch.exp(math.log(1e-3) + math.log(700.0)
                                * torch.rand(H, generator=g, device="cuda"))
    if op == "attention_step":
        s["state_in"] = normal(B, H, DK, DV, dtype=torch.float32, scale=4.0)
        return s
    s["lengths"] = _lengths(case, seed)
    if case["ragged"]:
        s["offsets"] = torch.tensor([sum(s["lengths"][:i]) for i in range(B + 1)],
                                    dtype=torch.int64).cuda()
    if case["states"]:
        s["state_in"] = normal(B, H, DK, DV, dtype=torch.float32, scale=4.0)
    if op == "attention_backward":
        s["dout"] = normal(T, H, DV)
        if case["states"]:
            s["dstate_out"] = normal(B, H, DK, DV, dtype=torch.float32)
    return s


# ---- the library's operators -------------------------------------------------

def _run_own(s):
    from paper_2605_09204_amd import linear

    c = s["case"]
    op = c["op"]
    get = s.get
    if op == "norm":
        return linear.lbi_layer_norm(s["x"], get("weight"), get("bias"), get("residual"), EPS)
    if op == "norm_backward":
        return linear.lbi_layer_norm_backward(s["dout"], s["x"], get("weight"), get("dresidual"),
                                              EPS)
    if op.startswith("projection"):
        act = {"none": linear.LBI_ACT_NONE, "silu": linear.LBI_ACT_SILU,
               "gelu": linear.LBI_ACT_GELU}[c["act"]]
        if op == "projection_backward":
            return linear.lbi_projection_backward(s["x"], s["weight"], s["dout"], act, get("pre"))
        out = torch.empty(c["T"], c["N"], dtype=STORE[c["stream"]], device="cuda")
        pre = torch.empty(c["T"], c["N"], dtype=s["x"].dtype, device="cuda") if c["pre"] else None
        linear.lbi_projection(s["x"], s["weight"], get("bias"), act, get("residual"), out=out,
                              pre=pre)
        return out, pre
    a = (s["q"], s["k"], s["v"], s["log_decay"])
    if op == "attention_step":
        new = torch.empty_like(s["state_in"])
        return linear.lbi_linear_attention_step(*a, s["state_in"], new, s["scale"]), new
    kw = {"scale": s["scale"], "offsets": get("offsets"), "sequences": c["B"],
          "state_in": get("state_in")}
    if op == "attention":
        new = torch.empty_like(s["state_in"]) if c["states"] else None
        return linear.lbi_linear_attention(*a, state_out=new, **kw), new
    return linear.lbi_linear_attention_backward(*a, s["dout"], dstate_out=get("dstate_out"), **kw)


# ---- their plain forms, in float32 -------------------------------------------

def _f(t):
    return None if t is None else t.float()


def _plain_norm(s):
    c = s["case"]
    t = _f(s["x"])
    if c["residual"]:
        t = t + _f(s["residual"])
    d = t - t.mean(1, keepdim=True)
    y = d * torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
    if c["affine"]:
        y = y * s["weight"] + s["bias"]
    return y.to(STORE[c["dtype"]]), t.to(STORE[c["stream"]]) if c["residual"] else None


def _plain_norm_backward(s):
    c = s["case"]
    t, dy = _f(s["x"]), _f(s["dout"])
    d = t - t.mean(1, keepdim=True)
    r = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
    n = d * r
    g = dy * s["weight"] if c["affine"] else dy
    dx = r * (g - g.mean(1, keepdim=True) - n * (g * n).mean(1, keepdim=True))
    if c["residual"]:
        dx = dx + _f(s["dresidual"])
    return dx.to(s["x"].dtype), (dy * n).sum(0), dy.sum(0)


def _act(name, v):
    if name == "silu":
        return v * torch.sigmoid(v)
    return 0.5 * v * (1.0 + torch.erf(v * 0.5 ** 0.5)) if name == "gelu" else v


def _act_slope(name, v):
    if name == "silu":
        g = torch.sigmoid(v)
        return g * (1.0 + v * (1.0 - g))
    return 0.5 * (1.0 + torch.erf(v * 0.5 ** 0.5)) \
        + v * torch.exp(-0.5 * v * v) * (2.0 * math.pi) ** -0.5


def _plain_projection(s):
    c = s["case"]
    z = _f(s["x"]) @ _f(s["weight"]).T
    if c["bias"]:
        z = z + s["bias"]
    y = _act(c["act"], z)
    if c["residual"]:
        y = y + _f(s["residual"])
    return y.to(STORE[c["stream"]]), z.to(s["x"].dtype) if c["pre"] else None


def _plain_projection_backward(s):
    c = s["case"]
    dz = _f(s["dout"])
    if c["act"] != "none":
        dz = dz * _act_slope(c["act"], _f(s["pre"]))
    dt = s["x"].dtype
    return (dz @ _f(s["weight"])).to(dt), (dz.T @ _f(s["x"])).to(dt), dz.sum(0)


def _plan(s):
    """Where each padded place [B, chunks, CHUNK] finds its row (T: none), how many of a chunk's
    places are filled, and each row's padded place."""
    c = s["case"]
    B, T = c["B"], c["T"]
    n = s["offsets"][1:] - s["offsets"][:-1] if c["ragged"] \
        else torch.full((B,), T // B, device="cuda")
    begin = torch.cumsum(n, 0) - n
    chunks = max(1, -(-max(s["lengths"] + [0]) // CHUNK))
    p = torch.arange(chunks * CHUNK, device="cuda")
    index = torch.where(p < n[:, None], begin[:, None] + p, T)
    filled = (n[:, None] - CHUNK * torch.arange(chunks, device="cuda")).clamp(0, CHUNK)
    seq = torch.repeat_interleave(torch.arange(B, device="cuda"), n, output_size=T)
    return index, filled, seq * (chunks * CHUNK) + torch.arange(T, device="cuda") - begin[seq]


def _plain_attention(s):
    """Forward, or the gradients where ``dout`` is there: chunks of tokens by products, the chunks
    joined by their states."""
    c = s["case"]
    B, T, H, KH, DK, DV = (c[k] for k in ("B", "T", "H", "KH", "DK", "DV"))
    dt, scale, ld = s["q"].dtype, s["scale"], s["log_decay"]
    share = H // KH
    if c["op"] == "attention_step":
        k, v = (_f(s[x]).repeat_interleave(share, 1) for x in ("k", "v"))
        new = torch.exp(ld)[:, None, None] * s["state_in"] + k[..., None] * v[..., None, :]
        return (scale * (_f(s["q"])[..., None] * new).sum(2)).to(dt), new
    index, filled, place = _plan(s)
    NC = filled.shape[1]

    def padded(t, n):  # [B, H, NC, CHUNK, width]
        t = torch.cat([t.float(), t.new_zeros((1,) + t.shape[1:], dtype=torch.float32)])[index]
        return t.view(B, NC, CHUNK, n, -1).permute(0, 3, 1, 2, 4)

    def shared(t):
        return t.repeat_interleave(share, 1).contiguous()

    def rows(t, n):  # back to [T, n, width]
        return t.permute(0, 2, 3, 1, 4).reshape(B * NC * CHUNK, n, -1)[place]

    q = scale * padded(s["q"], H).contiguous()
    k, v = shared(padded(s["k"], KH)), shared(padded(s["v"], KH))
    i = torch.arange(CHUNK, device="cuda")
    lag = (i[:, None] - i).float()
    fade = torch.where(lag >= 0, torch.exp(lag * ld[:, None, None]), 0.0)[None, :, None]
    from_start = torch.exp((i + 1.0) * ld[:, None])[None, :, None, :, None]
    left = filled[:, None, :, None] - 1.0 - i  # tokens of the chunk after each
    to_end = torch.where(left >= 0, torch.exp(left * ld[:, None, None]), 0.0)[..., None]
    whole = torch.exp(filled[:, None, :] * ld[:, None])[..., None, None]
    ends = (k * to_end).transpose(-1, -2).contiguous() @ v
    state = s["state_in"] if c["states"] else torch.zeros(B, H, DK, DV, device="cuda")
    starts = []
    for x in range(NC):
        starts.append(state)
        state = whole[:, :, x] * state + ends[:, :, x]
    S = torch.stack(starts, 2)
    P = q @ k.transpose(-1, -2).contiguous() * fade
    if c["op"] == "attention":
        o = P @ v + (from_start * q) @ S
        return rows(o, H).to(dt), state if c["states"] else None
    do = padded(s["dout"], H).contiguous()
    heads = (q * from_start).transpose(-1, -2).contiguous() @ do
    g = s["dstate_out"] if c["states"] else torch.zeros_like(state)
    grads = []
    for x in reversed(range(NC)):
        grads.append(g)
        g = whole[:, :, x] * g + heads[:, :, x]
    G = torch.stack(grads[::-1], 2)
    dP = do @ v.transpose(-1, -2).contiguous()
    e = dP * fade
    from_S = from_start * (do @ S.transpose(-1, -2).contiguous())
    to_G = to_end * (v @ G.transpose(-1, -2).contiguous())
    dq = e @ k + from_S
    dk = e.transpose(-1, -2).contiguous() @ q + to_G
    dv = P.transpose(-1, -2).contiguous() @ do + to_end * (k @ G)
    dld = (P * dP * lag).sum((0, 2, 3, 4)) \
        + (q * from_S * (i + 1.0)[:, None]).sum((0, 2, 3, 4)) \
        + (k * to_G * left[..., None]).sum((0, 2, 3, 4)) \
        + (filled[:, None, :, None, None] * whole * S * G).sum((0, 2, 3, 4))

    def unshared(t):
        return t.view(T, KH, share, -1).sum(2)
    return {"q": rows(scale * dq, H).to(dt), "k": unshared(rows(dk, H)).to(dt),
            "v": unshared(rows(dv, H)).to(dt), "log_decay": dld,
            "state_in": g if c["states"] else None}


def run(state):
    if own:
        return _run_own(state)
    op = state["case"]["op"]
    return {"norm": _plain_norm, "norm_backward": _plain_norm_backward,
            "projection": _plain_projection,
            "projection_backward": _plain_projection_backward}.get(op, _plain_attention)(state)


# ---- what a pass cannot do without -------------------------------------------

def work(case):
    """Each input read once, each output written once, and the operations of the
    formulas (the attention's as a recurrence)."""
    op, T = case["op"], case["T"]
    e = 4 if case["dtype"] == "f32" else 2
    f = 4 if case.get("stream") == "f32" else 2
    if op.startswith("norm"):
        D = case["D"]
        extra = T * D * f if case["residual"] else 0
        par = 8 * D if case["affine"] else 0
        if op == "norm_backward":  # dout, x, dresidual in; dx, dweight, dbias out
            return {"bytes": T * D * (e + 2 * f) + extra + par // 2 + 8 * D, "flops": 14 * T * D}
        return {"bytes": 2 * T * D * e + 2 * extra + par, "flops": 8 * T * D}
    if op.startswith("projection"):
        K, N = case["K"], case["N"]
        bias = 4 * N if case["bias"] else 0
        if op == "projection_backward":  # x, weight, dout, pre in; dx, dweight, dbias out
            pre = T * N * e if case["act"] != "none" else 0
            return {"bytes": 2 * (T + N) * K * e + T * N * f + pre + 4 * N,
                    "flops": 4 * T * K * N + 8 * T * N}
        return {"bytes": (T + N) * K * e + T * N * f * (2 if case["residual"] else 1) + bias
                + (T * N * e if case["pre"] else 0), "flops": 2 * T * K * N + 6 * T * N}
    B, H, KH, DK, DV = (case[k] for k in ("B", "H", "KH", "DK", "DV"))
    state = 4 * B * H * DK * DV if case.get("states") or op == "attention_step" else 0
    rows = T * e * (H * DK + KH * (DK + DV))
    if op == "attention_backward":  # q, k, v, dout in; their gradients and the decays' out
        return {"bytes": 2 * rows + T * e * H * DV + 3 * state + 8 * H,
                "flops": 14 * T * H * DK * DV}
    return {"bytes": rows + T * e * H * DV + 2 * state + 4 * H, "flops": 5 * T * H * DK * DV}


# ---- the definitions in 64 bits ----------------------------------------------

def exact(case, seed):
    """What ``run`` returns, in float64: the attention as the sum over all pairs of tokens,
    gradients by torch's automatic differentiation of the forward."""
    s = prepare(case, seed)
    op, T = case["op"], case["T"]
    keep = op.endswith("backward")
    skip = ("offsets", "dout", "dresidual", "dstate_out")
    v = {k: t.double().requires_grad_(keep) for k, t in s.items()
         if torch.is_tensor(t) and k not in skip}
    if op.startswith("norm"):
        t = v["x"] + v["residual"] if "residual" in v else v["x"]
        if "weight" not in v:
            D = case["D"]
            v["weight"] = torch.ones(D, dtype=torch.float64, device="cuda", requires_grad=keep)
            v["bias"] = torch.zeros(D, dtype=torch.float64, device="cuda", requires_grad=keep)
        y = v["weight"] * (t - t.mean(1, keepdim=True)) \
            / torch.sqrt(t.var(1, unbiased=False, keepdim=True) + EPS) + v["bias"]
        if op == "norm":
            return y, t if case["residual"] else None
        dx, dw, db = torch.autograd.grad(y, [v["x"], v["weight"], v["bias"]], s["dout"].double())
        return dx + s["dresidual"].double() if case["residual"] else dx, dw, db
    if op.startswith("projection"):
        shape = {"none": lambda z: z, "silu": torch.nn.functional.silu,
                 "gelu": torch.nn.functional.gelu}[case["act"]]
        if op == "projection":
            z = v["x"] @ v["weight"].T + (v["bias"] if case["bias"] else 0.0)
            y = shape(z) + (v["residual"] if case["residual"] else 0.0)
            return y, z if case["pre"] else None
        dz = s["dout"].double()
        if case["act"] != "none":
            (dz,) = torch.autograd.grad(shape(v["pre"]), v["pre"], dz)
        with torch.no_grad():
            return dz @ v["weight"], dz.T @ v["x"], dz.sum(0)
    B, H, KH, DK, DV = (case[k] for k in ("B", "H", "KH", "DK", "DV"))
    n = s.get("lengths", [1] * B)
    if sum(m * m for m in n) * H * (DK + DV) * (4 if keep else 1) > 1e13:
        return None  # too many pairs of tokens
    outs = torch.empty(T, H, DV, dtype=torch.float64, device="cuda")
    new = torch.empty(B, H, DK, DV, dtype=torch.float64, device="cuda")
    grad = {k: torch.zeros_like(v[k]) for k in ("q", "k", "v", "log_decay", "state_in") if k in v}
    begin = 0
    for b in range(B):
        L = n[b]
        at = slice(begin, begin + L)
        begin += L
        i = torch.arange(L, device="cuda", dtype=torch.float64)
        for h in range(H):
            kh = h // (H // KH)
            part = [v["q"][at, h], v["k"][at, kh], v["v"][at, kh], v["log_decay"][h]]
            if "state_in" in v:
                part.append(v["state_in"][b, h])
            if keep:
                part = [t.detach().requires_grad_() for t in part]
            q, k, w, a = part[:4]
            lag = i[:, None] - i
            fade = torch.exp(a * lag.clamp(min=0)) * (lag >= 0)
            o = ((q @ k.T) * fade) @ w
            last = (k * torch.exp(a * (L - 1 - i))[:, None]).T @ w
            if "state_in" in v:
                o = o + torch.exp(a * (i + 1))[:, None] * (q @ part[4])
                last = last + torch.exp(a * L) * part[4]
            o = s["scale"] * o
            if not keep:
                outs[at, h], new[b, h] = o, last
                continue
            of, by = [o], [s["dout"][at, h].double()]
            if case["states"]:
                of.append(last)
                by.append(s["dstate_out"][b, h].double())
            got = torch.autograd.grad(of, part, by, allow_unused=True)
            got = [torch.zeros_like(p) if x is None else x for p, x in zip(part, got)]
            grad["q"][at, h] += got[0]
            grad["k"][at, kh] += got[1]
            grad["v"][at, kh] += got[2]
            grad["log_decay"][h] += got[3]
            if "state_in" in v:
                grad["state_in"][b, h] += got[4]
    if keep:
        return {k: grad[k].detach() if k in grad else None
                for k in ("q", "k", "v", "log_decay", "state_in")}
    return outs, new if "state_in" in v else None
