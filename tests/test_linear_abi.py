"""The entry points of include/lbi_linear.h are declared, exported and refuse bad arguments before
anything reaches the GPU (runs without a GPU: no call here gets that far)."""
import ctypes
import os
import re
import subprocess

import pytest

from paper_2605_09204_amd import binding, linear

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "lbi_linear.h")

pytestmark = pytest.mark.skipif(not os.path.exists(binding.library_path()),
                                reason="library not built")

NULL, SHAPE, DTYPE, WORKSPACE, ALIGN, ALIAS = 1, 2, 3, 5, 7, 8
STEP = 1 << 34  # fake device addresses, far apart: never dereferenced, only validated
P = [STEP * (i + 1) for i in range(24)]


def declared():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return sorted(set(re.findall(r"\b(lbi_[a-z0-9_]+)\s*\(", text)))


def test_header_compiles_as_c_and_every_function_is_exported():
    src = '#include "lbi_linear.h"\nint main(void){return LBI_ATTENTION_MAX_H == 1024 ? 0 : 1;}\n'
    res = subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-fsyntax-only",
                          f"-I{os.path.join(ROOT, 'include')}", "-x", "c", "-"],
                         input=src, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    lib = linear.load()
    assert len(declared()) == 12
    for name in declared():
        assert getattr(lib, name).argtypes is not None, name


def test_limits_match_the_header():
    text = open(HEADER).read()
    for name in ("LBI_PROJECTION_MAX", "LBI_ATTENTION_MAX_DIM", "LBI_ATTENTION_MAX_H"):
        assert int(re.search(rf"#define {name} (\d+)", text).group(1)) == getattr(linear, name)
    shift = re.search(r"#define LBI_ATTENTION_MAX_LD \(1 << (\d+)\)", text).group(1)
    assert 1 << int(shift) == linear.LBI_ATTENTION_MAX_LD
    for name in ("LBI_ACT_NONE", "LBI_ACT_SILU", "LBI_ACT_GELU"):
        assert int(re.search(rf"{name} = (\d+)", text).group(1)) == getattr(linear, name)


def norm(x=P[0], ldx=64, res=P[1], ldr=64, w=P[2], b=P[5], out=P[3], ldo=64, total=P[4], ldt=64,
         T=5, D=64, eps=1e-5, dt=1, rdt=1):
    return linear.load().lbi_layer_norm(x, ldx, res, ldr, w, b, out, ldo, total, ldt, T, D, eps, dt,
                                        rdt, None)


def test_layer_norm_refusals():
    assert norm(dt=2) == DTYPE and norm(rdt=-1) == DTYPE
    assert norm(D=0) == SHAPE and norm(D=16385) == SHAPE and norm(T=-1) == SHAPE
    assert norm(eps=-1.0) == SHAPE and norm(eps=float("nan")) == SHAPE
    assert norm(ldx=63) == SHAPE and norm(ldo=0) == SHAPE
    assert norm(x=None) == NULL and norm(out=None) == NULL
    assert norm(res=None) == NULL  # residual_out without a residual
    assert norm(x=P[0] + 1) == ALIGN and norm(w=P[2] + 2) == ALIGN and norm(b=P[5] + 1) == ALIGN
    assert norm(out=P[0]) == ALIAS and norm(out=P[5]) == ALIAS
    assert norm(total=P[1], ldt=65) == ALIAS  # in place, but at another stride
    assert norm(T=0, x=None, w=None, b=None, out=None) == 0


def test_layer_norm_backward_refusals():
    need = linear.lbi_layer_norm_backward_workspace_bytes(5, 64)
    assert need > 0 and linear.lbi_layer_norm_backward_workspace_bytes(5, 0) == 0

    def back(dout=P[0], s=P[1], dr=P[3], ldr=64, ds=P[4], dw=P[5], db=P[7], ws=P[6], wsb=need):
        return linear.load().lbi_layer_norm_backward(dout, 64, s, 64, P[2], dr, ldr, ds, 64, dw, db,
                                                     5, 64, 1e-5, 1, 1, ws, wsb, None)
    assert back(wsb=need - 1) == WORKSPACE and back(ws=None) == WORKSPACE
    assert back(ws=P[6] + 16) == ALIGN and back(db=P[7] + 2) == ALIGN
    assert back(dout=None) == NULL and back(s=None) == NULL and back(ds=None) == NULL
    assert back(ds=P[0]) == ALIAS and back(ds=P[3], ldr=66) == ALIAS
    assert back(dw=P[7]) == ALIAS and back(db=P[6]) == ALIAS
    assert back(db=None, ws=None, wsb=0) == WORKSPACE  # dweight alone needs it too


def projection(x=P[0], ldx=64, w=P[1], ldw=64, b=P[2], res=P[3], ldr=96, out=P[4], ldo=96,
               pre=P[5], ldp=96, T=600, K=64, N=96, act=1, dt=1, odt=1, ws=None, wsb=0):
    return linear.load().lbi_projection(x, ldx, w, ldw, b, res, ldr, out, ldo, pre, ldp, T, K, N,
                                        act, dt, odt, ws, wsb, None)


def test_projection_refusals():
    assert projection(dt=2) == DTYPE and projection(odt=7) == DTYPE
    assert projection(act=3) == DTYPE and projection(act=-1) == DTYPE
    assert projection(K=0) == SHAPE and projection(N=65537) == SHAPE and projection(T=-1) == SHAPE
    assert projection(ldx=63) == SHAPE and projection(ldw=1) == SHAPE and projection(ldo=95) == SHAPE
    assert projection(x=None) == NULL and projection(w=None) == NULL and projection(out=None) == NULL
    assert projection(x=P[0] + 1) == ALIGN and projection(b=P[2] + 2) == ALIGN
    assert projection(out=P[0]) == ALIAS and projection(pre=P[4]) == ALIAS
    assert projection(out=P[3], ldr=97) == ALIAS and projection(out=P[1]) == ALIAS
    assert projection(T=0, x=None, w=None, out=None) == 0
    # few rows and a long sum: cut into partial sums
    lib = linear.load()
    need = lib.lbi_projection_workspace_bytes(100, 16384, 96, 1)
    long = dict(T=100, K=16384, ldx=16384, ldw=16384)
    assert need > 0
    assert projection(**long) == WORKSPACE
    assert projection(ws=P[6], wsb=need - 1, **long) == WORKSPACE
    assert projection(ws=P[6] + 8, wsb=need, **long) == ALIGN
    assert projection(ws=P[4], wsb=need, **long) == ALIAS
    assert lib.lbi_projection_workspace_bytes(0, 64, 64, 1) == 0
    assert lib.lbi_projection_workspace_bytes(64, 64, 64, 5) == 0


def test_projection_backward_refusals():
    lib = linear.load()
    need = lib.lbi_projection_backward_workspace_bytes(600, 64, 96, 1, 1, 1)
    assert need > 600 * 96 * 2 and lib.lbi_projection_backward_workspace_bytes(6, 0, 9, 1, 1, 1) == 0

    def back(x=P[0], w=P[1], dout=P[2], pre=P[3], dx=P[4], dw=P[5], ldw=64, db=P[6], act=1, dt=1,
             odt=1, ws=P[7], wsb=need, T=600):
        return lib.lbi_projection_backward(x, 64, w, 64, dout, 96, pre, 96, dx, 64, dw, ldw, db, T,
                                           64, 96, act, dt, odt, ws, wsb, None)
    assert back(dt=4) == DTYPE and back(act=9) == DTYPE and back(T=-2) == SHAPE
    assert back(wsb=need - 1) == WORKSPACE and back(ws=P[7] + 4) == ALIGN
    assert back(dout=None) == NULL and back(pre=None) == NULL
    assert back(w=None) == NULL and back(x=None) == NULL
    assert back(dx=P[0]) == ALIAS and back(dw=P[1]) == ALIAS and back(db=P[5]) == ALIAS
    assert back(dx=P[7]) == ALIAS and back(ldw=60) == SHAPE


def attention_struct(**kw):
    v = dict(q=P[0], ld_q=128, k=P[1], ld_k=64, v=P[2], ld_v=96, log_decay=P[3], state_in=P[4],
             offsets=None, T=6, sequences=2, H=4, KH=2, DK=32, DV=48, scale=0.5, dt=1)
    v.update(kw)
    return linear.AttentionInputs(**v)


def attention(o=P[5], ldo=192, so=P[6], ws=None, wsb=0, slots=None, ns=0, **kw):
    return linear.load().lbi_linear_attention(ctypes.byref(attention_struct(**kw)), o, ldo, so, slots,
                                              ns, ws, wsb, None)


BAD_ATTENTION = (dict(H=0), dict(H=1025), dict(KH=3), dict(KH=0), dict(DK=0), dict(DK=129),
                 dict(DV=0), dict(DV=129), dict(T=7), dict(T=-1), dict(sequences=0),
                 dict(sequences=1 << 32), dict(ld_q=127), dict(ld_k=63), dict(ld_v=95))


def test_attention_refusals():
    lib = linear.load()
    assert lib.lbi_linear_attention(None, P[5], 192, None, None, 0, None, 0, None) == NULL
    assert attention(dt=2) == DTYPE
    for bad in BAD_ATTENTION:
        assert attention(**bad) == SHAPE, bad
    assert attention(ldo=191) == SHAPE and attention(slots=P[8], ns=-1) == SHAPE
    for missing in ("q", "k", "v", "log_decay"):
        assert attention(**{missing: None}) == NULL, missing
    assert attention(o=None) == NULL
    assert attention(q=P[0] + 1) == ALIGN and attention(log_decay=P[3] + 2) == ALIGN
    assert attention(o=P[0]) == ALIAS and attention(so=P[4] + 64) == ALIAS
    assert attention(so=P[5]) == ALIAS and attention(so=P[3]) == ALIAS
    assert attention(T=0, sequences=0, q=None, log_decay=None, o=None) == 0
    # a long sequence of few heads is cut into ranges, which pass states through a workspace
    need = lib.lbi_linear_attention_workspace_bytes(4096, 1, 4, 2, 32, 48, 0, 1)
    assert need > 0 and lib.lbi_linear_attention_workspace_bytes(4096, 1, 4, 3, 32, 48, 0, 1) == 0
    long = dict(T=4096, sequences=1)
    assert attention(**long) == WORKSPACE
    assert attention(ws=P[9], wsb=need - 1, **long) == WORKSPACE
    assert attention(ws=P[9] + 8, wsb=need, **long) == ALIGN
    assert attention(ws=P[1], wsb=need, **long) == ALIAS

    def step(T=2, o=P[5], so=P[6], **kw):
        return lib.lbi_linear_attention_step(ctypes.byref(attention_struct(T=T, **kw)), o, 192, so,
                                             None, 0, None)
    assert step(T=4) == SHAPE and step(offsets=P[10]) == SHAPE and step(o=P[2]) == ALIAS
    assert step(state_in=None) == NULL and step(so=None) == NULL and step(o=None) == NULL


def test_attention_backward_refusals():
    lib = linear.load()
    need = lib.lbi_linear_attention_backward_workspace_bytes(6, 2, 4, 2, 32, 48, 0, 1)
    assert need > 0

    def back(ws=P[20], wsb=need, dout=P[7], grads=None, **kw):
        g = dict(dq=P[8], ld_dq=128, dk=P[9], ld_dk=64, dv=P[10], ld_dv=96, dlog_decay=P[11],
                 dstate_in=P[12])
        g.update(grads or {})
        return lib.lbi_linear_attention_backward(
            ctypes.byref(attention_struct(**kw)), dout, 192, None,
            ctypes.byref(linear.AttentionGradients(**g)), ws, wsb, None)
    assert back(wsb=need - 1) == WORKSPACE and back(ws=P[20] + 64) == ALIGN
    assert back(dout=None) == NULL
    for missing in ("dq", "dk", "dv"):
        assert back(grads={missing: None}) == NULL, missing
    for bad in BAD_ATTENTION:
        assert back(**bad) == SHAPE, bad
    assert back(ws=P[0]) == ALIAS and back(grads={"dq": P[1]}) == ALIAS
    assert back(grads={"dk": P[10]}) == ALIAS and back(grads={"dlog_decay": P[3]}) == ALIAS
    assert back(grads={"dstate_in": P[4] + 4}) == ALIAS and back(grads={"ld_dv": 95}) == SHAPE


def test_python_checks():
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 8)
    heads = torch.zeros(4, 2, 4)
    for call in (lambda: linear.lbi_layer_norm(x), lambda: linear.lbi_projection(x, x),
                 lambda: linear.lbi_linear_attention(heads, heads, heads, x[0, :2]),
                 lambda: linear.lbi_layer_norm(x, stream=3)):
        with pytest.raises(ValueError):
            call()  # not on a GPU
    with pytest.raises(TypeError):
        linear.lbi_linear_attention(heads.half(), heads, heads, x[0, :2])
    with pytest.raises(ValueError):
        linear._act(3)
    assert linear._heads("q", heads, (4,), torch.float32, -1) == (8, 2, 4)
    with pytest.raises(ValueError):
        linear._heads("q", torch.zeros(4, 2, 8)[..., :4], (4,), torch.float32, -1)
    # every entry point is called with its device current
    calls = open(linear.__file__).read()
    assert calls.count("_check(") == 0 and calls.count("    _run(dev, ") == 7
