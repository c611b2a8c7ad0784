"""The region block's entry points (include/lbi_block.h) are declared, exported and refuse bad
arguments before anything reaches the GPU (runs without a GPU: no call here gets that far)."""
import ctypes
import os
import re
import subprocess

import pytest

from paper_2605_09204_amd import binding, block

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "lbi_block.h")

pytestmark = pytest.mark.skipif(not os.path.exists(binding.library_path()),
                                reason="library not built")

NULL, SHAPE, DTYPE, WORKSPACE, ALIGN, ALIAS = 1, 2, 3, 5, 7, 8
STEP = 1 << 32  # fake device addresses, far apart: never dereferenced, only validated
P = [STEP * (i + 1) for i in range(24)]


def declared():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    return sorted(set(re.findall(r"\b(lbi_[a-z0-9_]+)\s*\(", text)))


def test_header_compiles_as_c_and_every_function_is_exported():
    src = '#include "lbi_block.h"\nint main(void){return LBI_SSM_MAX_N == 64 ? 0 : 1;}\n'
    res = subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-fsyntax-only",
                          f"-I{os.path.join(ROOT, 'include')}", "-x", "c", "-"],
                         input=src, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    lib = block.load()
    assert len(declared()) == 13
    for name in declared():
        assert getattr(lib, name).argtypes is not None, name


def test_limits_match_the_header():
    text = open(HEADER).read()
    for name in ("LBI_NORM_MAX_D", "LBI_SSM_MAX_D", "LBI_SSM_MAX_N", "LBI_CONV_MAX_W"):
        assert int(re.search(rf"#define {name} (\d+)", text).group(1)) == getattr(block, name)


def norm(x=P[0], ldx=64, res=P[1], ldr=64, w=P[2], out=P[3], ldo=64, total=P[4], ldt=64, T=5, D=64,
         eps=1e-5, dt=1, rdt=1):
    return block.load().lbi_rms_norm(x, ldx, res, ldr, w, out, ldo, total, ldt, T, D, eps, dt, rdt,
                                     None)


def test_norm_refusals():
    assert norm(dt=2) == DTYPE and norm(rdt=-1) == DTYPE
    assert norm(D=0) == SHAPE and norm(D=16385) == SHAPE and norm(T=-1) == SHAPE
    assert norm(eps=-1.0) == SHAPE and norm(eps=float("nan")) == SHAPE
    assert norm(ldx=63) == SHAPE and norm(ldo=0) == SHAPE
    assert norm(x=None) == NULL and norm(w=None) == NULL and norm(out=None) == NULL
    assert norm(res=None) == NULL  # residual_out without a residual
    assert norm(x=P[0] + 1) == ALIGN and norm(w=P[2] + 2) == ALIGN
    assert norm(out=P[0]) == ALIAS and norm(out=P[1] + 8) == ALIAS
    assert norm(total=P[1], ldt=65) == ALIAS  # in place, but at another stride
    assert norm(total=P[3] + 128) == ALIAS
    assert norm(T=0, x=None, w=None, out=None) == 0


def q8(q=P[3], ldq=64, scales=P[5], T=5, D=64, group=32, fmt=0, dt=1):
    return block.load().lbi_rms_norm_q8(P[0], 64, None, 0, P[2], q, ldq, scales, None, 0, T, D, 1e-5,
                                        group, fmt, dt, dt, None)


def test_norm_q8_refusals():
    assert q8(fmt=2) == DTYPE and q8(dt=5) == DTYPE
    assert q8(group=16) == SHAPE and q8(group=-32) == SHAPE and q8(group=256) == SHAPE
    assert q8(scales=None) == NULL and q8(q=None) == NULL
    assert q8(scales=P[3] + 64) == ALIAS and q8(scales=P[5] + 2) == ALIGN
    assert q8(T=0, q=None, scales=None) == 0


def norm_backward(dout=P[0], s=P[1], w=P[2], dr=P[3], ds=P[4], dw=P[5], T=5, D=64, ws=P[6],
                  wsb=None, ldr=64):
    need = block.lbi_rms_norm_backward_workspace_bytes(T, D)
    return block.load().lbi_rms_norm_backward(dout, 64, s, 64, w, dr, ldr, ds, 64, dw, T, D, 1e-5,
                                              1, 1, ws, need if wsb is None else wsb, None)


def test_norm_backward_refusals():
    need = block.lbi_rms_norm_backward_workspace_bytes(5, 64)
    assert need > 0 and block.lbi_rms_norm_backward_workspace_bytes(-1, 64) == 0
    assert norm_backward(wsb=need - 1) == WORKSPACE and norm_backward(ws=None) == WORKSPACE
    assert norm_backward(ws=P[6] + 16) == ALIGN
    assert norm_backward(s=None) == NULL and norm_backward(ds=None) == NULL
    assert norm_backward(ds=P[0]) == ALIAS and norm_backward(ds=P[3], ldr=66) == ALIAS
    assert norm_backward(dw=P[6]) == ALIAS and norm_backward(ws=P[1] & ~255) == ALIAS


def conv(x=P[0], ldx=64, w=P[1], out=P[2], si=P[3], so=P[4], slots=None, ns=0, off=None, T=6, B=2,
         D=64, W=4, dt=1):
    return block.load().lbi_ssm_conv(x, ldx, w, None, out, 64, si, so, slots, ns, off, T, B, D, W,
                                     1, dt, None)


def test_conv_refusals():
    assert conv(dt=3) == DTYPE
    assert conv(W=1) == SHAPE and conv(W=5) == SHAPE and conv(D=0) == SHAPE
    assert conv(T=7) == SHAPE and conv(B=0) == SHAPE and conv(T=-2) == SHAPE
    assert conv(T=7, off=P[9], so=P[3] + 64) == ALIAS  # the states overlap, but are not the same
    assert conv(ldx=(1 << 23) + 1) == SHAPE and conv(ldx=8) == SHAPE
    assert conv(slots=P[5], ns=-1) == SHAPE
    assert conv(x=None) == NULL and conv(w=None) == NULL and conv(out=None) == NULL
    assert conv(out=P[0] + 64) == ALIAS and conv(out=P[3]) == ALIAS
    assert conv(T=0, B=0, x=None, out=None) == 0
    lib = block.load()

    def step(si=P[3], so=P[4], n=2, out=P[2]):
        return lib.lbi_ssm_conv_step(P[0], 64, P[1], None, out, 64, si, so, None, 0, n, 64, 4, 1, 1,
                                     None)
    assert step(si=None) == NULL and step(so=None) == NULL and step(n=-1) == SHAPE
    assert step(out=P[0]) == ALIAS and step(n=0, si=None, so=None) == 0

    def back(T=6, ws=P[10], dw=P[6], dx=P[5], B=2):
        need = block.lbi_ssm_conv_backward_workspace_bytes(T, 64, 4)
        return lib.lbi_ssm_conv_backward(P[0], 64, P[1], None, P[2], 64, P[3], P[4], dx, 64, dw,
                                         None, P[7], None, T, B, 64, 4, 1, 1, ws, need, None)
    assert back(ws=None) == WORKSPACE and back(dw=None) == NULL and back(T=7) == SHAPE
    assert back(dx=P[0]) == ALIAS and back(dw=P[10] + 256) == ALIAS


def scan_struct(**kw):
    v = dict(u=P[0], ld_u=64, delta=P[1], ld_delta=64, z=P[2], ld_z=64, B=P[3], ld_B=32, C=P[4],
             ld_C=32, A=P[5], skip=None, delta_bias=None, state_in=P[6], offsets=None, T=6,
             sequences=2, D=64, N=16, G=2, softplus=1, dt=1)
    v.update(kw)
    return block.SsmInputs(**v)


def scan(y=P[8], so=P[9], ws=None, wsb=0, slots=None, ns=0, **kw):
    return block.load().lbi_ssm_scan(ctypes.byref(scan_struct(**kw)), y, 64, so, slots, ns, ws, wsb,
                                     None)


def test_scan_refusals():
    lib = block.load()
    assert lib.lbi_ssm_scan(None, P[8], 64, None, None, 0, None, 0, None) == NULL
    assert scan(dt=4) == DTYPE
    for bad in (dict(N=0), dict(N=65), dict(G=0), dict(G=3), dict(D=0), dict(D=65537), dict(T=7),
                dict(T=-1), dict(sequences=0), dict(ld_u=63), dict(ld_B=31),
                dict(ld_delta=(1 << 23) + 1)):
        assert scan(**bad) == SHAPE, bad
    assert scan(slots=P[11], ns=-2) == SHAPE
    for missing in ("u", "delta", "B", "C", "A"):
        assert scan(**{missing: None}) == NULL, missing
    assert scan(y=None) == NULL
    assert scan(u=P[0] + 1) == ALIGN and scan(A=P[5] + 2) == ALIGN
    assert scan(y=P[0]) == ALIAS and scan(so=P[5]) == ALIAS and scan(so=P[6] + 64) == ALIAS
    assert scan(T=0, sequences=0, u=None, A=None, y=None) == 0
    # long sequences of few channels are cut into ranges, which pass states through a workspace
    need = block.lbi_ssm_scan_workspace_bytes(4096, 1, 64, 16, 2, False)
    assert need > 0 and block.lbi_ssm_scan_workspace_bytes(4096, 1, 64, 65, 2, False) == 0
    long = dict(T=4096, sequences=1)
    assert scan(**long) == WORKSPACE and scan(ws=P[12], wsb=need - 1, **long) == WORKSPACE
    assert scan(ws=P[12] + 8, wsb=need, **long) == ALIGN
    assert scan(ws=P[1], wsb=need, **long) == ALIAS

    def step(T=2, y=P[8], so=P[9], **kw):
        return lib.lbi_ssm_scan_step(ctypes.byref(scan_struct(T=T, **kw)), y, 64, so, None, 0, None)
    assert step(T=4) == SHAPE and step(offsets=P[10]) == SHAPE
    assert step(state_in=None) == NULL and step(so=None) == NULL and step(y=P[2]) == ALIAS


def test_scan_backward_refusals():
    lib = block.load()
    need = block.lbi_ssm_scan_backward_workspace_bytes(6, 2, 64, 16, 2, False)
    assert need > 0

    def back(ws=P[20], wsb=need, dy=P[7], grads=None, **kw):
        g = dict(du=P[8], ld_du=64, ddelta=P[9], ld_ddelta=64, dz=P[10], ld_dz=64, dB=P[11],
                 ld_dB=64, dC=P[11] + 64, ld_dC=64, dA=P[13], dskip=None, ddelta_bias=None,
                 dstate_in=P[14])
        g.update(grads or {})
        return lib.lbi_ssm_scan_backward(ctypes.byref(scan_struct(**kw)), dy, 64, None,
                                         ctypes.byref(block.SsmGradients(**g)), ws, wsb, None)
    assert back(wsb=need - 1) == WORKSPACE and back(dy=None) == NULL
    for missing in ("du", "ddelta", "dz", "dB", "dC", "dA"):
        assert back(grads={missing: None}) == NULL, missing
    # dB and dC side by side in the rows of one tensor are apart, one element nearer they are not
    assert back(ws=P[0]) == ALIAS and back(grads={"dC": P[11] + 62}) == ALIAS
    assert back(grads={"du": P[1]}) == ALIAS and back(grads={"dA": P[13] + 1}) == ALIGN
    assert back(grads={"ld_dB": (1 << 23) + 1}) == SHAPE


def test_python_checks():
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 8)
    for call in (lambda: block.lbi_rms_norm(x, x[0]), lambda: block.lbi_ssm_conv(x, x[:8]),
                 lambda: block.lbi_ssm_scan(x, x, x, x, x)):
        with pytest.raises(ValueError):
            call()  # not on a GPU
    with pytest.raises(ValueError):
        block._row_stride("x", (2, 3, 4), (24, 4, 1))  # sequences of another stride
    with pytest.raises(ValueError):
        block._row_stride("x", (3, 4), (8, 2))
    assert block._row_stride("x", (2, 3, 4), (30, 10, 1)) == 10
    assert block._row_stride("x", (5, 1, 4), (10, 4, 1)) == 10
    assert block._row_stride("x", (3, 4), (0, 1)) == 0  # a broadcast row: the library refuses it


def test_build_refuses_register_spills():
    from paper_2605_09204_amd import build

    text = ("remark: Function Name: a [-R]\nremark:     VGPRs Spill: 0 [-R]\n"
            "remark: Function Name: b [-R]\nremark:     SGPRs Spill: 9 [-R]\n"
            "remark:     VGPRs Spill: 3 [-R]\n")
    assert build.spills(text) == ["b"]
