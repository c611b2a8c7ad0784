"""Which kernels the calls of test_gpu_linear_tiles.py and test_gpu_linear_ranges.py take: the tiles of
a projection's products and the ranges of an attention's tokens, from the library's own rules (host
code, runs without a GPU).  A rule that changes has to leave every kernel a call that is tested."""
import ctypes
import os

import pytest

from paper_2605_09204_amd import binding, linear

pytestmark = pytest.mark.skipif(not os.path.exists(binding.library_path()),
                                reason="library not built")

F32, BF16 = 0, 1


class ProductArgs(ctypes.Structure):
    """ProductArgs of csrc/lbi_linear_internal.h."""

    _fields_ = [(n, t) for names, t in (
        (("a", "b"), ctypes.c_void_p), (("ld_a", "ld_b"), ctypes.c_int64),
        (("a_cols", "b_cols"), ctypes.c_bool), (("M", "K"), ctypes.c_int64),
        (("N",), ctypes.c_int32), (("bias", "residual"), ctypes.c_void_p),
        (("ld_residual",), ctypes.c_int64), (("out",), ctypes.c_void_p),
        (("ld_out",), ctypes.c_int64), (("pre",), ctypes.c_void_p), (("ld_pre",), ctypes.c_int64),
        (("act",), ctypes.c_int), (("bf16", "out_bf16"), ctypes.c_bool),
        (("partial",), ctypes.c_void_p), (("splits",), ctypes.c_int32), (("split",), ctypes.c_int64),
        (("tile_m", "tile_n"), ctypes.c_int32)) for n in names]


def product_plan(M, K, N, dt, a_cols=False, b_cols=False):
    """(tile_m, tile_n, cuts of the sum)."""
    plan = getattr(linear.load(), "_ZN3lbi12plan_productERNS_11ProductArgsE")
    plan.argtypes, plan.restype = [ctypes.POINTER(ProductArgs)], ctypes.c_int64
    a = ProductArgs(M=M, K=K, N=N, bf16=dt == BF16, a_cols=a_cols, b_cols=b_cols)
    floats = plan(ctypes.byref(a))
    assert floats == (a.splits * M * N if a.splits > 1 else 0)
    return a.tile_m, a.tile_n, a.splits


def forward_plan(T, K, N, dt):
    return product_plan(T, K, N, dt)


def dx_plan(T, K, N, dt):
    return product_plan(T, N, K, dt, b_cols=True)


def dweight_plan(T, K, N, dt):
    return product_plan(N, T, K, dt, a_cols=True, b_cols=True)


# T, K, N and the plan in bf16 and float32.  Each tile comes with rows that whole 16-byte pieces hold
# and with odd ones, which go through registers; T, K and N leave remainders of the tiles and the
# stages.
WHOLE, WIDE = (128, 128, 1), (128, 64, 1)
FORWARD = [((8189, 200, 1032), WHOLE, WHOLE), ((8189, 203, 1030), WHOLE, WHOLE),
           ((4100, 200, 1000), WIDE, WHOLE), ((4099, 77, 999), WIDE, WHOLE),
           ((1000, 4104, 520), (128, 128, 11), (128, 128, 12)),
           ((1000, 4101, 517), (128, 128, 11), (128, 128, 12)),
           ((2100, 4104, 1032), WHOLE, WHOLE)]
DX = [((8189, 1032, 200), WHOLE, WHOLE), ((8189, 1030, 203), WHOLE, WHOLE),
      ((4100, 1000, 200), WIDE, WHOLE), ((4099, 999, 77), WIDE, WHOLE),
      ((1000, 520, 4104), (128, 128, 11), (128, 128, 12)),
      ((1000, 517, 4101), (128, 128, 11), (128, 128, 12))]
DWEIGHT = [((200, 4104, 2056), WHOLE, WHOLE), ((203, 4101, 2055), WHOLE, WHOLE),
           ((200, 2056, 2056), WIDE, WHOLE), ((77, 2055, 2057), WIDE, WHOLE),
           ((4104, 520, 1000), (128, 128, 11), (128, 128, 12)),
           ((4101, 517, 999), (128, 128, 11), (128, 128, 12))]


@pytest.mark.parametrize("plan,cases", [(forward_plan, FORWARD), (dx_plan, DX),
                                        (dweight_plan, DWEIGHT)])
def test_products_take_their_tiles(plan, cases):
    for sizes, bf16, f32 in cases:
        assert plan(*sizes, BF16) == bf16 and plan(*sizes, F32) == f32, sizes


def test_float32_products_have_no_tiles_of_128_by_64():
    """Fewer than 192 tiles of 128 x 128 are fewer than 384 of 128 x 64."""
    for M in range(1, 6000, 61):
        for N in range(1, 6000, 57):
            for K in (100, 5000):
                assert product_plan(M, K, N, F32)[:2] in ((128, 128), (64, 64))


class AttentionCut(ctypes.Structure):
    """AttentionCut of csrc/lbi_linear_internal.h."""

    _fields_ = [("ranges", ctypes.c_int64), ("tokens", ctypes.c_int64),
                ("per_sequence", ctypes.c_int32), ("joined", ctypes.c_bool)]


def attention_plan(lengths, H, KH, DK, DV, dt, backward):
    """(tiles of 64 tokens a range, ranges, whether states pass between ranges, values a thread of the
    carry)."""
    cut = getattr(linear.load(), "_ZN3lbi13attention_cutERK20lbi_attention_inputsbb")
    cut.argtypes = [ctypes.POINTER(linear.AttentionInputs), ctypes.c_bool, ctypes.c_bool]
    cut.restype = AttentionCut
    ragged = len(set(lengths)) > 1
    a = linear.AttentionInputs(T=sum(lengths), sequences=len(lengths), H=H, KH=KH, DK=DK, DV=DV,
                               dt=dt)
    c = cut(ctypes.byref(a), ragged, backward)
    chains = (1 if ragged else len(lengths)) * (2 if backward else 1)
    wide = DK * DV % 4 == 0 and chains * H * DK * DV // 4 >= 256 * 256
    return c.tokens // 64, c.ranges, c.joined, (4 if wide else 1) if c.joined else 0


# Lengths, H, KH, DK, DV, whose ranges of several tiles pass states on, forward and in the gradient, in
# both types: heads that fill the tiles' widths and heads that do not, equal sequences, one, and packed
# ones that begin in the middle of a range or last over several; both forms of the carry.
PACKED = [300, 1, 0, 1203, 64]
RANGES = [([520] * 3, 54, 18, 64, 64), (PACKED, 66, 22, 64, 64), ([1500], 72, 72, 64, 64),
          (PACKED, 48, 48, 48, 101), ([900] * 2, 36, 12, 48, 101), ([1500], 48, 48, 48, 101),
          (PACKED, 66, 22, 40, 56), (PACKED, 24, 8, 128, 128), ([700] * 2, 24, 24, 128, 128),
          (PACKED, 48, 48, 64, 128), (PACKED, 48, 48, 128, 64)]


def test_attention_is_cut_into_ranges_of_several_tiles():
    carries = {False: set(), True: set()}
    for lengths, H, KH, DK, DV in RANGES:
        for dt in (F32, BF16):
            for backward in (False, True):
                tiles, ranges, joined, carry = attention_plan(lengths, H, KH, DK, DV, dt, backward)
                assert joined and tiles >= 3 and ranges >= 4, (lengths, H, DK, DV, dt, backward)
                carries[backward].add((carry, len(set(lengths)) > 1))
    # the gradient's carry of single values is that of few heads (test_gpu_linear_use.py)
    assert carries[False] >= {(1, True), (4, True), (4, False), (1, False)}
    assert carries[True] >= {(4, True), (4, False)}
    for lengths in ([5001], [4100, 31, 1500, 0, 900]):
        assert attention_plan(lengths, 1, 1, 12, 20, BF16, True)[2:] == (True, 1)
