"""Limits of the region block's entry points that need no GPU: refusals by size, before any pointer
is used."""
import os

import pytest
import torch

from paper_2605_09204_amd import binding, block
from test_block_abi import SHAPE, scan

pytestmark = pytest.mark.skipif(not os.path.exists(binding.library_path()),
                                reason="library not built")


def test_more_sequences_than_can_be_numbered():
    n = (1 << 32) + 8
    assert scan(T=n, sequences=n) == SHAPE
    lib = block.load()
    assert lib.lbi_ssm_scan_workspace_bytes(1 << 24, 1 << 24, 1536, 16, 1, 0) == 0  # no ranges to join


def test_build_refuses_scratch():
    from paper_2605_09204_amd import build

    text = ("remark: Function Name: a [-R]\nremark:     ScratchSize [bytes/lane]: 0 [-R]\n"
            "remark:     VGPRs Spill: 0 [-R]\nremark: Function Name: b [-R]\n"
            "remark:     ScratchSize [bytes/lane]: 20 [-R]\nremark:     SGPRs Spill: 20 [-R]\n"
            "remark:     VGPRs Spill: 0 [-R]\nremark: Function Name: c [-R]\n"
            "remark:     ScratchSize [bytes/lane]: 8 [-R]\nremark:     VGPRs Spill: 2 [-R]\n")
    assert build.spills(text) == ["b", "c"]


def test_sizes_that_32_bits_do_not_hold():
    """They were cut to 32 bits: a group of 2^32 + 128 features wrote scales for groups of 128."""
    assert block._int32("n", (1 << 31) - 1) == (1 << 31) - 1 and block._int32("n", -5) == -5
    for size in (1 << 31, (1 << 32) + 128, -(1 << 31) - 1):
        with pytest.raises(ValueError):
            block._int32("n", size)
    with pytest.raises(ValueError):
        block._batch((6, 8), None, (1 << 64) + 1, 0)
    meta = torch.empty((1 << 32) + 2, 2, 8, device="meta")
    with pytest.raises(ValueError, match="out of range"):
        block._states(meta, None, torch.empty(1, dtype=torch.int32), 1, (2, 8), torch.float32, 0)
