"""Limits of the region block's entry points that need no GPU: refusals by size, before any pointer
is used."""
import os

import pytest

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
