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
