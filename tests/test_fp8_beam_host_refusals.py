"""Calls of the 8-bit cache and of beam search that are refused before anything is enqueued (no GPU needed)."""

import pytest
import torch

from tests.test_cache_host import _expect
from tests.test_fp8_beam_host import _fp8


@pytest.fixture(scope="module")
def C():
    from paper_2609_05821_gb300 import _build
    _build.build()
    from paper_2609_05821_gb300 import conduit
    return conduit


def test_a_plain_reordering_takes_a_plain_cache(C):
    """A quantised cache's record is another one than a plain cache's."""
    i32 = lambda *n: torch.zeros(n, dtype=torch.int32)
    packed = C.PackedKv(torch.zeros((1, 4, 2, C.packed_page_bytes(64, 16)), dtype=torch.uint8), 4, 64, 16, i32(4, 3))
    for kv in (_fp8(C, R=4), packed):
        _expect(C, C.ERR_INVALID_ARG, C.conduit_kv_reorder, kv, i32(4), 2, i32(4, 3), i32(4), match="KvCache")
