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


def test_sizes_past_32_bits_are_not_cut(C):
    """A vocabulary, candidates or groups of 2^32 and a few are not the few."""
    meta = lambda *n, dtype=torch.bfloat16: torch.empty(n, dtype=dtype, device="meta")
    f32, i32 = torch.float32, torch.int32
    for vocab in (2 ** 31, 2 ** 32 + 5):
        _expect(C, C.ERR_UNSUPPORTED, C.conduit_beam_select, meta(2, vocab), meta(2, dtype=f32), 2, match="vocab")
    for groups in (2 ** 31, 2 ** 32 + 2):
        _expect(C, C.ERR_UNSUPPORTED, C.conduit_beam_select, meta(groups, 4), meta(groups, dtype=f32), 1, match="groups")
    _expect(C, C.ERR_UNSUPPORTED, C.conduit_beam_select, meta(2, 4), meta(2, dtype=f32), 2, 2 ** 32 + 2, match="num_out")
    table = meta(2 ** 32 + 2, 1, dtype=i32)
    pool = torch.zeros((1, 4, 2, C.fp8_page_bytes(64, 16)), dtype=torch.uint8, device="meta")
    kv = C.Fp8Kv(pool, 4, 64, 16, table)
    n = 2 ** 32 + 2
    _expect(C, C.ERR_UNSUPPORTED, C.conduit_fp8_reorder, kv, meta(n, dtype=i32), 1, meta(n, 1, dtype=i32), meta(n, dtype=i32), match="groups")
