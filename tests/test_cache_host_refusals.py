"""Calls on growing caches that are refused on the host, and that a refusal changes nothing (no GPU needed).

Every refused call fails its checks before anything is enqueued.
"""

import pytest
import torch

from tests.test_cache_host import BF, C, _append_kw, _expect, _packed, _seqs  # noqa: F401 (C is a fixture)


def _paged(C, R=2, ps=16, mp=3, hkv=2, d=64):
    pool = torch.zeros((1, 4, hkv, ps, d), dtype=BF)
    return C.KvCache(pool, pool.clone(), 4, ps, torch.zeros((R, mp), dtype=torch.int32))


def test_append_needs_a_page_table_row_per_request(C):
    s, kw = _seqs(C, (0, 1, 3)), _append_kw(C)
    _expect(C, C.ERR_INVALID_ARG, C.conduit_kv_append, _paged(C, R=1), s, **kw, match="page table")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_packed_append, _packed(C, R=1), s, **kw, match="page table")


def test_read_needs_a_row_of_the_destinations_page_table_per_request(C):
    batch = C.Batch([0, 5, 9], [0, 5, 9], [0, 1, 2], [0, 1, 2], device="cpu")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_packed_read, _packed(C), batch, _paged(C, R=1), match="page table")


def test_read_refuses_strided_starts(C):
    batch = C.Batch([0, 5, 9], [0, 5, 9], [0, 1, 2], [0, 1, 2], device="cpu")
    dst = C.KvCache(torch.zeros((1, 2, 9, 64), dtype=BF), torch.zeros((1, 2, 9, 64), dtype=BF), 4)
    first = torch.arange(4, dtype=torch.int32)[::2]
    _expect(C, C.ERR_INVALID_ARG, C.conduit_packed_read, _packed(C), batch, dst, first=first, match="first")
