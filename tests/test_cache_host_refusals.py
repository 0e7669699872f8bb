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


def _contexts(C, lens=(5, 7)):
    from paper_2609_05821_gb300 import context
    ctx = context.PackedContexts(len(lens), 40, 1, 4, 2, 64, device="cpu")
    ctx.lens.copy_(torch.tensor(lens, dtype=torch.int32))
    return ctx


@pytest.mark.parametrize("rows,given", [([3, 2], 4), ([3], 3), ([3, 2, 1], 6), ([6, -1], 5), ([], 0)])
def test_a_refused_append_leaves_the_lengths(C, rows, given):
    ctx = _contexts(C)
    kw = _append_kw(C, T=given)
    _expect(C, C.ERR_INVALID_ARG, ctx.append, rows, kw["k"], kw["v"])
    assert ctx.lens.tolist() == [5, 7]
    _expect(C, C.ERR_INVALID_ARG, ctx.attend, rows, kw["q"])


def test_a_refused_step_leaves_the_lengths(C):
    ctx = _contexts(C)
    step = ctx.decoder()
    for bad in (dict(d=32), dict(T=3), dict(dtype=torch.float32)):
        kw = _append_kw(C, **{"T": 2, **bad})
        with pytest.raises(C.ConduitError):
            step(kw["q"], kw["k"], kw["v"])
        assert ctx.lens.tolist() == [5, 7]


def test_attention_refuses_contexts_whose_chunks_pass_32_bits(C):
    """A key's place is counted in 32 bits, whole chunks past the last key included."""
    pages = 2 ** 21 - 1  # of 1024 tokens
    pool = torch.zeros((1, 1, 1, C.packed_page_bytes(64, 1024)), dtype=torch.uint8)
    kv = C.PackedKv(pool, 1, 64, 1024, torch.zeros((1, pages), dtype=torch.int32))
    for dtype in (BF, torch.float32):
        for max_len in (2 ** 31 - 1, 2 ** 31 - 2 ** 20 + 1):
            seqs = _seqs(C, (0, 1), max_len)
            _expect(C, C.ERR_UNSUPPORTED, C.conduit_packed_attn_workspace_size, kv, seqs, dtype, match="tokens")
            _expect(C, C.ERR_UNSUPPORTED, C.conduit_packed_attn, kv, seqs, torch.zeros((1, 1, 1, 64), dtype=dtype),
                    workspace=torch.zeros(8, dtype=torch.uint8), match="tokens")
        assert C.conduit_packed_attn_workspace_size(kv, _seqs(C, (0, 1), 2 ** 31 - 2 ** 20), dtype) > 0
        narrow = _packed(C)  # what the table holds counts, where that is less
        assert C.conduit_packed_attn_workspace_size(narrow, _seqs(C, (0, 1), 2 ** 31 - 1), dtype) == 0


@pytest.mark.parametrize("tokens", [8, 10])
def test_read_refuses_a_destination_of_other_tokens(C, tokens):
    """A contiguous cache of the batch's 9 tokens is written with their stride; any other size is not one."""
    batch = C.Batch([0, 5, 9], [0, 5, 9], [0, 1, 2], [0, 1, 2], device="cpu")
    dst = C.KvCache(torch.zeros((1, 2, tokens, 64), dtype=BF), torch.zeros((1, 2, tokens, 64), dtype=BF), 4)
    _expect(C, C.ERR_INVALID_ARG, C.conduit_packed_read, _packed(C), batch, dst, match="tokens")
