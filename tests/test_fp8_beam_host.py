"""8-bit cache, beam selection and reordering on the host: sizes and argument checks (no GPU needed).

Every refused call fails its checks, which run before anything is enqueued.
"""

import ctypes
import re

import pytest
import torch

from tests.test_cache_host import BF, _expect, _rope, _seqs


@pytest.fixture(scope="module")
def C():
    from paper_2609_05821_gb300 import _build
    _build.build()
    from paper_2609_05821_gb300 import conduit
    return conduit


def _fp8(C, L=1, P=4, hq=4, hkv=2, d=64, ps=16, R=2, mp=3):
    pool = torch.zeros((L, P, hkv, max(C.fp8_page_bytes(d, ps), 16)), dtype=torch.uint8)
    return C.Fp8Kv(pool, hq, d, ps, torch.zeros((R, mp), dtype=torch.int32))


def _rows(h, L=1, T=3, d=64, dtype=BF):
    return torch.zeros((L, T, h, d), dtype=dtype)


def test_symbols(C):
    import os
    header = open(os.path.join(os.path.dirname(C.__file__), "..", "include", "conduit.h")).read()
    names = set(re.findall(r"\b(conduit_[a-z0-9_]+)\s*\(", re.sub(r"/\*.*?\*/", "", header, flags=re.S)))
    lib = ctypes.CDLL(C.LIB_PATH)
    for name in ("conduit_fp8_page_bytes", "conduit_fp8_append", "conduit_fp8_read", "conduit_fp8_attn",
                 "conduit_fp8_attn_workspace_size", "conduit_beam_select", "conduit_kv_reorder", "conduit_packed_reorder",
                 "conduit_fp8_reorder"):
        assert name in names and hasattr(lib, name)


def test_page_bytes(C):
    assert C.fp8_page_bytes(128, 16) == 32 * 128 + 16
    assert C.fp8_page_bytes(32, 1024) == 64 * (32 * 32 + 16)
    for d, ps in ((16, 16), (288, 16), (120, 16), (128, 8), (128, 24), (128, 2048), (0, 16), (-32, 16), (128, 0), (128, -16)):
        assert C.fp8_page_bytes(d, ps) == -1


def test_cache_refusals(C):
    pool = torch.zeros((1, 4, 2, 32 * 64 + 16), dtype=torch.uint8)
    table = torch.zeros((2, 3), dtype=torch.int32)
    _expect(C, C.ERR_INVALID_ARG, C.Fp8Kv, pool[..., :-16].contiguous(), 4, 64, 16, table, match="bytes")
    _expect(C, C.ERR_INVALID_ARG, C.Fp8Kv, pool.int(), 4, 64, 16, table, match="uint8")
    _expect(C, C.ERR_INVALID_ARG, C.Fp8Kv, pool, 4, 64, 16, table[0], match="page_table")
    _expect(C, C.ERR_UNSUPPORTED, C.Fp8Kv.empty, 1, 4, 4, 2, 64, 8, table, "cpu", match="16")
    # the 4-bit calls do not take an 8-bit cache, nor the other way round
    kv, s = _fp8(C), _seqs(C)
    _expect(C, C.ERR_INVALID_ARG, C.conduit_packed_attn, kv, s, _rows(4), match="PackedKv")
    packed = C.PackedKv(torch.zeros((1, 4, 2, C.packed_page_bytes(64, 16)), dtype=torch.uint8), 4, 64, 16, table)
    _expect(C, C.ERR_INVALID_ARG, C.conduit_fp8_attn, packed, s, _rows(4), match="Fp8Kv")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_fp8_append, packed, s, _rows(2), _rows(2), match="Fp8Kv")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_packed_reorder, kv, torch.zeros(2, dtype=torch.int32), 2, table, table[:, 0], match="PackedKv")


def test_append_refusals(C):
    kv, s = _fp8(C), _seqs(C)
    _expect(C, C.ERR_INVALID_ARG, C.conduit_fp8_append, kv, s, _rows(2), _rows(2, dtype=torch.float32), match="v is")
    _expect(C, C.ERR_UNSUPPORTED, C.conduit_fp8_append, kv, s, _rows(2, dtype=torch.half), _rows(2, dtype=torch.half), match="dtype")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_fp8_append, kv, s, _rows(2, T=4), _rows(2, T=4), match="k is")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_fp8_append, kv, s, _rows(2), _rows(2), _rope(C), None, match="pos")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_fp8_append, kv, _seqs(C, (0, 1, 2, 3)), _rows(2), _rows(2), match="page table")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_fp8_append, kv, s, _rows(2), _rows(2), _rope(C, 128), torch.zeros((2, 3), dtype=torch.int32),
            match="rot_dim")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_fp8_append, _fp8(C, hq=3), s, _rows(2), _rows(2), match="multiple")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_fp8_append, kv, s, _rows(2), _rows(2), None, None, _rows(4),
            torch.zeros((1, 1, 4, 64), dtype=BF).expand(1, 3, 4, 64), match="overlap")
    # no rows: no work
    none = C.Seqs([0, 0, 0], torch.zeros(2, dtype=torch.int32), 40)
    assert C.conduit_fp8_append(kv, none, _rows(2, T=0), _rows(2, T=0)) is None


def test_attention_refusals(C):
    kv, s, q = _fp8(C), _seqs(C), _rows(4)
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    _expect(C, C.ERR_INVALID_ARG, C.conduit_fp8_attn, kv, s, q, scale=-1.0, workspace=ws, match="scale")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_fp8_attn, kv, s, q, scale=float("inf"), workspace=ws, match="scale")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_fp8_attn, kv, s, q, limits=torch.zeros(2, dtype=torch.int32), match="limits")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_fp8_attn, kv, s, q, lse=torch.zeros(5), match="lse")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_fp8_attn, kv, s, _rows(3), match="q is")
    long = C.Seqs([0, 1, 3], torch.zeros(2, dtype=torch.int32), 1 << 20)
    big = _fp8(C, mp=1 << 16)
    need = C.conduit_fp8_attn_workspace_size(big, long)
    assert need > 0
    _expect(C, C.ERR_WORKSPACE, C.conduit_fp8_attn, big, long, q, workspace=torch.zeros(256, dtype=torch.uint8))
    _expect(C, C.ERR_UNSUPPORTED, C.conduit_fp8_attn_workspace_size, _fp8(C, mp=(2 ** 31 - 1) // 16, R=1),
            C.Seqs([0, 1], torch.zeros(1, dtype=torch.int32), 2 ** 31 - 1), match="tokens")


def test_read_refusals(C):
    kv = _fp8(C)
    batch = C.Batch([0, 5, 9], [0, 5, 9], [0, 1, 2], [0, 1, 2], device="cpu")
    k = torch.zeros((1, 2, 9, 64), dtype=BF)
    dst = C.KvCache(k, k.clone(), 4)
    _expect(C, C.ERR_INVALID_ARG, C.conduit_fp8_read, kv, batch, dst, torch.zeros(3, dtype=torch.int32), match="first")
    small = C.KvCache(k[:, :, :8].contiguous(), k[:, :, :8].contiguous(), 4)
    _expect(C, C.ERR_INVALID_ARG, C.conduit_fp8_read, kv, batch, small, match="tokens")
    other = C.KvCache(torch.zeros((1, 2, 9, 32), dtype=BF), torch.zeros((1, 2, 9, 32), dtype=BF), 4)
    _expect(C, C.ERR_INVALID_ARG, C.conduit_fp8_read, kv, batch, other, match="head_dim")


def test_select_refusals(C):
    z, s = torch.zeros((4, 10)), torch.zeros(4)
    _expect(C, C.ERR_INVALID_ARG, C.conduit_beam_select, z, s, 3, match="groups")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_beam_select, z, s, 0, match="groups")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_beam_select, z.t(), torch.zeros(10), 2, match="contiguous")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_beam_select, z, s[:3], 2, match="sums")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_beam_select, z, s.double(), 2, match="sums")
    _expect(C, C.ERR_UNSUPPORTED, C.conduit_beam_select, z.half(), s, 2, match="dtype")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_beam_select, z, s, 2, 0, match="num_out")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_beam_select, z, s, 2, 33, match="num_out")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_beam_select, torch.zeros((33, 10)), torch.zeros(33), 33, match="width")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_beam_select, z[:, :0], s, 2, match="vocab")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_beam_select, z[:1].expand(4, 10), s, 2, match="row_stride")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_beam_select, z, s, 2, 4, score=torch.zeros((2, 3)), match="score")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_beam_select, z, s, 2, 4, token=torch.zeros((2, 4)), match="token")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_beam_select, z, torch.zeros(4, device="meta"), 2, match="sums is on")
    got = C.conduit_beam_select(z[:0], s[:0], 2)
    assert [x.shape for x in got] == [(0, 2)] * 3


def test_select_in_place_refusals(C):
    """Scores over the sums of other groups, which may not have been read."""
    z, buf = torch.zeros((4, 10)), torch.zeros(8)
    _expect(C, C.ERR_INVALID_ARG, C.conduit_beam_select, z, buf[:4], 2, 4, score=buf.view(2, 4), match="may be sums")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_beam_select, z, buf[:4], 2, 1, score=buf[:2].view(2, 1), match="may be sums")


def test_reorder_refusals(C):
    kv = _fp8(C, R=4)
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)
    home = i32((4, 3))
    run = C.conduit_fp8_reorder
    _expect(C, C.ERR_INVALID_ARG, run, kv, i32(4), 3, home, i32(4), match="groups")
    _expect(C, C.ERR_INVALID_ARG, run, kv, i32(4), 2, home[:3].contiguous(), i32(4), match="home")
    _expect(C, C.ERR_INVALID_ARG, run, kv, i32(4), 2, home, i32(3), match="lens")
    _expect(C, C.ERR_INVALID_ARG, run, kv, i32(4).long(), 2, home, i32(4), match="parent")
    _expect(C, C.ERR_INVALID_ARG, run, kv, i32(6), 2, i32((6, 3)), i32(6), match="page table")
    _expect(C, C.ERR_INVALID_ARG, run, _fp8(C, R=33), i32(33), 33, i32((33, 3)), i32(33), match="width")
    flat = torch.zeros((1, 2, 9, 64), dtype=BF)
    _expect(C, C.ERR_UNSUPPORTED, C.conduit_kv_reorder, C.KvCache(flat, flat.clone(), 4), i32(4), 2, home, i32(4), match="paged")
    _expect(C, C.ERR_INVALID_ARG, run, kv, i32(4), 2, kv.page_table, i32(4), match="home")
    run(kv, i32(0), 2, i32((0, 3)), i32(0))  # no groups: no work
