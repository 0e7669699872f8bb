"""Rotary, append and 4-bit cache calls on the host: argument checks (no GPU needed).

Every call here fails its checks, which run before anything is enqueued.
"""

import ctypes

import pytest
import torch

BF = torch.bfloat16


@pytest.fixture(scope="module")
def C():
    from paper_2609_05821_gb300 import _build
    _build.build()
    from paper_2609_05821_gb300 import conduit
    return conduit


def _expect(C, code, fn, *args, match=None, **kw):
    with pytest.raises(C.ConduitError, match=match) as ei:
        fn(*args, **kw)
    assert ei.value.code == code, str(ei.value)


def _rope(C, rot=64, axis=None, layout="halves", n=10):
    return C.Rope(torch.zeros((n, rot // 2, 2)), axis or [0, 1] * (rot // 4), layout)


def _seqs(C, off=(0, 1, 3), max_len=40):
    return C.Seqs(list(off), torch.zeros(len(off) - 1, dtype=torch.int32), max_len)


def _packed(C, L=1, P=4, hq=4, hkv=2, d=64, ps=16, R=2, mp=3):
    pool = torch.zeros((L, P, hkv, max(C.packed_page_bytes(d, ps), 16)), dtype=torch.uint8)
    return C.PackedKv(pool, hq, d, ps, torch.zeros((R, mp), dtype=torch.int32))


def test_page_bytes(C):
    assert C.packed_page_bytes(128, 16) == 16 * 160
    assert C.packed_page_bytes(32, 8) == 8 * 40
    assert C.packed_page_bytes(256, 1024) == 1024 * 320
    for d, ps in ((16, 16), (288, 16), (120, 16), (128, 4), (128, 24), (128, 2048), (0, 16), (-32, 16), (128, 0), (128, -8)):
        assert C.packed_page_bytes(d, ps) == -1


def test_rope_refusals(C):
    x, pos = torch.zeros((3, 2, 64), dtype=BF), torch.zeros((2, 3), dtype=torch.int32)
    r = _rope(C)
    _expect(C, C.ERR_INVALID_ARG, C.conduit_rope, r, x, pos[:1].contiguous(), match="pos")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_rope, r, x, pos.long(), match="pos")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_rope, r, x, None, match="pos")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_rope, _rope(C, 128), x, pos, match="rot_dim")
    _expect(C, C.ERR_UNSUPPORTED, C.conduit_rope, r, x.half(), pos, match="dtype")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_rope, r, x.transpose(1, 2), pos)
    _expect(C, C.ERR_INVALID_ARG, C.conduit_rope, r, x, pos, out=torch.zeros((3, 2, 32), dtype=BF), match="out")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_rope, r, x, pos, out=torch.zeros((3, 2, 64)), match="out")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_rope, r, x, pos, out=torch.zeros((3, 1, 64), dtype=BF).expand(3, 2, 64),
            match="overlap")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_rope, _rope(C, axis=[0, 1, 2, 4] * 8), x,
            torch.zeros((5, 3), dtype=torch.int32), match="num_axes")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_rope, _rope(C, axis=[0, -1] * 16), x, pos[:1].contiguous(), match="axis")
    _expect(C, C.ERR_UNSUPPORTED, C.conduit_rope, r, torch.zeros((3, 2, 258), dtype=BF), pos, match="head_dim")
    _expect(C, C.ERR_INVALID_ARG, C.Rope, torch.zeros((4, 8, 2)), [0] * 7, match="axis")
    _expect(C, C.ERR_INVALID_ARG, C.Rope, torch.zeros((4, 8, 2)), [0] * 8, "rows", match="layout")
    _expect(C, C.ERR_INVALID_ARG, C.Rope, torch.zeros((4, 8, 2), dtype=torch.float64), [0] * 8, match="table")


def _append_kw(C, L=1, T=3, hq=4, hkv=2, d=64, dtype=BF):
    row = lambda h: torch.zeros((L, T, h, d), dtype=dtype)
    return dict(k=row(hkv), v=row(hkv), q=row(hq), q_out=row(hq))


def test_kv_append_refusals(C):
    pool = torch.zeros((1, 4, 2, 16, 64), dtype=BF)
    kv = C.KvCache(pool, pool.clone(), 4, 16, torch.zeros((2, 3), dtype=torch.int32))
    s, kw = _seqs(C), _append_kw(C)
    flat = torch.zeros((1, 2, 64, 64), dtype=BF)
    _expect(C, C.ERR_UNSUPPORTED, C.conduit_kv_append, C.KvCache(flat, flat.clone(), 4), s, **kw, match="paged")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_kv_append, kv, s, **{**kw, "k": kw["k"].float()})
    _expect(C, C.ERR_INVALID_ARG, C.conduit_kv_append, kv, s, **{**kw, "v": kw["v"].float()}, match="v is")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_kv_append, kv, s, **{**kw, "k": kw["k"][:, :2]}, match="k is")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_kv_append, kv, _seqs(C, (0, 3, 2)), **_append_kw(C, T=2), match="non-decreasing")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_kv_append, kv, _seqs(C, (1, 1, 3)), **kw, match="start at 0")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_kv_append, kv, _seqs(C, max_len=-1), **kw, match="max_len")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_kv_append, kv, s, **kw, rope=_rope(C), match="pos")
    _expect(C, C.ERR_INVALID_ARG, C.Seqs, [0, 1], torch.zeros(2, dtype=torch.int32), 4, match="lens")
    _expect(C, C.ERR_INVALID_ARG, C.Seqs, [0, 1], torch.zeros(1), 4, match="lens")
    # straight through the ABI: q without q_out
    k = C._rows(kw["k"], "k", 1, 3, 2, 64)
    code = C._lib.conduit_kv_append(kv.ref(), s.ref(), None, None, k, k, k, None, None, None)
    assert code == C.ERR_INVALID_ARG and b"together" in C._lib.conduit_last_error_string()
    assert C._lib.conduit_kv_append(kv.ref(), None, None, None, k, k, None, None, None, None) == C.ERR_INVALID_ARG


def test_packed_refusals(C):
    s, kw = _seqs(C), _append_kw(C)
    for bad in (dict(d=48), dict(ps=12), dict(ps=4), dict(d=288)):
        kv = _packed(C, **bad)
        d = bad.get("d", 64)
        _expect(C, C.ERR_UNSUPPORTED, C.conduit_packed_append, kv, s, **_append_kw(C, d=d), match="head_dim")
        _expect(C, C.ERR_UNSUPPORTED, C.conduit_packed_attn, kv, s, torch.zeros((1, 3, 4, d), dtype=BF), match="head_dim")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_packed_append, _packed(C, hq=3), s, **_append_kw(C, hq=3), match="multiple")
    _expect(C, C.ERR_INVALID_ARG, C.PackedKv, torch.zeros((1, 4, 2, 100), dtype=torch.uint8), 4, 64, 16,
            torch.zeros((2, 3), dtype=torch.int32), match="bytes")
    kv = _packed(C)
    _expect(C, C.ERR_UNSUPPORTED, C.conduit_packed_append, kv, s, **_append_kw(C, dtype=torch.float16), match="dtype")
    q = torch.zeros((1, 3, 4, 64), dtype=BF)
    ws = torch.zeros(8, dtype=torch.uint8)
    _expect(C, C.ERR_INVALID_ARG, C.conduit_packed_attn, kv, s, q[:, :2], match="q is")
    for scale in (-1.0, float("nan"), float("inf")):
        _expect(C, C.ERR_INVALID_ARG, C.conduit_packed_attn, kv, s, q, scale=scale, match="scale")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_packed_attn, kv, s, q, limits=torch.zeros(2, dtype=torch.int32), match="limits")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_packed_attn, kv, s, q, lse=torch.zeros((1, 4, 2)), match="lse")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_packed_attn, _packed(C, R=1), s, q, match="page table")
    # a context of many chunks with a workspace that is too small
    long = _packed(C, mp=40000)
    big = _seqs(C, max_len=600000)
    assert C.conduit_packed_attn_workspace_size(long, big) > 8
    _expect(C, C.ERR_WORKSPACE, C.conduit_packed_attn, long, big, q, workspace=ws)
    # straight through the ABI: dtype, NULL pointers
    n = ctypes.c_size_t(0)
    assert C._lib.conduit_packed_attn_workspace_size(kv.ref(), s.ref(), 2, ctypes.byref(n)) == C.ERR_INVALID_ARG
    assert C._lib.conduit_packed_attn_workspace_size(kv.ref(), s.ref(), 1, None) == C.ERR_INVALID_ARG
    assert C._lib.conduit_packed_attn(kv.ref(), s.ref(), 1, None, 0.0, None, None, None, None, 0, None,
                                      None) == C.ERR_INVALID_ARG


def test_packed_read_refusals(C):
    kv = _packed(C)
    batch = C.Batch([0, 5, 9], [0, 5, 9], [0, 1, 2], [0, 1, 2], device="cpu")
    flat = lambda L=1, h=2, d=64: C.KvCache(torch.zeros((L, h, 9, d), dtype=BF), torch.zeros((L, h, 9, d), dtype=BF), 2 * h)
    for dst in (flat(L=2), flat(h=1), flat(d=32)):
        _expect(C, C.ERR_INVALID_ARG, C.conduit_packed_read, kv, batch, dst, match="dst")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_packed_read, kv, batch, flat(), first=torch.zeros(1, dtype=torch.int32), match="first")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_packed_read, _packed(C, R=1), batch, flat(), match="page table")
    bad = C.Batch([0, 0, 9], [0, 0, 9], [0, 1, 2], [0, 1, 2], device="cpu")
    _expect(C, C.ERR_INVALID_ARG, C.conduit_packed_read, kv, bad, flat())


def test_calls_without_rows_do_nothing(C):
    s = _seqs(C, (0, 0, 0))
    empty = dict(k=torch.zeros((1, 0, 2, 64), dtype=BF), v=torch.zeros((1, 0, 2, 64), dtype=BF))
    before = C.conduit_launch_count()
    assert C.conduit_packed_append(_packed(C), s, **empty) is None
    C.conduit_packed_attn(_packed(C), s, torch.zeros((1, 0, 4, 64), dtype=BF))
    assert C.conduit_launch_count() == before
