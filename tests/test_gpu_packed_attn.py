"""Attention over the 4-bit cache against softmax attention in 64 bits over the values that the cache stands for.

Tolerances, per (row, head), from what it sees: A = max_j scale sum_i |q_i k_ji| bounds
every logit. fp32 rows: a logit is off by at most d 2^-23 A; bf16 rows run with fp16
operands, so keys may be rounded by 2^-11 and a logit by (d 2^-23 + 2^-11) A more. A
logit error e changes every weight by a factor within e^(+-2 e), so the output is off by
(e^(2 e) - 1) max|V| at most; sums of N terms add N 2^-24 max|V|, fp16 weights and
values 2^-10 max|V|, the rounding of a bf16 output 2^-8 |out|. The log-sum-exp is off
by e, and 2^-22 relative for its own arithmetic.
"""

import numpy as np
import pytest
import torch

from tests import cache_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def C():
    from paper_2609_05821_gb300 import _build
    _build.build()
    from paper_2609_05821_gb300 import conduit
    return conduit


def _context(rng, N, hkv, d, nan_at=None):
    """Packed groups of N tokens: K with unequal channels and a few large tokens, V of unequal sizes."""
    k = rng.standard_normal((N, hkv, d)) * np.exp(0.5 * rng.standard_normal((1, hkv, d)))
    k[rng.random(N) < 0.05] *= 2
    v = rng.standard_normal((N, hkv, d)) * np.exp(0.7 * rng.standard_normal((N, 1, 1)))
    if nan_at is not None:
        k[nan_at], v[nan_at] = np.nan, np.nan
    return R.pack_groups(k), R.pack_groups(v)


def _cache(C, seed, L, hq, hkv, d, ps, lens, device="cuda", pages_past=0, nan_at=None):
    """A 4-bit cache with those contexts in shuffled pages; everything no token has is 0xFF (NaN parameters)."""
    rng = np.random.default_rng(seed)
    need = [-(-n // ps) for n in lens]
    P = sum(need) + 2
    order = rng.permutation(P)
    table = np.full((len(lens), max(max(need), 1)), P + 7, dtype=np.int32)  # pages that no token has do not exist
    pool = np.full((L, P, hkv, C.packed_page_bytes(d, ps)), 0xFF, dtype=np.uint8)
    kv, at = [], 0
    G, half = d // 32, ps * d // 2
    for r, n in enumerate(lens):
        table[r, :need[r]] = order[at:at + need[r]]
        per = []
        for l in range(L):
            groups = _context(rng, n, hkv, d, nan_at)
            per.append(groups)
            for p in range(need[r]):
                rows = slice(p * ps, min(n, (p + 1) * ps))
                c = rows.stop - rows.start
                for g in range(hkv):
                    rec = R.page_record(*[a[rows, g] for part in groups for a in part])
                    w = pool[l, table[r, p], g]
                    w[:c * d // 2] = rec[:c * d // 2]
                    w[half:half + c * d // 2] = rec[c * d // 2:c * d]
                    w[2 * half:2 * half + c * 4 * G] = rec[c * d:c * d + c * 4 * G]
                    o = 2 * half + ps * 4 * G
                    w[o:o + c * 4 * G] = rec[c * d + c * 4 * G:]
        kv.append(per)
        at += need[r]
    return C.PackedKv(torch.from_numpy(pool).to(device), hq, d, ps, torch.from_numpy(table)), kv


def _check(C, kv, groups, lens, rows, q, limits, out, lse, scale, bf16):
    L, T, hq, d = q.shape
    want_seen = []
    for n, c in zip(lens, rows):
        want_seen += [max(0, n - c + i + 1) for i in range(c)]
    seen = np.array(want_seen) if limits is None else limits.cpu().numpy().astype(np.int64)
    t = 0
    for r, (n, c) in enumerate(zip(lens, rows)):
        for l in range(L if c else 0):
            k, v = (R.values(*part) for part in groups[r][l])
            s = np.clip(seen[t:t + c], 0, n)
            wo, wl, A, big = R.attend(q[l, t:t + c].double().cpu().numpy(), k, v, s, scale)
            got = out[l, t:t + c].double().cpu().numpy()
            e = (d * 2.0 ** -23 + (2.0 ** -11 if bf16 else 0.0)) * A
            tol = (np.expm1(2 * e) + (n + 16) * 2.0 ** -24 + (2.0 ** -10 if bf16 else 0.0)) * big
            tol = tol[..., None] + (2.0 ** -8 if bf16 else 2.0 ** -22) * np.abs(wo)
            assert np.array_equal(np.isnan(got), np.isnan(wo)), (r, l)
            bad = ~np.isnan(wo) & ~(np.abs(got - wo) <= tol)
            assert not bad.any(), (r, l, float(np.nanmax(np.abs(got - wo) - tol)), np.argwhere(bad)[:3])
            if lse is not None:
                gl = lse[l, :, t:t + c].double().cpu().numpy()
                assert np.array_equal(np.isneginf(gl), np.isneginf(wl)) and np.array_equal(np.isnan(gl), np.isnan(wl))
                fin = np.isfinite(wl)
                assert np.all(np.abs(gl - wl)[fin] <= (e.T + 2.0 ** -22 * np.abs(wl) + n * 2.0 ** -24 + 2.0 ** -21)[fin])
        t += c


BF, F = torch.bfloat16, torch.float32
# (dtype, L, hq, hkv, d, page, cached tokens, rows, limits)
CASES = [
    (BF, 1, 7, 1, 128, 16, (1,), (1,), None),                          # one token, one key
    (BF, 1, 28, 4, 128, 16, (1025, 31, 32, 33, 0), (1, 1, 1, 1, 1), None),   # an empty context
    (BF, 2, 14, 2, 64, 8, (700, 9), (3, 5), None),
    (BF, 1, 6, 2, 96, 32, (257, 64, 65), (2, 0, 9), None),
    (BF, 1, 16, 16, 128, 64, (300, 129), (1, 4), None),                # one query head per KV head
    (BF, 1, 32, 2, 128, 128, (515,), (3,), None),                      # 16 query heads per KV head
    (BF, 1, 9, 3, 128, 16, (5, 40), (9, 40), None),                    # more rows than keys: rows that see nothing
    (BF, 1, 28, 4, 128, 16, (530, 70), (40, 19), "random"),            # limits of their own, some 0
    (BF, 1, 4, 2, 32, 16, (90,), (4,), None),
    (BF, 1, 4, 4, 160, 8, (70,), (2,), "random"),
    (BF, 1, 2, 1, 256, 1024, (1500,), (2,), None),
    (F, 1, 6, 2, 96, 8, (37, 300), (1, 5), None),
    (F, 2, 14, 2, 64, 8, (1500, 1, 2000), (1, 1, 3), "random"),
    (F, 1, 4, 1, 128, 16, (3000,), (1,), None),
    (F, 1, 3, 3, 256, 32, (95,), (7,), None),
    (BF, 1, 28, 4, 128, 16, (2048, 4100, 777), (64, 33, 150), None),   # query prefixes
    (BF, 1, 8, 8, 64, 32, (900,), (200,), None),
]


@pytest.mark.parametrize("dtype,L,hq,hkv,d,ps,lens,rows,limits", CASES)
def test_attention(C, dtype, L, hq, hkv, d, ps, lens, rows, limits):
    kv, groups = _cache(C, d + len(lens), L, hq, hkv, d, ps, lens)
    T = sum(rows)
    gen = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn((L, T, hq + 2, d), generator=gen, device="cuda").to(dtype)
    q = x[:, :, 1:1 + hq]  # rows of a wider projection
    lim = None
    if limits:
        n = torch.repeat_interleave(torch.tensor(lens), torch.tensor(rows))
        lim = (torch.rand(T, generator=torch.Generator().manual_seed(5)) * (n + 1)).int()
        lim[::3] = 0
        lim[1::5] = n[1::5].int() + 100  # past the context: clamped
        lim = lim.cuda()
    seqs = C.Seqs(np.concatenate([[0], np.cumsum(rows)]), torch.tensor(lens, dtype=torch.int32, device="cuda"), max(lens))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    lse = torch.zeros((L, hq, T), device="cuda")
    out = C.conduit_packed_attn(kv, seqs, q, limits=lim, lse=lse, status=status)
    assert C.conduit_read_status(status) == C.OK
    _check(C, kv, groups, lens, rows, q, lim, out, lse, d ** -0.5, dtype == BF)
    again = C.conduit_packed_attn(kv, seqs, q, limits=lim)
    assert torch.equal(again, out)


@pytest.mark.parametrize("dtype", [BF, F])
def test_nan_tokens_reach_only_rows_that_see_them(C, dtype):
    """A token packed from NaN: rows that end before it, in the same tile of keys and in others, stay finite."""
    lens, rows, nan_at = (170,), (60,), 140
    kv, groups = _cache(C, 3, 1, 7, 1, 128, 16, lens, nan_at=nan_at)
    q = torch.randn((1, 60, 7, 128), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(dtype)
    seqs = C.Seqs([0, 60], torch.tensor(lens, dtype=torch.int32, device="cuda"), 170)
    out = C.conduit_packed_attn(kv, seqs, q)
    _check(C, kv, groups, lens, rows, q, None, out, None, 128 ** -0.5, dtype == BF)
    assert torch.isfinite(out[0, :30]).all() and torch.isnan(out[0, 30:].float()).all()
    # a NaN in the values alone
    k, v = groups[0][0]
    clean, _ = _cache(C, 3, 1, 7, 1, 128, 16, lens)
    kv.pool[..., :16 * 64] = clean.pool[..., :16 * 64]
    at = 16 * 128
    kv.pool[..., at:at + 16 * 16] = clean.pool[..., at:at + 16 * 16]
    out = C.conduit_packed_attn(kv, seqs, q)
    assert torch.isfinite(out[0, :30]).all() and torch.isnan(out[0, 30:].float()).all()


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("power", [-100, 60])
def test_query_sizes(C, dtype, power):
    """Queries far outside fp16's range with a scale that makes up for it."""
    lens, rows = (333,), (2,)
    kv, groups = _cache(C, 9, 1, 4, 2, 64, 16, lens)
    q = torch.randn((1, 2, 4, 64), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    q[0, :, 1] *= 2.0 ** -20  # heads of unequal sizes
    q = (q * 2.0 ** power).to(dtype)
    seqs = C.Seqs([0, 2], torch.tensor(lens, dtype=torch.int32, device="cuda"), 333)
    scale = 0.125 * 2.0 ** -power
    lse = torch.zeros((1, 4, 2), device="cuda")
    out = C.conduit_packed_attn(kv, seqs, q, scale=scale, lse=lse)
    _check(C, kv, groups, lens, rows, q, None, out, lse, scale, dtype == BF)


@pytest.mark.parametrize("dtype", [BF, F])
def test_peaked_and_wide_logits(C, dtype):
    """Logits hundreds apart: one key takes all, and running maxima that rise along the context."""
    lens, rows = (900,), (3,)
    kv, groups = _cache(C, 11, 1, 4, 2, 128, 16, lens)
    k = R.values(*groups[0][0][0])
    q = torch.zeros((1, 3, 4, 128))
    for i, j in enumerate((10, 450, 880)):
        q[0, i] = torch.from_numpy(8 * k[j]).float().repeat_interleave(2, 0)
    q = q.to("cuda", dtype)
    seqs = C.Seqs([0, 3], torch.tensor(lens, dtype=torch.int32, device="cuda"), 900)
    lse = torch.zeros((1, 4, 3), device="cuda")
    out = C.conduit_packed_attn(kv, seqs, q, lse=lse)
    _check(C, kv, groups, lens, rows, q, None, out, lse, 128 ** -0.5, dtype == BF)


def test_many_chunks_and_growing_lengths(C):
    """A long context cut into chunks; the same call replayed from a graph with lengths that grow."""
    L, hq, hkv, d, ps, n = 1, 8, 2, 64, 64, 20000
    kv, groups = _cache(C, 21, L, hq, hkv, d, ps, (n,))
    q = torch.randn((1, 1, hq, d), generator=torch.Generator(device="cuda").manual_seed(4), device="cuda").to(BF)
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    seqs = C.Seqs([0, 1], lens, n)
    ws = torch.empty(C.conduit_packed_attn_workspace_size(kv, seqs), dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(q), torch.zeros((1, hq, 1), device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    call = lambda: C.conduit_packed_attn(kv, seqs, q, out=out, lse=lse, workspace=ws, status=status)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for m in (1, 255, 256, 257, 1024, 19999, n):
        lens.fill_(m)
        ws.fill_(0xFF)  # what a workspace held before reaches no result
        graph.replay()
        torch.cuda.synchronize()
        _check(C, kv, groups, (m,), (1,), q, None, out, lse, d ** -0.5, True)
    assert C.conduit_read_status(status) == C.OK


def test_lengths_and_pages_out_of_range(C):
    """Bad device data is flagged, without a fault."""
    kv, _ = _cache(C, 2, 1, 4, 2, 64, 16, (64, 64))
    q = torch.randn((1, 2, 4, 64), device="cuda").to(BF)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    lens = torch.tensor([64, 64], dtype=torch.int32, device="cuda")
    seqs = C.Seqs([0, 1, 2], lens, 64)
    good = C.conduit_packed_attn(kv, seqs, q)
    for bad in (65, 1 << 30, -1):
        lens[0] = bad
        C.conduit_clear_status(status)
        out = C.conduit_packed_attn(kv, seqs, q, status=status)
        assert C.conduit_read_status(status) == C.ERR_INDEX
        assert torch.equal(out[0, 1], good[0, 1])
    assert torch.all(out[0, 0] == 0)  # -1 counts as 0 keys
    lens[0] = 64
    kv.page_table[0, 2] = 1 << 20
    C.conduit_clear_status(status)
    out = C.conduit_packed_attn(kv, seqs, q, status=status)
    assert C.conduit_read_status(status) == C.ERR_INDEX
    assert torch.equal(out[0, 1], good[0, 1])


def test_many_rows_that_see_nothing(C):
    """Contexts far shorter than the call's rows, in more CTAs than SMs: blocks of rows without a key are zeros."""
    lens, rows = (1, 3, 0, 2) * 12, (90, 128, 60, 41) * 12
    kv, groups = _cache(C, 31, 1, 28, 4, 128, 16, lens)
    T = sum(rows)
    q = torch.randn((1, T, 28, 128), generator=torch.Generator(device="cuda").manual_seed(6), device="cuda").to(BF)
    seqs = C.Seqs(np.concatenate([[0], np.cumsum(rows)]), torch.tensor(lens, dtype=torch.int32, device="cuda"), 3)
    lse = torch.zeros((1, 28, T), device="cuda")
    for _ in range(4):
        out = C.conduit_packed_attn(kv, seqs, q, lse=lse)
        t = 0
        for n, c in zip(lens, rows):
            assert torch.all(out[0, t:t + c - n] == 0) and torch.all(lse[0, :, t:t + c - n] == -float("inf"))
            t += c
        assert torch.isfinite(out.float()).all()
    _check(C, kv, groups, lens, rows, q, None, out, lse, 128 ** -0.5, True)


# Rows of an odd number of column tiles and more blocks than SMs: the blocks with one tile are cut into
# key chunks of their own, those with two are not.
LAST_IN_CHUNKS = [
    (BF, 2, 16, 16, 64, 16, (1500, 1340, 700, 3, 1024), (44, 139, 28, 131, 146), "random"),
    (BF, 2, 16, 16, 64, 32, (2300, 2049, 60, 769, 2300), (32, 41, 138, 142, 148), None),
]


@pytest.mark.parametrize("dtype,L,hq,hkv,d,ps,lens,rows,limits", LAST_IN_CHUNKS)
def test_last_blocks_in_chunks(C, dtype, L, hq, hkv, d, ps, lens, rows, limits):
    table = torch.zeros((len(lens), -(-max(lens) // ps)), dtype=torch.int32)
    kv = C.PackedKv.empty(L, 1, hq, hkv, d, ps, table)
    seqs = C.Seqs(np.concatenate([[0], np.cumsum(rows)]), torch.tensor(lens, dtype=torch.int32, device="cuda"), max(lens))
    per_chunk = L * len(lens) * hkv * 128 * (4 * d + 8)  # partial results of one tile per request and KV head
    assert 2 * per_chunk <= C.conduit_packed_attn_workspace_size(kv, seqs, dtype) <= 8 * per_chunk + 256
    test_attention(C, dtype, L, hq, hkv, d, ps, lens, rows, limits)


def test_other_stream(C):
    kv, groups = _cache(C, 8, 1, 8, 2, 128, 16, (777,))
    q = torch.randn((1, 1, 8, 128), device="cuda").to(BF)
    seqs = C.Seqs([0, 1], torch.tensor([777], dtype=torch.int32, device="cuda"), 777)
    want = C.conduit_packed_attn(kv, seqs, q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = C.conduit_packed_attn(kv, seqs, q)
    side.synchronize()
    assert torch.equal(got, want)


def test_context_past_four_gigabytes(C):
    """Pages whose offset does not fit in 32 bits."""
    hkv, d, ps = 4, 128, 16
    P = (1 << 32) // (hkv * ps * 160) + 100
    small, groups = _cache(C, 13, 1, 28, hkv, d, ps, (50,))
    table = torch.tensor([[P - 1, 3, P - 50, P - 2]], dtype=torch.int32)
    pool = torch.empty((1, P, hkv, ps * 160), dtype=torch.uint8, device="cuda")
    pool[:, table[0].long().cuda()] = small.pool[:, small.page_table[0].long()]
    kv = C.PackedKv(pool, 28, d, ps, table)
    q = torch.randn((1, 1, 28, d), device="cuda").to(BF)
    seqs = C.Seqs([0, 1], torch.tensor([50], dtype=torch.int32, device="cuda"), 50)
    assert torch.equal(C.conduit_packed_attn(kv, seqs, q), C.conduit_packed_attn(small, seqs, q))
    f = q.float()
    assert torch.equal(C.conduit_packed_attn(kv, seqs, f), C.conduit_packed_attn(small, seqs, f))
