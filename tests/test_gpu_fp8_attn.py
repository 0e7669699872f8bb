"""Attention over the 8-bit cache against softmax attention in 64 bits over the values that the cache stands for.

Tolerances, per (row, head), from what it sees: A = max_j scale sum_i |q_i k_ji| bounds
every logit. Keys, values and (but for a power of two) queries enter exactly in either type, so a logit is off by its
fp32 sum alone, e = (d + 4) 2^-23 A at most (tensor cores truncate: twice a rounding). A
logit error e changes every weight by a factor within e^(+-2 e), so the output is off by
(e^(2 e) - 1) max|V| at most; sums of N terms add N 2^-23 max|V|, weights in fp16 (bf16 rows) 2^-11
of a weight or 2^-32 of the largest, the rounding of a bf16 output 2^-8 |out|. The log-sum-exp is off
by e, and 2^-22 relative for its own arithmetic.
"""

import numpy as np
import pytest
import torch

from tests import cache_reference as R
from tests import fp8_reference as F

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def C():
    from paper_2609_05821_gb300 import _build
    _build.build()
    from paper_2609_05821_gb300 import conduit
    return conduit


def _context(rng, N, hkv, d, k_nan=None, v_nan=None, sizes=0.7):
    """Blocks of N tokens: K with unequal channels and a few large tokens, V of unequal sizes."""
    k = rng.standard_normal((N, hkv, d)) * np.exp(0.5 * rng.standard_normal((1, hkv, d)))
    k[rng.random(N) < 0.05] *= 2
    v = rng.standard_normal((N, hkv, d)) * np.exp(sizes * rng.standard_normal((N, 1, 1)))
    for at, x in ((k_nan, k), (v_nan, v)):
        for j, g, i in at or ():
            x[j, g, i] = np.nan
    heads = []
    for g in range(hkv):
        pair = F.Blocks(N, d), F.Blocks(N, d)
        for b, x in zip(pair, (k, v)):
            if N:
                b.append(0, x[:, g].astype(np.float32))
        heads.append(pair)
    return heads


def _cache(C, seed, L, hq, hkv, d, ps, lens, **kw):
    """An 8-bit cache with those contexts in shuffled pages; everything no token has is 0xFF (NaN codes)."""
    rng = np.random.default_rng(seed)
    need = [-(-n // ps) for n in lens]
    P = sum(need) + 2
    order = rng.permutation(P)
    table = np.full((len(lens), max(max(need), 1)), P + 7, dtype=np.int32)  # pages that no token has do not exist
    pool = np.full((L, P, hkv, C.fp8_page_bytes(d, ps)), 0xFF, dtype=np.uint8)
    step, at, kv = 32 * d + 16, 0, []
    for r, n in enumerate(lens):
        table[r, :need[r]] = order[at:at + need[r]]
        at += need[r]
        per = []
        for l in range(L):
            heads = _context(rng, n, hkv, d, **kw)
            for g, (k, v) in enumerate(heads):
                for b in range(-(-n // 16)):
                    o = 16 * b % ps // 16 * step
                    F.put_block(pool[l, table[r, 16 * b // ps], g, o:o + step], k, v, b)
            per.append(heads)
        kv.append(per)
    return C.Fp8Kv(torch.from_numpy(pool).cuda(), hq, d, ps, torch.from_numpy(table)), kv


def _check(groups, lens, rows, q, limits, out, lse, scale, bf16):
    L, T, hq, d = q.shape
    seen = [max(0, n - c + i + 1) for n, c in zip(lens, rows) for i in range(c)]
    seen = np.array(seen) if limits is None else limits.cpu().numpy().astype(np.int64)
    t = 0
    for r, (n, c) in enumerate(zip(lens, rows)):
        for l in range(L if c else 0):
            k, v = (np.stack([h[w].values(n) for h in groups[r][l]], axis=1) for w in (0, 1))
            s = np.clip(seen[t:t + c], 0, n)
            wo, wl, A, big = R.attend(q[l, t:t + c].double().cpu().numpy(), k, v, s, scale)
            got = out[l, t:t + c].double().cpu().numpy()
            e = (d + 4) * 2.0 ** -23 * A
            tol = (np.expm1(2 * e) + (n + 16) * 2.0 ** -23 + (2.0 ** -11 if bf16 else 0.0)) * big
            tol = tol[..., None] + (2.0 ** -8 if bf16 else 2.0 ** -22) * np.abs(wo)
            tol = np.where(np.isnan(tol), 0, tol)
            assert np.array_equal(np.isnan(got), np.isnan(wo)), (r, l, np.argwhere(np.isnan(got) != np.isnan(wo))[:4])
            some = ~np.isnan(big)  # a NaN value leaves no bound for the other dims of its row: the finite ones are compared below
            bad = ~np.isnan(wo) & ~(np.abs(got - wo) <= tol) & some[..., None]
            assert not bad.any(), (r, l, float(np.nanmax(np.abs(got - wo) - tol)), np.argwhere(bad)[:3])
            if lse is not None:
                gl = lse[l, :, t:t + c].double().cpu().numpy()
                assert np.array_equal(np.isneginf(gl), np.isneginf(wl)) and np.array_equal(np.isnan(gl), np.isnan(wl))
                fin = np.isfinite(wl)
                off = np.abs(np.where(fin, gl, 0) - np.where(fin, wl, 0))
                assert np.all(off[fin] <= (e.T + 2.0 ** -22 * np.abs(wl) + n * 2.0 ** -23 + 2.0 ** -21)[fin]), off[fin].max()
        t += c


def _seqs(C, lens, rows, most=None):
    return C.Seqs(np.concatenate([[0], np.cumsum(rows)]), torch.tensor(lens, dtype=torch.int32, device="cuda"),
                  max(lens) if most is None else most)


# (dtype, L, hq, hkv, d, page, cached tokens, rows, limits)
CASES = [
    (BF, 1, 7, 1, 128, 16, (1,), (1,), None),                          # one token, one key
    (BF, 1, 28, 4, 128, 16, (1025, 31, 32, 33, 0), (1, 1, 1, 1, 1), None),   # an empty context
    (BF, 1, 28, 4, 128, 16, (15, 16, 17, 1), (1, 1, 1, 1), None),
    (BF, 2, 14, 2, 64, 16, (700, 9), (3, 5), None),
    (BF, 1, 6, 2, 96, 32, (257, 64, 65), (2, 0, 9), None),
    (BF, 1, 16, 16, 128, 64, (300, 129), (1, 4), None),                # one query head per KV head
    (BF, 1, 32, 2, 128, 128, (515,), (3,), None),                      # 16 query heads per KV head
    (BF, 1, 9, 3, 128, 16, (5, 40), (9, 40), None),                    # more rows than keys: rows that see nothing
    (BF, 1, 28, 4, 128, 16, (530, 70), (40, 19), "random"),            # limits of their own, some 0
    (BF, 1, 4, 2, 32, 16, (90,), (4,), None),
    (BF, 1, 4, 4, 160, 16, (70,), (2,), "random"),
    (BF, 1, 2, 1, 256, 1024, (1500,), (2,), None),
    (F32, 1, 6, 2, 96, 16, (37, 300), (1, 5), None),
    (F32, 2, 14, 2, 64, 16, (1500, 1, 2000), (1, 1, 3), "random"),
    (F32, 1, 4, 1, 128, 16, (3000,), (1,), None),
    (F32, 1, 3, 3, 256, 32, (95,), (7,), None),
    (F32, 1, 2, 1, 32, 16, (33,), (2,), "random"),
    (BF, 1, 28, 4, 128, 16, (2048, 4100, 777), (64, 33, 150), None),   # query prefixes
    (BF, 1, 28, 4, 96, 64, (1030, 100), (37, 60), "random"),
    (BF, 1, 8, 8, 64, 32, (900,), (200,), None),
    (BF, 2, 8, 2, 128, 16, (130, 0, 128), (128, 0, 65), "random"),
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
    seqs = _seqs(C, lens, rows)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    lse = torch.zeros((L, hq, T), device="cuda")
    out = C.conduit_fp8_attn(kv, seqs, q, limits=lim, lse=lse, status=status)
    assert C.conduit_read_status(status) == C.OK
    _check(groups, lens, rows, q, lim, out, lse, d ** -0.5, dtype == BF)
    again = C.conduit_fp8_attn(kv, seqs, q, limits=lim)
    assert torch.equal(again, out)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [1, 4, 60])
def test_nan_codes_reach_only_rows_that_see_them(C, dtype, rows):
    """NaN keys and values: rows that end before them, in the same tile of keys and in others, stay finite, and a NaN
    value reaches its own dim alone."""
    n = 170
    q = torch.randn((1, rows, 7, 128), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(dtype)
    first = n - rows
    for k_nan, v_nan in (([(first, 0, 3)], None), (None, [(first, 0, 3), (n - 1, 0, 77)]), (None, [(5, 0, 127)])):
        kv, groups = _cache(C, 3, 1, 7, 1, 128, 16, (n,), k_nan=k_nan, v_nan=v_nan)
        limits = torch.arange(rows, dtype=torch.int32, device="cuda") + first  # the first row ends before `first`
        for lim in (limits, None):
            out = C.conduit_fp8_attn(kv, _seqs(C, (n,), (rows,)), q, limits=lim)
            _check(groups, (n,), (rows,), q, lim, out, None, 128 ** -0.5, dtype == BF)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("power", [-100, 60])
def test_query_sizes(C, dtype, power):
    """Queries far outside fp16's range with a scale that makes up for it."""
    lens, rows = (333,), (2,)
    kv, groups = _cache(C, 9, 1, 4, 2, 64, 16, lens)
    q = torch.randn((1, 2, 4, 64), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    q[0, :, 1] *= 2.0 ** -20  # heads of unequal sizes
    q = (q * 2.0 ** power).to(dtype)
    scale = 0.125 * 2.0 ** -power
    lse = torch.zeros((1, 4, 2), device="cuda")
    out = C.conduit_fp8_attn(kv, _seqs(C, lens, rows), q, scale=scale, lse=lse)
    _check(groups, lens, rows, q, None, out, lse, scale, dtype == BF)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [3, 48])
def test_peaked_and_wide_logits(C, dtype, rows):
    """Logits hundreds apart: one key takes all, and running maxima that rise along the context."""
    n = 900
    kv, groups = _cache(C, 11, 1, 4, 2, 128, 16, (n,))
    k = np.stack([h[0].values(n) for h in groups[0][0]], axis=1)
    q = torch.zeros((1, rows, 4, 128))
    for i in range(rows):
        q[0, i] = torch.from_numpy(8 * k[(10, 450, 845)[i % 3]]).float().repeat_interleave(2, 0)
    q = q.to("cuda", dtype)
    lse = torch.zeros((1, 4, rows), device="cuda")
    out = C.conduit_fp8_attn(kv, _seqs(C, (n,), (rows,)), q, lse=lse)
    _check(groups, (n,), (rows,), q, None, out, lse, 128 ** -0.5, dtype == BF)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [1, 40])
def test_scales_far_apart(C, dtype, rows):
    """Blocks of values 2^20 apart in size and blocks of zeros: every block's share is there at its size."""
    n, d = 400, 64
    rng = np.random.default_rng(4)
    kv, groups = _cache(C, 4, 1, 2, 1, d, 16, (n,))
    k = F.Blocks(n, d)
    v = F.Blocks(n, d)
    x = rng.standard_normal((n, d)).astype(np.float32)
    y = rng.standard_normal((n, d)).astype(np.float32)
    for b in range(n // 16):
        y[16 * b:16 * b + 16] *= 2.0 ** (-20 + 40 * (b % 3 == 1)) if b % 3 else 0.0
        x[16 * b:16 * b + 16] *= 2.0 ** (3 * (b % 2))
    k.append(0, x)
    v.append(0, y)
    pool = np.full((1, -(-n // 16), 1, 32 * d + 16), 0xFF, dtype=np.uint8)
    for b in range(n // 16):
        F.put_block(pool[0, b, 0], k, v, b)
    kv = C.Fp8Kv(torch.from_numpy(pool).cuda(), 2, d, 16, torch.arange(n // 16, dtype=torch.int32)[None])
    q = torch.randn((1, rows, 2, d), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").to(dtype)
    for limit in (16, 33, 400):  # the first block holds zeros, the second large values
        lim = torch.full((rows,), limit, dtype=torch.int32, device="cuda")
        lse = torch.zeros((1, 2, rows), device="cuda")
        out = C.conduit_fp8_attn(kv, _seqs(C, (n,), (rows,)), q, limits=lim, lse=lse)
        _check([[[(k, v)]]], (n,), (rows,), q, lim, out, lse, d ** -0.5, dtype == BF)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("sizes", [(0.0, 2.0 ** 68, 1.0), (2.0 ** 68, 0.0, 2.0 ** -30), (2.0 ** -30, 1.0, 2.0 ** 68)])
def test_scales_as_far_apart_as_allowed(C, dtype, rows, sizes):
    """Value scales 2^100 apart, in every order: the smaller blocks' weights still count in the denominator."""
    n, d = 2048, 128
    rng = np.random.default_rng(14)
    k, v = F.Blocks(n, d), F.Blocks(n, d)
    y = rng.uniform(0.5, 1.75, (n, d)).astype(np.float32)  # one sign: a lost denominator shows whole
    for b in range(n // 16):
        y[16 * b:16 * b + 16] *= np.float32(sizes[b % 3])
    k.append(0, 0.1 * rng.standard_normal((n, d)).astype(np.float32))
    v.append(0, y)
    assert max(v.exp) - min(v.exp) <= 100
    pool = np.full((1, n // 16, 1, 32 * d + 16), 0xFF, dtype=np.uint8)
    for b in range(n // 16):
        F.put_block(pool[0, b, 0], k, v, b)
    kv = C.Fp8Kv(torch.from_numpy(pool).cuda(), 2, d, 16, torch.arange(n // 16, dtype=torch.int32)[None])
    q = torch.randn((1, rows, 2, d), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").to(dtype)
    for limit in (17, 33, 49, n):
        lim = torch.full((rows,), limit, dtype=torch.int32, device="cuda")
        lse = torch.zeros((1, 2, rows), device="cuda")
        out = C.conduit_fp8_attn(kv, _seqs(C, (n,), (rows,)), q, limits=lim, lse=lse)
        _check([[[(k, v)]]], (n,), (rows,), q, lim, out, lse, d ** -0.5, dtype == BF)


@pytest.mark.parametrize("rows", [1, 40])
def test_small_weights_keep_their_share(C, rows):
    """A quarter of a million keys whose weights are 2^-24 of the largest one: together 2^-6 of the output."""
    n, d = 1 << 18, 64
    per = n // 1024
    block = np.zeros(32 * d + 16, dtype=np.uint8)
    k, v = F.Blocks(16, d), F.Blocks(16, d)
    k.append(0, np.zeros((16, d), dtype=np.float32))
    v.append(0, np.ones((16, d), dtype=np.float32))
    F.put_block(block, k, v, 0)
    pool = torch.from_numpy(np.tile(block, 64))[None, None, None].cuda().repeat(1, per, 1, 1)
    k0, v0 = F.Blocks(16, d), F.Blocks(16, d)
    x = np.zeros((16, d), dtype=np.float32)
    x[0, 0] = 1.0
    k0.append(0, x)
    y = np.ones((16, d), dtype=np.float32)
    y[0] = 0.0
    v0.append(0, y)
    head = np.zeros(32 * d + 16, dtype=np.uint8)
    F.put_block(head, k0, v0, 0)
    pool[0, 0, 0, :32 * d + 16] = torch.from_numpy(head).cuda()
    kv = C.Fp8Kv(pool, 1, d, 1024, torch.arange(per, dtype=torch.int32)[None])
    q = torch.zeros((1, rows, 1, d), device="cuda", dtype=BF)
    q[..., 0] = 16.0
    scale = 24 * float(np.log(2.0)) / 16.0
    lim = torch.full((rows,), n, dtype=torch.int32, device="cuda")
    out = C.conduit_fp8_attn(kv, _seqs(C, (n,), (rows,)), q, scale=scale, limits=lim)
    w = 2.0 ** -24 * (n - 1)
    want = w / (1 + w)
    assert torch.all((out.double() - want).abs() <= want * (2.0 ** -8 + 2.0 ** -10))


def test_many_chunks_and_growing_lengths(C):
    """A long context cut into chunks; the same call replayed from a graph with lengths that grow."""
    hq, hkv, d, ps, n = 8, 2, 64, 64, 20000
    kv, groups = _cache(C, 21, 1, hq, hkv, d, ps, (n,))
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    seqs = C.Seqs([0, 1], lens, n)
    q = torch.randn((1, 1, hq, d), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(BF)
    out, lse = torch.empty_like(q), torch.empty((1, hq, 1), device="cuda")
    ws = torch.empty(C.conduit_fp8_attn_workspace_size(kv, seqs, BF), dtype=torch.uint8, device="cuda")
    call = lambda: C.conduit_fp8_attn(kv, seqs, q, out=out, lse=lse, workspace=ws)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call()
    torch.cuda.synchronize()
    for now in (n, 1, 17, 4095, 12001, 0):
        lens.fill_(now)
        graph.replay()
        torch.cuda.synchronize()
        _check(groups, (now,), (1,), q, None, out, lse, d ** -0.5, True)


def test_lengths_and_pages_out_of_range(C):
    """A length past the bound is clamped, a page outside of the pool is flagged; nothing else is touched."""
    kv, groups = _cache(C, 8, 1, 4, 2, 128, 16, (60,))
    q = torch.randn((1, 1, 4, 128), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(BF)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = C.conduit_fp8_attn(kv, _seqs(C, (61,), (1,), most=60), q, status=status)
    assert C.conduit_read_status(status) == C.ERR_INDEX
    _check(groups, (60,), (1,), q, None, out, None, 128 ** -0.5, True)
    C.conduit_clear_status(status)
    kv.page_table[0, 1] = -1
    C.conduit_fp8_attn(kv, _seqs(C, (60,), (1,)), q, status=status)
    assert C.conduit_read_status(status) == C.ERR_INDEX


def test_on_a_stream_of_the_callers(C):
    kv, groups = _cache(C, 8, 1, 28, 4, 128, 16, (3000,))
    stream = torch.cuda.Stream()
    for rows in (1, 50):
        q = torch.randn((1, rows, 28, 128), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(BF)
        stream.wait_stream(torch.cuda.current_stream())
        out = C.conduit_fp8_attn(kv, _seqs(C, (3000,), (rows,)), q, stream=stream)
        stream.synchronize()
        _check(groups, (3000,), (rows,), q, None, out, None, 128 ** -0.5, True)
