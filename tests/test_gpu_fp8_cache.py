"""Append to the 8-bit cache and the read back, bit for bit against numpy; bytes that no token has stay as they were."""

import numpy as np
import pytest
import torch

from tests import fp8_reference as F

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def C():
    from paper_2609_05821_gb300 import _build
    _build.build()
    from paper_2609_05821_gb300 import conduit
    return conduit


class Cache:
    """An 8-bit cache of shuffled pages beside its plain form."""

    def __init__(self, C, seed, L, hq, hkv, d, ps, R, capacity):
        rng = np.random.default_rng(seed)
        self.C, self.rng, self.ps, self.d = C, rng, ps, d
        per = -(-capacity // ps)
        self.table = rng.permutation(R * per + 2)[:R * per].reshape(R, per).astype(np.int32)
        self.bytes = np.full((L, R * per + 2, hkv, C.fp8_page_bytes(d, ps)), 0xA5, dtype=np.uint8)
        self.kv = C.Fp8Kv(torch.from_numpy(self.bytes).cuda(), hq, d, ps, torch.from_numpy(self.table))
        self.plain = [[[(F.Blocks(per * ps, d), F.Blocks(per * ps, d)) for _ in range(hkv)] for _ in range(R)] for _ in range(L)]

    def put(self):
        """The plain form's blocks into the expected bytes."""
        step = 32 * self.d + 16
        for l, requests in enumerate(self.plain):
            for r, heads in enumerate(requests):
                for g, (k, v) in enumerate(heads):
                    for b, e in enumerate(k.exp):
                        if e is not None:
                            rec = self.bytes[l, self.table[r, 16 * b // self.ps], g]
                            at = 16 * b % self.ps // 16 * step
                            F.put_block(rec[at:at + step], k, v, b)
        return self.bytes


def _turn(rows, pos, rope):
    if rope is None:
        return rows
    table, axis, layout = rope
    return F.rotate32(rows, pos, table, axis, layout)


# (dtype, L, hq, hkv, d, page, rot, layout, appended per request and call)
CASES = [
    (BF, 1, 7, 1, 128, 16, 128, "halves", [(1,), (1,), (14,), (1,), (40,)]),
    (BF, 2, 4, 2, 64, 32, 32, "halves", [(37, 16, 0), (3, 1, 5), (0, 15, 11)]),
    (BF, 1, 6, 3, 96, 16, 96, "pairs", [(20, 33), (13, 1)]),
    (F32, 1, 2, 2, 32, 64, 20, "halves", [(70, 1), (1, 62)]),
    (F32, 2, 3, 3, 128, 16, 0, "halves", [(17,), (2,)]),
    (BF, 1, 2, 1, 160, 16, 64, "pairs", [(19, 5), (3, 3)]),
    (F32, 1, 4, 2, 256, 128, 256, "halves", [(150,), (30,)]),
    (BF, 1, 5, 5, 32, 16, 14, "pairs", [(9, 31), (8, 2)]),
]


@pytest.mark.parametrize("dtype,L,hq,hkv,d,ps,rot,layout,calls", CASES)
@pytest.mark.parametrize("strided", [False, True])
def test_append_and_read(C, dtype, L, hq, hkv, d, ps, rot, layout, calls, strided):
    R = len(calls[0])
    most = max(sum(c[r] for c in calls) for r in range(R)) + 3
    cache = Cache(C, d + R, L, hq, hkv, d, ps, R, most)
    gen = torch.Generator(device="cuda").manual_seed(d)
    axis = [i % 2 for i in range(rot // 2)]
    table = C.rope_table(10000.0, rot, 300) if rot else None
    rope = C.Rope(table, axis, layout) if rot else None
    lens = torch.zeros(R, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    total = [0] * R
    for n_call, rows in enumerate(calls):
        T = sum(rows)
        x = torch.randn((L, T, hq + 2 * hkv + 1, d), generator=gen, device="cuda")
        # tokens of unequal size, larger ones later: scales that grow over earlier tokens
        x *= torch.exp(torch.randn((L, T, 1, 1), generator=gen, device="cuda") + 1.5 * n_call)
        x[:, :, hq] *= 1e-3
        x = x.to(dtype)
        q, k, v = x[:, :, :hq], x[:, :, hq:hq + hkv], x[:, :, hq + hkv:hq + 2 * hkv]
        if not strided:
            q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
        pos = torch.randint(0, 300, (2, T), dtype=torch.int32, generator=gen, device="cuda")
        total = [a + b for a, b in zip(total, rows)]
        lens.copy_(torch.tensor(total, dtype=torch.int32))
        seqs = C.Seqs(np.concatenate([[0], np.cumsum(rows)]), lens, most)
        q_rot = C.conduit_fp8_append(cache.kv, seqs, k, v, rope, pos if rot else None, q, status=status)
        plain = (table.cpu().numpy(), axis, layout) if rot else None
        kf, vf, at = k.float().cpu().numpy(), v.float().cpu().numpy(), 0
        for r, n in enumerate(rows):
            for l in range(L if n else 0):
                turned = _turn(kf[l, at:at + n], pos[:, at:at + n].cpu().numpy(), plain)
                for g in range(hkv):
                    cache.plain[l][r][g][0].append(total[r] - n, turned[:, g])
                    cache.plain[l][r][g][1].append(total[r] - n, vf[l, at:at + n, g])
            at += n
        assert C.conduit_read_status(status) == C.OK
        got = cache.kv.pool.cpu().numpy()
        assert np.array_equal(got, cache.put()), np.argwhere(got != cache.bytes)[:4]
        if rot:
            assert torch.equal(q_rot, C.conduit_rope(rope, q, pos))
        else:
            assert torch.equal(q_rot, q)
    # back, from a start inside of a block, to a contiguous and a paged cache of either type
    first = [min(2 + r, n - 1) for r, n in enumerate(total)]
    n_read = [n - f for n, f in zip(total, first)]
    off = np.concatenate([[0], np.cumsum(n_read)])
    ids = list(range(R + 1))
    batch = C.Batch(off, off, ids, ids)
    for paged in (0, 24):
        for to in (BF, F32):
            if paged:
                per = -(-max(n_read) // paged)
                pages = torch.randperm(R * per, generator=torch.Generator().manual_seed(1)).view(R, per).int()
                shape = (L, R * per, hkv, paged, d)
                dst = C.KvCache(torch.full(shape, 7.0, dtype=to, device="cuda"), torch.full(shape, 7.0, dtype=to, device="cuda"),
                                hq, paged, pages)
            else:
                shape = (L, hkv, int(off[-1]), d)
                dst = C.KvCache(torch.full(shape, 7.0, dtype=to, device="cuda"), torch.full(shape, 7.0, dtype=to, device="cuda"), hq)
            C.conduit_fp8_read(cache.kv, batch, dst, torch.tensor(first, dtype=torch.int32, device="cuda"), status=status)
            assert C.conduit_read_status(status) == C.OK
            for l in range(L):
                for r in range(R):
                    for g in range(hkv):
                        for which, tensor in ((0, dst.k), (1, dst.v)):
                            want = cache.plain[l][r][g][which].values(total[r])[first[r]:]
                            want = torch.from_numpy(want).to(to)
                            if paged:
                                got = tensor[l, pages[r].long(), g].reshape(-1, d).cpu()
                                assert (got[n_read[r]:] == 7.0).all()
                                got = got[:n_read[r]]
                            else:
                                got = tensor[l, g, off[r]:off[r + 1]].cpu()
                            assert torch.equal(got, want)


def test_ends_of_the_range(C):
    """Zeros, numbers at the ends of fp32 and between codes, and tops at the border of an exponent."""
    d, ps = 64, 16
    cache = Cache(C, 1, 1, 1, 1, d, ps, 1, 96)
    x = np.zeros((96, 1, d), dtype=np.float32)
    x[16:32] = 2.0 ** -45 * np.arange(d) / 7
    x[32:48] = np.linspace(-3.4e38, 3.4e38, d)
    x[48:64, 0, 3] = np.float32(448.0) * np.float32(2.0 ** -3)
    x[64:80, 0, 3] = np.nextafter(np.float32(56.0), np.float32(57.0))
    x[80:96] = (np.arange(16)[:, None, None] * d + np.arange(d)) * 448.0 / 1023  # between all codes
    rows = torch.from_numpy(x)[None].cuda()
    lens = torch.tensor([96], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    C.conduit_fp8_append(cache.kv, C.Seqs([0, 96], lens, 96), rows, -rows, status=status)
    assert C.conduit_read_status(status) == C.OK
    for g, (k, v) in enumerate(cache.plain[0][0]):
        k.append(0, x[:, 0])
        v.append(0, -x[:, 0])
    got, want = cache.kv.pool.cpu().numpy(), cache.put()
    assert np.array_equal(got, want), np.argwhere(got != want)[:4]


@pytest.mark.parametrize("dtype", [BF, F32])
def test_what_is_not_finite(C, dtype):
    """A NaN or an infinity is held as NaN, leaves the others of its block alone and is flagged."""
    cache = Cache(C, 2, 1, 2, 2, 128, 16, 1, 48)
    x = torch.randn((1, 40, 2, 128), generator=torch.Generator().manual_seed(1)).to(dtype)
    y = torch.randn((1, 40, 2, 128), generator=torch.Generator().manual_seed(2)).to(dtype)
    x[0, 3, 0, 5], x[0, 17, 1, 9], y[0, 39, 0, 0] = float("nan"), float("inf"), -float("inf")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    lens = torch.tensor([40], dtype=torch.int32, device="cuda")
    C.conduit_fp8_append(cache.kv, C.Seqs([0, 40], lens, 48), x.cuda(), y.cuda(), status=status)
    assert C.conduit_read_status(status) == C.ERR_NONFINITE
    for g, (k, v) in enumerate(cache.plain[0][0]):
        k.append(0, x[0, :, g].float().numpy())
        v.append(0, y[0, :, g].float().numpy())
    got, want = cache.kv.pool.cpu().numpy(), cache.put()
    # a NaN's sign is not specified
    nan = (got & 0x7F == 0x7F) & (want & 0x7F == 0x7F)
    assert np.array_equal(np.where(nan, 0, got), np.where(nan, 0, want))
    batch = C.Batch([0, 40], [0, 40], [0, 1], [0, 1])
    dst = C.KvCache(torch.zeros((1, 2, 40, 128), device="cuda"), torch.zeros((1, 2, 40, 128), device="cuda"), 2)
    C.conduit_fp8_read(cache.kv, batch, dst)
    assert torch.equal(torch.isnan(dst.k[0].cpu()).nonzero(), torch.tensor([[0, 3, 5], [1, 17, 9]]))
    assert torch.equal(torch.isnan(dst.v[0].cpu()).nonzero(), torch.tensor([[0, 39, 0]]))


def test_rows_out_of_range_are_left_out(C):
    """Positions outside of the table, pages outside of the pool, slots past the context: flagged and not written, the
    other rows of the block are."""
    d, L = 128, 2
    cache = Cache(C, 3, L, 2, 1, d, 16, 3, 48)
    table = cache.table.copy()
    table[1, 1] = 10 ** 6
    cache.kv = C.Fp8Kv(cache.kv.pool, 2, d, 16, torch.from_numpy(table))
    rope = C.Rope(C.rope_table(100.0, d, 50), [0] * (d // 2))
    rows, total = (20, 30, 9), (20, 30, 53)
    T = sum(rows)
    x = torch.randn((L, T, 4, d), generator=torch.Generator().manual_seed(4)).cuda()
    pos = (torch.arange(T, dtype=torch.int32) % 50)[None]
    pos[0, 4], pos[0, 25] = -1, 50
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    lens = torch.tensor(total, dtype=torch.int32, device="cuda")
    q_out = torch.full((L, T, 2, d), 9.0, device="cuda")
    C.conduit_fp8_append(cache.kv, C.Seqs(np.concatenate([[0], np.cumsum(rows)]), lens, 48), x[:, :, :1], x[:, :, 1:2], rope,
                         pos.cuda(), x[:, :, 2:], q_out, status=status)
    assert C.conduit_read_status(status) == C.ERR_INDEX
    ok = np.ones(T, dtype=bool)
    ok[[4, 25]] = False
    ok[20 + 16:50] = False     # the second request's second page does not exist
    ok[50 + 4:] = False        # slots 48 .. 52
    xf = x.float().cpu().numpy()
    shown = np.clip(pos.numpy(), 0, 49)
    at = 0
    for r, n in enumerate(rows):
        for l in range(L):
            part = slice(at, at + n)
            turned = F.rotate32(xf[l, part, :1], shown[:, part], rope.table.cpu().numpy(), [0] * (d // 2))
            k, v = cache.plain[l][r][0]
            if r == 2:  # slots 44 .. 47 of a block whose earlier tokens are the pool's pattern
                continue
            k.append(total[r] - n, turned[:, 0], ok[part])
            v.append(total[r] - n, xf[l, part, 1], ok[part])
        at += n
    got, want = cache.kv.pool.cpu().numpy(), cache.put()
    pages = np.setdiff1d(np.arange(got.shape[1]), cache.table[2])
    assert np.array_equal(got[:, pages], want[:, pages])
    untouched = cache.table[2, :2]
    assert (got[:, untouched] == 0xA5).all()
    assert np.array_equal((q_out != 9.0).any(-1).any(-1).all(0).cpu().numpy(), ok)


def test_a_block_that_begins_anew_forgets_its_scale(C):
    """A context that is cut at a block's start and filled again; one that is cut inside of a block keeps the larger scale."""
    cache = Cache(C, 5, 1, 1, 1, 64, 16, 1, 32)
    k, v = cache.plain[0][0][0]
    lens = torch.zeros(1, dtype=torch.int32, device="cuda")
    gen = torch.Generator().manual_seed(1)
    for begin, n, size in ((0, 32, 100.0), (16, 5, 1.0), (18, 3, 0.01), (0, 1, 0.5)):
        x = size * torch.randn((1, n, 1, 64), generator=gen)
        lens.fill_(begin + n)
        C.conduit_fp8_append(cache.kv, C.Seqs([0, n], lens, 32), x.cuda(), 2 * x.cuda())
        k.append(begin, x[0, :, 0].numpy())
        v.append(begin, 2 * x[0, :, 0].numpy())
        assert np.array_equal(cache.kv.pool.cpu().numpy(), cache.put()), (begin, n)


def test_append_is_captured_and_replayed(C):
    """One token a step from a graph, with lengths that grow on the device."""
    R, d = 3, 128
    cache = Cache(C, 6, 1, 4, 2, d, 16, R, 64)
    lens = torch.tensor([5, 0, 30], dtype=torch.int32, device="cuda")
    rows = torch.zeros((1, R, 4, d), dtype=BF, device="cuda")
    k, v = rows[:, :, :2], rows[:, :, 2:]
    gen = torch.Generator(device="cuda").manual_seed(3)
    seqs = C.Seqs(list(range(R + 1)), lens, 64)
    first = torch.randn((1, 35, 4, d), generator=gen, device="cuda").to(BF)
    C.conduit_fp8_append(cache.kv, C.Seqs([0, 5, 5, 35], lens, 64), first[:, :, :2], first[:, :, 2:])
    f = first.float().cpu().numpy()
    for g in range(2):
        for r, part in ((0, slice(0, 5)), (2, slice(5, 35))):
            cache.plain[0][r][g][0].append(0, f[0, part, g])
            cache.plain[0][r][g][1].append(0, f[0, part, 2 + g])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            lens.add_(1)
            C.conduit_fp8_append(cache.kv, seqs, k, v)
    torch.cuda.synchronize()
    at = [5, 0, 30]
    for step in range(20):
        rows.copy_(torch.randn(rows.shape, generator=gen, device="cuda") * 1.3 ** step)
        graph.replay()
        f = rows.float().cpu().numpy()
        for r in range(R):
            for g in range(2):
                cache.plain[0][r][g][0].append(at[r], f[0, r:r + 1, g])
                cache.plain[0][r][g][1].append(at[r], f[0, r:r + 1, 2 + g])
            at[r] += 1
    assert np.array_equal(cache.kv.pool.cpu().numpy(), cache.put())


def test_lengths_that_no_context_has(C):
    """Lengths below the call's rows, negative ones and the ends of 32 bits: flagged, nothing written."""
    cache = Cache(C, 7, 1, 2, 1, 64, 16, 2, 32)
    x = torch.randn((1, 6, 4, 64), generator=torch.Generator().manual_seed(4)).cuda()
    before = cache.kv.pool.clone()
    for lens in ((0, 0), (-1, -2 ** 31), (2 ** 31 - 1, -2 ** 31 + 2), (36, 2 ** 31 - 1)):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        q_out = torch.full((1, 6, 2, 64), 9.0, device="cuda")
        seqs = C.Seqs([0, 3, 6], torch.tensor(lens, dtype=torch.int32, device="cuda"), 32)
        C.conduit_fp8_append(cache.kv, seqs, x[:, :, :1], x[:, :, 1:2], q=x[:, :, 2:], q_out=q_out, status=status)
        assert C.conduit_read_status(status) == C.ERR_INDEX
        assert torch.equal(cache.kv.pool, before) and (q_out == 9.0).all()
