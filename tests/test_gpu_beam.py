"""Beam selection and the contexts that follow it, against plain forms.

Selection: the order inside a beam is that of the logits. A beam's log-sum-exp is off by EPS at most (sums of
exponentials that are 2^-22 off, and the rounding of numbers up to 32 x 2^-24), the same for all of its candidates and for
beams of equal rows and sums; so candidates of two unequal beams may change places where their 64-bit scores are within 2 EPS,
and everything else is compared exactly. A score is rounded to fp32 once more.
Reordering moves bytes: everything is compared exactly.
"""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
EPS = 2.0 ** -21


@pytest.fixture(scope="module")
def C():
    from paper_2609_05821_gb300 import _build
    _build.build()
    from paper_2609_05821_gb300 import conduit
    return conduit


def _scores(logits, sums):
    z = logits.double().cpu().numpy()
    with np.errstate(invalid="ignore", divide="ignore"):
        top = z.max(-1, keepdims=True)
        base = np.where(np.isfinite(top), top, 0)
        lse = np.log(np.exp(z - base).sum(-1, keepdims=True)) + base
        s = sums.double().cpu().numpy()[:, None] + (z - lse)
    bad = np.isnan(z).any(-1) | np.isposinf(z).any(-1) | ~(sums.cpu().numpy() < np.inf)
    s[bad] = -np.inf
    return np.where(np.isnan(s), -np.inf, s), bad.any()


def _check_select(C, logits, sums, width, n, status_want=0, **kw):
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    score, parent, token = C.conduit_beam_select(logits, sums, width, n, status=status, **kw)
    want, flagged = _scores(logits, sums)
    assert C.conduit_read_status(status) == (C.ERR_NONFINITE if flagged else C.OK)
    G, V = logits.shape[0] // width, logits.shape[1]
    for g in range(G):
        s = want[g * width:(g + 1) * width].ravel()
        order = np.argsort(-s, kind="stable")[:n]
        best = s[order]
        got_s, got_p, got_t = (x[g].double().cpu().numpy() for x in (score, parent, token))
        for i in range(n):
            if i >= len(order) or best[i] == -np.inf:
                assert got_s[i] == -np.inf and got_p[i] == g * width and got_t[i] == 0, (g, i)
                continue
            assert abs(got_s[i] - best[i]) <= EPS + 2.0 ** -24 * abs(best[i]), (g, i, got_s[i], best[i])
            flat = int((got_p[i] - g * width) * V + got_t[i])
            close = np.unique(np.nonzero(np.abs(s - best[i]) <= 2 * EPS)[0] // V)
            own = g * width + order[i] // V
            if all(torch.equal(logits[g * width + w], logits[own]) and sums[g * width + w] == sums[own] for w in close):
                assert flat == order[i], (g, i, flat, order[i])
            else:
                assert abs(s[flat] - best[i]) <= 2 * EPS
        assert len(set(zip(got_p[got_s > -np.inf], got_t[got_s > -np.inf]))) == (got_s > -np.inf).sum()
    return score, parent, token


# (dtype, groups, width, vocab, n, padding of a row)
SELECT = [
    (F32, 1, 4, 32000, 8, 0),
    (BF, 3, 8, 50021, 16, 3),
    (BF, 2, 1, 1, 1, 0),
    (F32, 2, 3, 2, 6, 1),            # all candidates are chosen
    (F32, 5, 5, 7, 32, 0),
    (BF, 2, 32, 999, 32, 5),
    (F32, 1, 7, 100003, 14, 1),
    (BF, 70, 2, 301, 4, 0),
    (BF, 1, 16, 8, 20, 0),
    (F32, 1, 1, 300000, 32, 0),
]


@pytest.mark.parametrize("dtype,G,width,vocab,n,pad", SELECT)
def test_select(C, dtype, G, width, vocab, n, pad):
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    z = 3 * torch.randn((G * width, vocab + pad), generator=gen, device="cuda")
    z[:, vocab:] = 1e4  # behind the rows
    z = z.to(dtype)
    sums = -5 * torch.rand(G * width, generator=gen, device="cuda")
    _check_select(C, z[:, :vocab], sums, width, n)


def test_select_equal_scores(C):
    """Equal logits, equal beams, sorted rows both ways and zeros of both signs: the lowest index first."""
    for dtype in (F32, BF):
        z = torch.zeros((6, 5000), device="cuda", dtype=dtype)
        z[3:] = torch.tensor([0.0, -0.0], device="cuda", dtype=dtype).repeat(2500)
        sums = torch.tensor([-1.0, -1.0, -1.0, -2.0, -1.5, -1.5], device="cuda")
        score, parent, token = _check_select(C, z, sums, 3, 10)
        assert parent[0].tolist() == [0] * 10 and token[0].tolist() == list(range(10))
        assert parent[1].tolist() == [4] * 10 and token[1].tolist() == list(range(10))
        up = torch.arange(20001, device="cuda", dtype=torch.float32).to(dtype) / 1024
        _check_select(C, torch.stack([up, up.flip(0), up, up]), torch.zeros(4, device="cuda"), 2, 9)


def test_select_left_out(C):
    """Beams of -inf, rows of -inf, few finite logits, NaN and +inf."""
    inf = float("inf")
    z = torch.randn((8, 3000), generator=torch.Generator().manual_seed(1)).cuda()
    sums = torch.tensor([0.0, -inf, -inf, -inf, -1.0, -2.0, -3.0, -inf], device="cuda")
    _check_select(C, z, sums, 4, 8)
    w = z.clone()
    w[0] = -inf
    w[4, 5:] = -inf
    w[5, 7:] = -inf
    w[6, :] = -inf
    _check_select(C, w, sums, 4, 20)          # 12 candidates in the second group, none in the first
    for bad in (float("nan"), inf):
        w = z.clone()
        w[4, 2999] = bad
        _check_select(C, w, sums, 4, 6)
        s = sums.clone()
        s[5] = bad
        _check_select(C, z, s, 4, 6)


def test_select_large_and_small_logits(C):
    z = torch.randn((4, 40000), generator=torch.Generator().manual_seed(3)).cuda()
    for size in (1e-6, 1e30):
        _check_select_scaled = z * size
        score, parent, token = C.conduit_beam_select(_check_select_scaled, torch.zeros(4, device="cuda"), 4, 4)
        want, _ = _scores(_check_select_scaled, torch.zeros(4))
        best = np.sort(want.ravel())[::-1][:4]
        assert np.allclose(score[0].double().cpu().numpy(), best, rtol=2.0 ** -22, atol=EPS)


def test_select_over_its_sums(C):
    """Scores take the place of the sums: the same bits as beside them."""
    g = torch.Generator(device="cuda").manual_seed(8)
    z = 3 * torch.randn((4 * 90, 1003), generator=g, device="cuda")
    sums = -5 * torch.rand(4 * 90, generator=g, device="cuda")
    want = C.conduit_beam_select(z, sums, 4)
    buf = sums.clone()
    got = C.conduit_beam_select(z, buf, 4, score=buf.view(90, 4))
    assert got[0].data_ptr() == buf.data_ptr() and all(torch.equal(a, b) for a, b in zip(want, got))


def test_select_is_captured_and_repeats_bits(C):
    z = torch.randn((16, 70001), generator=torch.Generator().manual_seed(3)).cuda().to(BF)
    sums = torch.zeros(16, device="cuda")
    want = [x.clone() for x in C.conduit_beam_select(z, sums, 8, 16)]
    out = [torch.empty_like(x) for x in want]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            C.conduit_beam_select(z, sums, 8, 16, *out)
    torch.cuda.synchronize()
    for _ in range(5):
        for x in out:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    for a, b in zip(C.conduit_beam_select(z, sums, 8, 16, stream=stream), want):
        stream.synchronize()
        assert torch.equal(a, b)


# ------------------------------------------------------------------ reordering
def _make(C, kind, L, hkv, d, ps, n, per, seed):
    """A cache with random bytes, `home` pages in random order, and a view of what a page holds as rows of bytes."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    P = n * per + 1
    home = torch.randperm(n * per, generator=gen, device="cuda").view(n, per).int()
    table = home.clone()
    if kind in ("bf16", "f32"):
        dt = BF if kind == "bf16" else F32
        k, v = (torch.randn((L, P, hkv, ps, d), generator=gen, device="cuda").to(dt) for _ in range(2))
        kv = C.KvCache(k, v, hkv, ps, table)
        parts = lambda: [x.view(torch.uint8) for x in (kv.k, kv.v)]  # [L, P, hkv, ps, bytes]
        return kv, home, parts, 1
    cls = C.PackedKv if kind == "packed" else C.Fp8Kv
    pool = torch.randint(0, 256, (L, P, hkv, cls.page_bytes(d, ps)), generator=gen, device="cuda", dtype=torch.uint8)
    kv = cls(pool, hkv, d, ps, table)
    if kind == "fp8":
        return kv, home, lambda: [kv.pool.view(L, P, hkv, ps // 16, 32 * d + 16)], 16
    c, p = ps * d // 2, ps * d // 8
    return kv, home, lambda: [kv.pool[..., a:b].unflatten(-1, (ps, -1)) for a, b in
                              ((0, c), (c, 2 * c), (2 * c, 2 * c + p), (2 * c + p, 2 * c + 2 * p))], 1


REORDER = {"bf16": "conduit_kv_reorder", "f32": "conduit_kv_reorder", "packed": "conduit_packed_reorder", "fp8": "conduit_fp8_reorder"}


@pytest.mark.parametrize("kind", list(REORDER))
@pytest.mark.parametrize("L,hkv,d,ps,G,width,lens", [
    (2, 3, 64, 16, 3, 4, (37, 0, 48)),
    (1, 1, 32, 32, 2, 1, (5, 64)),
    (1, 2, 128, 16, 1, 32, (31,)),
    (3, 2, 96, 64, 2, 9, (65, 127)),
    (1, 4, 256, 16, 5, 2, (1, 15, 16, 17, 47)),
])
def test_reorder(C, kind, L, hkv, d, ps, G, width, lens):
    n, per = G * width, 130 // ps + 1
    kv, home, parts, unit = _make(C, kind, L, hkv, d, ps, n, per, 3)
    rng = np.random.default_rng(7)
    home_h = home.cpu().numpy()
    # whole pages are anyone's of the group, the begun one is the beam's own
    table = home_h.copy()
    for b in range(n):
        g = b // width
        for i in range(lens[g] // ps):
            table[b, i] = home_h[g * width + rng.integers(width), i]
    kv.page_table.copy_(torch.from_numpy(table))
    for step in range(3):
        parent = np.concatenate([g * width + (rng.permutation(width) if step == 0 else rng.integers(0, width, width)) for g in range(G)])
        lens_dev = torch.tensor(np.repeat(lens, width), dtype=torch.int32, device="cuda")
        if step == 2:  # beams that are not continued may have any length
            for b in set(range(n)) - set(parent.tolist()):
                lens_dev[b] = int(rng.integers(0, 3))
        before = [x.cpu().numpy().copy() for x in parts()]
        table = kv.page_table.cpu().numpy().copy()
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        getattr(C, REORDER[kind])(kv, torch.from_numpy(parent).int().cuda(), width, home, lens_dev, status=status)
        assert C.conduit_read_status(status) == C.OK
        want_table = table.copy()
        after = [x.cpu().numpy() for x in parts()]
        want = [x.copy() for x in before]
        for b in range(n):
            length = lens[b // width]
            w, rest = divmod(length, ps)
            want_table[b, :w], want_table[b, w:] = table[parent[b], :w], home_h[b, w:]
            if rest and parent[b] != b:
                used = -(-rest // unit)
                for x, y in zip(want, before):
                    x[:, home_h[b, w], :, :used] = y[:, home_h[parent[b], w], :, :used]
        assert np.array_equal(kv.page_table.cpu().numpy(), want_table)
        assert np.array_equal(lens_dev.cpu().numpy(), np.repeat(lens, width))
        for x, y, part in zip(after, want, range(9)):
            if kind == "packed" and part >= 2:  # parameters move 16 bytes at a time: up to the last whole row group
                ok = x == y
                used_rows = {b: lens[b // width] % ps for b in range(n)}
                for b in range(n):
                    w = lens[b // width] // ps
                    if used_rows[b] and parent[b] != b:
                        ok[:, home_h[b, w], :, used_rows[b]:] = True  # rows that no token has
                assert ok.all()
            else:
                assert np.array_equal(x, y), part


def test_reorder_leaves_a_group_that_does_not_fit(C):
    """Parents of another group, of unequal lengths, a begun page that is not the beam's own, lengths and pages out of range."""
    kv, home, parts, _ = _make(C, "fp8", 1, 2, 64, 16, 6, 3, 5)
    good = torch.tensor([1, 1, 0, 4, 5, 3], dtype=torch.int32, device="cuda")

    def run(parent=good, lens=(20,) * 6, table=None, home_now=home):
        kv.page_table.copy_(home if table is None else table)
        pool, lens_dev = kv.pool.clone(), torch.tensor(lens, dtype=torch.int32, device="cuda")
        was, was_len = kv.page_table.clone(), lens_dev.clone()
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        C.conduit_fp8_reorder(kv, parent, 3, home_now, lens_dev, status=status)
        assert C.conduit_read_status(status) == C.ERR_INDEX
        assert torch.equal(kv.page_table[:3], was[:3]) and torch.equal(lens_dev[:3], was_len[:3])
        left = home[:3].flatten().long()
        assert torch.equal(kv.pool[:, left], pool[:, left])
        assert not torch.equal(kv.pool, pool)  # the second group is served

    for bad in (-1, 3, 2 ** 31 - 1, -2 ** 31):
        parent = good.clone()
        parent[2] = bad
        run(parent)
    run(lens=(20, 21, 20, 20, 20, 20))
    run(lens=(-1, -1, -1, 20, 20, 20))
    run(lens=(49, 49, 49, 20, 20, 20))
    table = home.clone()
    table[1, 1] = home[0, 1]
    run(table=table)
    away = home.clone()
    away[2, 1] = 10 ** 6
    run(home_now=away)
    assert parts()[0].shape[1] == 19


def test_reorder_from_the_first_beam_and_captured(C):
    """A prompt in one beam reaches the others; the same call from a graph."""
    kv, home, parts, _ = _make(C, "bf16", 2, 2, 64, 16, 4, 4, 6)
    lens = torch.tensor([37, 0, 0, 0], dtype=torch.int32, device="cuda")
    parent = torch.zeros(4, dtype=torch.int32, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            C.conduit_kv_reorder(kv, parent, 4, home, lens)
    torch.cuda.synchronize()
    k = kv.k.clone()
    graph.replay()
    torch.cuda.synchronize()
    assert lens.tolist() == [37] * 4
    for b in range(4):
        assert kv.page_table[b, :2].tolist() == home[0, :2].tolist() and kv.page_table[b, 2:].tolist() == home[b, 2:].tolist()
        assert torch.equal(kv.k[:, home[b, 2], :, :5], k[:, home[0, 2], :, :5])


def test_a_group_that_is_cut_to_whole_pages(C):
    """After lengths are cut, a reordering of each beam to itself gives every beam its own pages from there on."""
    kv, home, parts, _ = _make(C, "fp8", 1, 1, 32, 16, 3, 4, 9)
    kv.page_table[1:, :3] = home[0, :3]  # beams 1 and 2 share the first one's pages
    lens = torch.full((3,), 16, dtype=torch.int32, device="cuda")
    pool = kv.pool.clone()
    C.conduit_fp8_reorder(kv, torch.arange(3, dtype=torch.int32, device="cuda"), 3, home, lens)
    assert torch.equal(kv.page_table[:, 1:], home[:, 1:]) and torch.equal(kv.page_table[:, 0], home[0, :1].expand(3))
    assert torch.equal(kv.pool, pool) and lens.tolist() == [16] * 3
