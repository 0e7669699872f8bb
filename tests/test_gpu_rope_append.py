"""Rotary positions and the append to paged and 4-bit caches against plain 64-bit forms.

Tolerances. A rotated element is two products and a sum in fp32: at most
3 x 2^-24 (|x1| + |x2|) off, then one rounding to the row's type: it lies between the
roundings of the two ends of that interval. Values and codes are moved or packed by defined roundings and
have to be equal.
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


def _draw(seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *shape, dtype=torch.float32: torch.randn(shape, generator=gen, device="cuda").to(dtype)


def _close(got, x, want, dtype, half, layout):
    y = got.double()
    pair = x.double().abs()
    # |x1| + |x2| of each pair, at both of its dims; passing dims have no error
    reach = torch.zeros_like(pair)
    p = torch.arange(half, device=x.device)
    i1, i2 = (p, p + half) if layout == "halves" else (2 * p, 2 * p + 1)
    reach[..., i1] = reach[..., i2] = pair[..., i1] + pair[..., i2]
    room = 3 * 2.0 ** -24 * reach
    lo, hi = ((want + e).to(dtype).double() for e in (-room, room))
    assert torch.all((lo <= y) & (y <= hi)), float(torch.maximum(lo - y, y - hi).max())


# (dtype, L, T, H, d, rot, axis pattern, layout, strided)
ROPE = [
    (torch.bfloat16, 1, 1, 1, 128, 128, "t", "halves", False),
    (torch.bfloat16, 1, 37, 28, 128, 128, "thw", "halves", True),
    (torch.bfloat16, 2, 5, 3, 64, 32, "hw", "pairs", False),
    (torch.bfloat16, 3, 7, 2, 72, 36, "hw", "halves", False),    # 18 pairs: no whole chunks
    (torch.bfloat16, 1, 513, 5, 96, 96, "interleaved", "halves", True),
    (torch.float32, 1, 129, 16, 80, 40, "hw", "pairs", False),
    (torch.float32, 2, 3, 4, 256, 256, "thw", "halves", True),
    (torch.float32, 1, 9, 2, 6, 2, "t", "pairs", False),
    (torch.bfloat16, 1, 11, 2, 16, 14, "t", "halves", False),
    (torch.bfloat16, 1, 1025, 4, 128, 64, "interleaved", "pairs", False),
]


def _axis(pattern, half):
    if pattern == "t":
        return [0] * half
    if pattern == "hw":
        return [0] * (half // 2) + [1] * (half - half // 2)
    if pattern == "thw":
        a = half // 4
        return [0] * (half - 2 * (3 * half // 8)) + [1] * (3 * half // 8) + [2] * (3 * half // 8) if a else [0] * half
    return [i % 3 for i in range(half)]


@pytest.mark.parametrize("dtype,L,T,H,d,rot,pattern,layout,strided", ROPE)
@pytest.mark.parametrize("inverse", [False, True])
def test_rope(C, dtype, L, T, H, d, rot, pattern, layout, strided, inverse):
    draw = _draw(T + d)
    axis = _axis(pattern, rot // 2)
    A = max(axis) + 1
    table = C.rope_table(10000.0, rot, 5000)
    pos = torch.randint(0, 5000, (A, T), dtype=torch.int32, device="cuda")
    rope = C.Rope(table, axis, layout)
    x = draw(L, T, H + 3, d, dtype=dtype)[:, :, 1:1 + H] if strided else draw(L, T, H, d, dtype=dtype)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = C.conduit_rope(rope, x, pos, inverse=inverse, status=status)
    want = R.rotate(x, pos, table, axis, layout, inverse)
    _close(out, x, want, dtype, rot // 2, layout)
    assert C.conduit_read_status(status) == C.OK
    # in place, and on another stream
    y = x.clone() if not strided else x
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    C.conduit_rope(rope, y, pos, out=y, inverse=inverse, stream=side)
    side.synchronize()
    assert torch.equal(y, out)


def test_rope_gradient(C):
    """The inverse is the gradient: against differences of <rotation(x), w>, in fp32 on well scaled inputs.

    The function is linear, so a central difference of step 2^-3 has only rounding: n terms of size about 1 in
    64 bits on rotated rows that are 3 x 2^-24 (|x1|+|x2|) off, over a step of 2^-2."""
    T, H, d, rot = 5, 3, 32, 24
    axis = _axis("thw", rot // 2)
    table = C.rope_table(100.0, rot, 50)
    pos = torch.randint(0, 50, (max(axis) + 1, T), dtype=torch.int32, device="cuda")
    for layout in ("halves", "pairs"):
        rope = C.Rope(table, axis, layout)
        draw = _draw(3)
        x, w = draw(T, H, d), draw(T, H, d)
        grad = C.conduit_rope(rope, w, pos, inverse=True)
        for i in (0, 5, 11, 12, 13, 23, 24, 31):
            e = torch.zeros_like(x)
            e[:, :, i] = 2.0 ** -3
            f = lambda z: (C.conduit_rope(rope, z, pos).double() * w.double()).sum(-1)
            diff = (f(x + e) - f(x - e)) / 2.0 ** -2
            room = 4 * (6 * 2.0 ** -24 * (x.abs().amax() + 1) * w.double().abs().sum(-1)) * 4
            assert torch.all((diff - grad[:, :, i].double()).abs() <= room)


def test_rope_position_out_of_range(C):
    table = C.rope_table(100.0, 64, 10)
    rope = C.Rope(table, [0, 1] * 16)
    x = _draw(0)(4, 2, 64, dtype=torch.bfloat16)
    pos = torch.tensor([[0, 10, 9, 3], [1, 1, -1, 9]], dtype=torch.int32, device="cuda")
    out = torch.full_like(x, 7.0)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    C.conduit_rope(rope, x, pos, out=out, status=status)
    assert C.conduit_read_status(status) == C.ERR_INDEX
    good = pos.clamp(0, 9)
    want = C.conduit_rope(rope, x, good)
    assert torch.equal(out[[0, 3]], want[[0, 3]]) and torch.all(out[[1, 2]] == 7.0)


def test_rope_no_rows(C):
    rope = C.Rope(C.rope_table(100.0, 64, 10), [0] * 32)
    x = torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    assert C.conduit_rope(rope, x, torch.empty((1, 0), dtype=torch.int32, device="cuda")).shape == (0, 2, 64)


def _table_of(lens, ps, spare=2, seed=0):
    """A page table with shuffled pages, and the number of pages."""
    need = [-(-n // ps) for n in lens]
    order = np.random.default_rng(seed).permutation(sum(need) + spare)
    table = np.zeros((len(lens), max(max(need), 1)), dtype=np.int32)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n]
        at += n
    return table, sum(need) + spare


# (dtype, L, hq, hkv, d, rot, page, cached tokens, rows of the call, strided)
APPEND = [
    (torch.bfloat16, 1, 7, 1, 128, 128, 16, (1,), (1,), True),
    (torch.bfloat16, 2, 28, 4, 128, 128, 16, (40, 16, 17, 300), (1, 16, 0, 47), True),
    (torch.bfloat16, 1, 4, 2, 64, 32, 8, (100, 9), (100, 2), False),
    (torch.bfloat16, 1, 2, 2, 96, 36, 32, (33,), (33,), False),
    (torch.float32, 2, 6, 2, 96, 96, 64, (70, 1), (65, 1), True),
    (torch.float32, 1, 3, 3, 32, 0, 16, (5, 60), (5, 3), False),
]


def _append_setup(C, dtype, L, hq, hkv, d, rot, lens, rows, strided):
    draw = _draw(d + len(lens))
    T = sum(rows)
    x = draw(L, T, hq + 2 * hkv, d, dtype=dtype)
    q, k, v = x[:, :, :hq], x[:, :, hq:hq + hkv], x[:, :, hq + hkv:]
    if not strided:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    seqs = C.Seqs(np.concatenate([[0], np.cumsum(rows)]), torch.tensor(lens, dtype=torch.int32, device="cuda"), max(lens))
    if not rot:
        return q, k, v, seqs, None, None, None, None
    axis = _axis("thw", rot // 2)
    table = C.rope_table(10000.0, rot, 700)
    pos = torch.randint(0, 700, (max(axis) + 1, T), dtype=torch.int32, device="cuda")
    return q, k, v, seqs, C.Rope(table, axis), pos, table, axis


@pytest.mark.parametrize("dtype,L,hq,hkv,d,rot,ps,lens,rows,strided", APPEND)
def test_kv_append(C, dtype, L, hq, hkv, d, rot, ps, lens, rows, strided):
    q, k, v, seqs, rope, pos, table, axis = _append_setup(C, dtype, L, hq, hkv, d, rot, lens, rows, strided)
    pages, P = _table_of(lens, ps)
    pool = [torch.full((L, P, hkv, ps, d), 3.0, dtype=dtype, device="cuda") for _ in range(2)]
    kv = C.KvCache(*pool, hq, ps, torch.from_numpy(pages))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    q_out = C.conduit_kv_append(kv, seqs, k, v, rope, pos, q, status=status)
    assert C.conduit_read_status(status) == C.OK
    turn = (lambda x: R.rotate(x, pos, table, axis)) if rot else (lambda x: x.double())
    _close(q_out, q, turn(q), dtype, rot // 2, "halves")
    want_k = turn(k)
    written = torch.zeros((P, ps), dtype=torch.bool)
    t = 0
    for r, (n, c) in enumerate(zip(lens, rows)):
        for i in range(c):
            j = n - c + i
            page, row = int(pages[r, j // ps]), j % ps
            assert torch.equal(kv.v[:, page, :, row], v[:, t])
            _close(kv.k[:, page, :, row], k[:, t], want_k[:, t], dtype, rot // 2, "halves")
            written[page, row] = True
            t += 1
    for p in pool:  # nothing else was touched
        assert torch.all(p.permute(1, 3, 0, 2, 4)[~written.cuda()] == 3.0)


@pytest.mark.parametrize("dtype,L,hq,hkv,d,rot,ps,lens,rows,strided", [c for c in APPEND if c[4] % 32 == 0])
def test_packed_append_and_read(C, dtype, L, hq, hkv, d, rot, ps, lens, rows, strided):
    q, k, v, seqs, rope, pos, table, axis = _append_setup(C, dtype, L, hq, hkv, d, rot, lens, rows, strided)
    pages, P = _table_of(lens, ps)
    kv = C.PackedKv.empty(L, P, hq, hkv, d, ps, torch.from_numpy(pages))
    kv.pool.fill_(0xA5)
    before = kv.pool.clone()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    q_out = C.conduit_packed_append(kv, seqs, k, v, rope, pos, q, status=status)
    assert C.conduit_read_status(status) == C.OK
    turn = (lambda x: R.rotate(x, pos, table, axis)) if rot else (lambda x: x.double())
    _close(q_out, q, turn(q), dtype, rot // 2, "halves")
    # the rotated key in fp32, operation by operation, is what is packed
    if rot:
        cs = table[pos.long()[torch.as_tensor(axis, device="cuda")].T, torch.arange(rot // 2, device="cuda")][:, None]
        x, h = k.float(), rot // 2
        kk = x.clone()
        kk[..., :h] = x[..., :h] * cs[..., 0] - x[..., h:rot] * cs[..., 1]
        kk[..., h:rot] = x[..., h:rot] * cs[..., 0] + x[..., :h] * cs[..., 1]
    else:
        kk = k.float()
    ref = [R.pack_groups(y.cpu().numpy()) for y in (kk, v.float())]  # [L, T, Hkv, ...]
    want = before.cpu().numpy().copy()
    G, half = d // 32, ps * d // 2
    t = 0
    for r, (n, c) in enumerate(zip(lens, rows)):
        for i in range(c):
            j = n - c + i
            page, row = int(pages[r, j // ps]), j % ps
            for l in range(L):
                for g in range(hkv):
                    rec = R.page_record(*[a[l, t, g][None] for part in ref for a in part])
                    w = want[l, page, g]
                    w[row * d // 2:(row + 1) * d // 2] = rec[:d // 2]
                    w[half + row * d // 2:half + (row + 1) * d // 2] = rec[d // 2:d]
                    at = 2 * half + row * 4 * G
                    w[at:at + 4 * G] = rec[d:d + 4 * G]
                    at += ps * 4 * G
                    w[at:at + 4 * G] = rec[d + 4 * G:]
            t += 1
    assert np.array_equal(kv.pool.cpu().numpy(), want)
    # a packed value is half a step off at most, and the roundings of s and m
    for part, x in zip(ref, (kk, v.float())):
        y = R.values(*part)
        s, m = (np.repeat(p.astype(np.float64)[..., 0], 32, axis=-1) for p in part[1:])
        room = s * (0.5 + 2.0 ** -20) + 2.0 ** -11 * (np.abs(m) + 16 * s) + 2.0 ** -24
        assert np.all(np.abs(y - x.cpu().double().numpy()) <= room)
    # back into a plain cache: contiguous from token `first`, and paged from the start
    R_ = len(lens)
    some = [r for r in range(R_) if rows[r]]
    if len(some) == R_:
        off = np.concatenate([[0], np.cumsum(rows)]).tolist()
        batch = C.Batch(off, off, list(range(R_ + 1)), list(range(R_ + 1)))
        first = torch.tensor([n - c for n, c in zip(lens, rows)], dtype=torch.int32, device="cuda")
        wk, wv = (torch.from_numpy(R.values(*part)).transpose(1, 2).to(dtype) for part in ref)  # [L, Hkv, T, d]
        dst = C.KvCache(torch.zeros((L, hkv, sum(rows), d), dtype=dtype, device="cuda"),
                        torch.zeros((L, hkv, sum(rows), d), dtype=dtype, device="cuda"), hq)
        C.conduit_packed_read(kv, batch, dst, first=first, status=status)
        assert C.conduit_read_status(status) == C.OK
        assert torch.equal(dst.k.cpu(), wk) and torch.equal(dst.v.cpu(), wv)
        if rows == lens:
            need = [-(-n // 16) for n in lens]
            tab = torch.zeros((R_, max(need)), dtype=torch.int32)
            at = 0
            for r, n in enumerate(need):
                tab[r, :n] = torch.arange(at, at + n)
                at += n
            paged = C.KvCache(torch.zeros((L, at, hkv, 16, d), dtype=dtype, device="cuda"),
                              torch.zeros((L, at, hkv, 16, d), dtype=dtype, device="cuda"), hq, 16, tab)
            C.conduit_packed_read(kv, batch, paged, status=status)
            assert C.conduit_read_status(status) == C.OK
            for r, n in enumerate(lens):
                for which, want_ in ((paged.k, wk), (paged.v, wv)):
                    got = which[:, tab[r, :need[r]].long().cuda()].transpose(1, 2).flatten(2, 3)[:, :, :n]
                    assert torch.equal(got.cpu(), want_[:, :, off[r]:off[r] + n])


def test_packed_append_edge_values(C):
    """Constant groups, huge values, infinities and NaN: what they stand for, and the flag."""
    d, ps = 64, 8
    x = torch.zeros((1, 5, 1, d), device="cuda")
    x[0, 0] = 2.5                       # s = 0: the group is its mid
    x[0, 1, 0, :32] = 1e30              # clipped
    x[0, 1, 0, 32:] = torch.linspace(-1e-7, 1e-7, 32, device="cuda")
    x[0, 2, 0, 3] = float("inf")
    x[0, 3, 0, 40] = float("nan")
    x[0, 4] = torch.linspace(-61440, 61440, d, device="cuda")
    table = torch.zeros((1, 1), dtype=torch.int32)
    kv = C.PackedKv.empty(1, 1, 1, 1, d, ps, table)
    lens = torch.tensor([2], dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    C.conduit_packed_append(kv, C.Seqs([0, 2], lens, 5), x[:, :2], x[:, :2], status=status)
    assert C.conduit_read_status(status) == C.OK
    lens.fill_(5)
    C.conduit_packed_append(kv, C.Seqs([0, 3], lens, 5), x[:, 2:], x[:, 2:], status=status)
    assert C.conduit_read_status(status) == C.ERR_NONFINITE
    batch = C.Batch([0, 5], [0, 5], [0, 1], [0, 1])
    dst = C.KvCache(torch.zeros((1, 1, 5, d), device="cuda"), torch.zeros((1, 1, 5, d), device="cuda"), 1)
    C.conduit_packed_read(kv, batch, dst)
    want = torch.from_numpy(R.values(*R.pack_groups(x.cpu().numpy()))).float()[0, :, 0]
    for got in (dst.k, dst.v):
        got = got[0, 0].cpu()
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(), want.nan_to_num())
    assert torch.all(want[0] == 2.5) and want[3, :32].eq(0).all() and want[3, 32:].isnan().all()
    assert want[2, 3] >= 60000 and torch.isfinite(want[4]).all()


@pytest.mark.parametrize("packed", [False, True])
def test_append_out_of_range(C, packed):
    """Tokens, pages and positions outside of their arrays: the rows are left out, flagged, and nothing else is written."""
    d, ps, P = 64, 8, 3
    pages = torch.tensor([[0, 1], [2, 7], [-1, 0]], dtype=torch.int32)  # pages 7 and -1 do not exist
    x = _draw(1)(1, 6, 3, d, dtype=torch.bfloat16)
    q, k, v = x[:, :, :1], x[:, :, 1:2], x[:, :, 2:]
    # request 0: tokens 15, 16 (past the table); request 1: 7, 8 (page 7); request 2: 0, 1 (page -1)
    seqs = C.Seqs([0, 2, 4, 6], torch.tensor([17, 9, 2], dtype=torch.int32, device="cuda"), 17)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    q_out = torch.full_like(q, 9.0)
    if packed:
        kv = C.PackedKv.empty(1, P, 1, 1, d, ps, pages)
        kv.pool.zero_()
        C.conduit_packed_append(kv, seqs, k, v, q=q, q_out=q_out, status=status)
        used = kv.pool[0, :, 0, :ps * d // 2].view(P, ps, -1).ne(0).any(-1)
    else:
        kv = C.KvCache(torch.zeros((1, P, 1, ps, d), dtype=torch.bfloat16, device="cuda"),
                       torch.zeros((1, P, 1, ps, d), dtype=torch.bfloat16, device="cuda"), 1, ps, pages)
        C.conduit_kv_append(kv, seqs, k, v, q=q, q_out=q_out, status=status)
        used = kv.k[0, :, 0].ne(0).any(-1)
    assert C.conduit_read_status(status) == C.ERR_INDEX
    assert used.nonzero().tolist() == [[1, 7], [2, 7]]
    assert torch.equal(q_out[0, [0, 2]], q[0, [0, 2]]) and torch.all(q_out[0, [1, 3, 4, 5]] == 9.0)


def test_append_past_four_gigabytes(C):
    """Pages whose offset does not fit in 32 bits."""
    d, ps, hkv = 128, 16, 4
    for packed in (False, True):
        nbytes = hkv * (ps * 160 if packed else ps * d * 2)
        P = (1 << 32) // nbytes + 1000
        pages = torch.tensor([[P - 1, 0]], dtype=torch.int32)
        x = _draw(2)(1, 20, 3 * hkv, d, dtype=torch.bfloat16)
        q, k, v = x[:, :, :hkv], x[:, :, hkv:2 * hkv], x[:, :, 2 * hkv:]
        seqs = C.Seqs([0, 20], torch.tensor([20], dtype=torch.int32, device="cuda"), 20)
        batch = C.Batch([0, 20], [0, 20], [0, 1], [0, 1])
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        if packed:
            kv = C.PackedKv.empty(1, P, hkv, hkv, d, ps, pages)
            C.conduit_packed_append(kv, seqs, k, v, status=status)
            dst = C.KvCache(*[torch.zeros((1, hkv, 20, d), device="cuda") for _ in range(2)], hkv)
            C.conduit_packed_read(kv, batch, dst, status=status)
            got_k, got_v = dst.k.transpose(1, 2).cpu().numpy(), dst.v.transpose(1, 2).cpu().numpy()
            for got, src in ((got_k, k), (got_v, v)):
                assert np.array_equal(got, R.values(*R.pack_groups(src.float().cpu().numpy())))
        else:
            kv = C.KvCache(*[torch.empty((1, P, hkv, ps, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)],
                           hkv, ps, pages)
            C.conduit_kv_append(kv, seqs, k, v, status=status)
            for pool, src in ((kv.k, k), (kv.v, v)):
                assert torch.equal(pool[0, P - 1].transpose(0, 1), src[0, :16])
                assert torch.equal(pool[0, 0, :, :4].transpose(0, 1), src[0, 16:])
        assert C.conduit_read_status(status) == C.OK
        del kv
        torch.cuda.empty_cache()
