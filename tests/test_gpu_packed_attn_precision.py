"""Attention over the 4-bit cache where few bits would show, against 64-bit softmax attention.

Keys and values are constant over each group of 32 dims, so that the cache holds them exactly
and only the attention's own roundings are left.
"""

import numpy as np
import pytest
import torch

from tests import cache_reference as R

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module")
def C():
    from paper_2609_05821_gb300 import _build
    _build.build()
    from paper_2609_05821_gb300 import conduit
    return conduit


def _flat_cache(C, k, v, hq, ps=16):
    """A cache of one layer and request with the rows k, v [N, Hkv, d]."""
    n, hkv, d = k.shape
    table = torch.arange(-(-n // ps), dtype=torch.int32)[None]
    kv = C.PackedKv.empty(1, table.numel(), hq, hkv, d, ps, table)
    seqs = C.Seqs([0, n], torch.tensor([n], dtype=torch.int32, device="cuda"), n)
    dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).float().cuda()[None]
    C.conduit_packed_append(kv, seqs, dev(k), dev(v))
    return kv


@pytest.mark.parametrize("below", [20.4, 26.3])
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("n,rows", [(700, 1), (9000, 1), (700, 40), (2500, 40)])
def test_weights_far_below_the_largest(C, d, n, rows, below):
    """One key in 32 has the largest logit and the value 0; the others weigh 2^-below of it, and all of
    the output comes from them.

    Weights may be off by 2^-11 of themselves or by 2^-32 of the row's largest one: N keys beside N / 32
    largest put the output off by 32 x 2^-32 max|V|. Logits are off by d 2^-23 of their size, the bf16
    output by 2^-8."""
    hkv, G = 1, 7
    k, v = np.zeros((n, hkv, d)), np.ones((n, hkv, d))
    k[::32], v[::32] = 1.0, 0.0
    kv = _flat_cache(C, k, v, hkv * G)
    scale = float(np.float32(below * np.log(2) / d))
    q = torch.ones((1, rows, hkv * G, d), dtype=BF, device="cuda")
    seqs = C.Seqs([0, rows], torch.tensor([n], dtype=torch.int32, device="cuda"), n)
    lse = torch.zeros((1, hkv * G, rows), device="cuda")
    out = C.conduit_packed_attn(kv, seqs, q, scale=scale, lse=lse)
    seen = np.arange(n - rows + 1, n + 1)
    want, wl, A, _ = R.attend(q[0].double().cpu().numpy(), k, v, seen, scale)
    e = d * 2.0 ** -23 * A[..., None]
    tol = (np.expm1(2 * e) + 2.0 ** -11 + 2.0 ** -8) * want + 32 * 2.0 ** -32
    got = out[0].double().cpu().numpy()
    assert np.all(np.abs(got - want) <= tol), float(np.max(np.abs(got - want) / want))
    # sums count n terms in fp32
    gl = lse[0].double().cpu().numpy()
    assert np.all(np.abs(gl - wl) <= e[..., 0].T + 2.0 ** -22 * np.abs(wl) + n * 2.0 ** -24 + 2.0 ** -21)


def _between_halves(rng, n, hkv, d):
    """Keys that the cache holds exactly, almost all of them half way between two fp16 numbers, on the
    same side of the one they round to: group scale 2^-11, mid 1, codes 1 and 5."""
    c = rng.choice([1, 5], size=(n, hkv, d // 32, 32))
    c[..., 0], c[..., 1] = -8, 7
    return (1 + c * 2.0 ** -11).reshape(n, hkv, d)


@pytest.mark.parametrize("d", [64, 96, 128])
def test_rows_that_see_few_keys_have_exact_logits(C, d):
    """Many rows, in a call whose max_len is long: rows that see less than 2,048 keys carry fp32 rounding
    only in their log-sum-exp, whatever max_len and the other rows. A key in one fp16 number
    would put a logit off by 0.9 x 2^-11 of its size here."""
    rng = np.random.default_rng(d)
    hkv, G, ps = 2, 7, 16
    lens, rows = (37, 2047, 2600, 3000, 130), (37, 40, 64, 40, 12)
    T, most = sum(rows), 4096
    need = [-(-n // ps) for n in lens]
    first = np.concatenate([[0], np.cumsum(need)])
    table = torch.zeros((len(lens), most // ps), dtype=torch.int32)
    for r, n in enumerate(need):
        table[r, :n] = torch.arange(first[r], first[r] + n)
    kv = C.PackedKv.empty(1, int(first[-1]), hkv * G, hkv, d, ps, table)
    K = [_between_halves(rng, n, hkv, d) for n in lens]
    V = [rng.choice([-1.0, 1.0, 2.0], size=(n, hkv, d // 32, 1)).repeat(32, -1).reshape(n, hkv, d) for n in lens]
    dev_lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    dev = lambda x: torch.from_numpy(np.concatenate(x)).float().cuda()[None]
    C.conduit_packed_append(kv, C.Seqs(np.concatenate([[0], np.cumsum(lens)]), dev_lens, most), dev(K), dev(V))
    limits = np.concatenate([np.arange(1, 38), np.full(40, 2047), rng.integers(0, 2601, 64), rng.integers(2048, 3001, 40),
                             np.arange(119, 131)])
    limits[80:83] = 0, 1, 2600
    q = torch.ones((1, T, hkv * G, d), dtype=BF, device="cuda")
    seqs = C.Seqs(np.concatenate([[0], np.cumsum(rows)]), dev_lens, most)
    lse = torch.zeros((1, hkv * G, T), device="cuda")
    scale = float(np.float32(10 / d))
    out = C.conduit_packed_attn(kv, seqs, q, scale=scale, lse=lse,
                                limits=torch.from_numpy(limits.astype(np.int32)).cuda())
    t = 0
    for r, (n, c) in enumerate(zip(lens, rows)):
        seen = limits[t:t + c]
        wo, wl, A, big = R.attend(q[0, t:t + c].double().cpu().numpy(), K[r], V[r], seen, scale)
        gl, got = lse[0, :, t:t + c].double().cpu().numpy(), out[0, t:t + c].double().cpu().numpy()
        assert np.array_equal(np.isneginf(gl), np.isneginf(wl))
        few = np.broadcast_to(seen < 2048, gl.shape)
        e = (d * 2.0 ** -23 + np.where(few, 0.0, 2.0 ** -11)) * A.T
        room = e + 2.0 ** -22 * np.abs(wl) + n * 2.0 ** -24 + 2.0 ** -21
        fin = np.isfinite(wl)
        assert np.all(np.abs(gl[fin] - wl[fin]) <= room[fin]), (r, float(np.max(np.abs(gl[fin] - wl[fin]))))
        tol = ((np.expm1(2 * e.T) + 2.0 ** -10 + (n + 16) * 2.0 ** -24) * big)[..., None] + 2.0 ** -8 * np.abs(wo)
        assert np.all(np.abs(got - wo) <= tol), r
        t += c


def test_context_of_two_thousand_million_keys(C):
    """The longest context: all keys alike, values 0 but for the last 3,000 pages, which are 1. The output is their
    share. Sums of a lane count up to 2^17 equal weights one by one: at most 2^17 x 2^-24 off."""
    d, ps, n, last = 64, 1024, 2 ** 31 - 2 ** 20, 3000
    table = torch.zeros((1, n // ps), dtype=torch.int32)
    table[0, -last:] = 1
    kv = C.PackedKv.empty(1, 2, 1, 1, d, ps, table)
    fill = C.PackedKv(kv.pool, 1, d, ps, torch.arange(2, dtype=torch.int32)[None])
    k = torch.zeros((1, 2 * ps, 1, d), device="cuda")
    v = torch.cat([torch.zeros_like(k[:, :ps]), torch.ones_like(k[:, ps:])], 1)
    both = torch.tensor([2 * ps], dtype=torch.int32, device="cuda")
    C.conduit_packed_append(fill, C.Seqs([0, 2 * ps], both, 2 * ps), k, v)
    seqs = C.Seqs([0, 1], torch.tensor([n], dtype=torch.int32, device="cuda"), n)
    lse, status = torch.zeros((1, 1, 1), device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    out = C.conduit_packed_attn(kv, seqs, torch.ones((1, 1, 1, d), dtype=BF, device="cuda"), lse=lse, status=status)
    assert C.conduit_read_status(status) == C.OK
    share = last * ps / n
    assert torch.all((out.double() - share).abs() <= (2 * 2.0 ** -7 + 2.0 ** -8) * share)
    assert abs(float(lse[0, 0, 0]) - np.log(n)) <= 2.0 ** -7 + 2.0 ** -19
