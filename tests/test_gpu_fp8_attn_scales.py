"""Attention over the 8-bit cache whose values' scales lie anywhere in their range, against 64 bits.

Tolerances as in test_gpu_fp8_attn.py, and one term more: on the tensor cores a weight is 2^(x + v - reference), x its logit in
log2 units, 2^v its value's scale. x is up to X = A log2(e), v within [-40, 119], and the reference follows x + v, so the two
subtractions round numbers up to 160 + 2 X, 2^-24 of them each, and so does the reference's logarithm in the
log-sum-exp. A weight, and so a sum of weights, is then off by a factor within 1 +- 3 (160 + 2 X) ln 2 2^-24.
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


def _one_head(C, hq, k, v):
    """A cache of one layer, request and KV head over the Blocks k and v."""
    n, d = k.codes.shape
    pool = np.full((1, n // 16, 1, 32 * d + 16), 0xFF, dtype=np.uint8)
    for b in range(n // 16):
        F.put_block(pool[0, b, 0], k, v, b)
    return C.Fp8Kv(torch.from_numpy(pool).cuda(), hq, d, 16, torch.arange(n // 16, dtype=torch.int32)[None])


def _attend(C, kv, n, q, limit):
    T = q.shape[1]
    lse = torch.zeros((1, q.shape[2], T), device="cuda")
    seqs = C.Seqs([0, T], torch.tensor([n], dtype=torch.int32, device="cuda"), n)
    out = C.conduit_fp8_attn(kv, seqs, q, limits=torch.full((T,), limit, dtype=torch.int32, device="cuda"), lse=lse)
    return out, lse


# sizes of the blocks of 16 values, one after another
SIZES = [
    (0.0, 2.0 ** 100),
    (2.0 ** 100, 0.0),
    (0.0, 2.0 ** 126),
    (2.0 ** 126, 0.0),
    (2.0 ** 126, 1.0),
    (1.0, 2.0 ** 126),
    (2.0 ** 75, 2.0 ** -30, 0.0),
    (2.0 ** -30, 2.0 ** 60, 2.0 ** 126, 0.0, 1.0),
    (2.0 ** 126, 2.0 ** 126, 2.0 ** 126, 2.0 ** 126, 2.0 ** 126, 2.0 ** 126, 2.0 ** 126, 2.0 ** 126, 0.0),
]


@pytest.mark.parametrize("n", [96, 2064, 9008])
@pytest.mark.parametrize("dtype,rows", [(BF, 1), (BF, 3), (BF, 40), (BF, 200), (F32, 1), (F32, 3)])
def test_scales_anywhere_in_their_range(C, dtype, rows, n):
    """Zeros and small values beside values of up to 2^127, in every order: each key counts in the denominator. One warp's
    and several warps' blocks, a cluster's and a workspace's chunks, one column tile and two."""
    d = 64 if n == 96 else 128
    rng = np.random.default_rng(n + rows)
    for sizes in SIZES:
        k, v = F.Blocks(n, d), F.Blocks(n, d)
        y = rng.uniform(0.5, 1.75, (n, d)).astype(np.float32)  # one sign: a lost denominator shows whole
        for b in range(n // 16):
            y[16 * b:16 * b + 16] *= np.float32(sizes[b % len(sizes)])
        k.append(0, 0.1 * rng.standard_normal((n, d)).astype(np.float32))
        v.append(0, y)
        kv = _one_head(C, 2, k, v)
        q = torch.randn((1, rows, 2, d), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").to(dtype)
        K, V = k.values(n)[:, None], v.values(n)[:, None]
        for limit in (17, 33, 49, n - 3, n):
            out, lse = _attend(C, kv, n, q, limit)
            few = min(rows, 3)  # of equal rows' worth of checking, the last
            wo, wl, A, big = R.attend(q[0, rows - few:].double().cpu().numpy(), K, V, np.full(few, limit), d ** -0.5)
            e = (d + 4) * 2.0 ** -23 * A + (3 * (160 + 2 * A / np.log(2)) * np.log(2) * 2.0 ** -24 if dtype == BF else 0.0)
            tol = (np.expm1(2 * e) + (limit + 16) * 2.0 ** -23 + (2.0 ** -11 if dtype == BF else 0.0)) * big
            tol = tol[..., None] + (2.0 ** -8 if dtype == BF else 2.0 ** -22) * np.abs(wo)
            got = out[0, rows - few:].double().cpu().numpy()
            assert np.all(np.abs(got - wo) <= tol), (sizes, limit, float(np.max((np.abs(got - wo) - tol) / big[..., None])))
            off = np.abs(lse[0, :, rows - few:].double().cpu().numpy() - wl)
            assert np.all(off <= e.T + 2.0 ** -22 * np.abs(wl) + limit * 2.0 ** -23 + 2.0 ** -21), (sizes, limit, off.max())
        again, lse2 = _attend(C, kv, n, q, n)
        assert torch.equal(again, out) and torch.equal(lse2, lse)


@pytest.mark.parametrize("dtype,d", [(F32, 64), (F32, 128), (F32, 256), (BF, 32), (BF, 160)])
@pytest.mark.parametrize("n", [96, 5008])
def test_large_values_on_the_cuda_cores(C, dtype, d, n):
    """Values of up to 2^127: fp32 sums of weights times values stay in range, in one chunk and in several; and values near the
    least keep their bits."""
    rng = np.random.default_rng(n + d)
    for size in (2.0 ** 126, 2.0 ** 110, 2.0 ** -40):
        k, v = F.Blocks(n, d), F.Blocks(n, d)
        y = (rng.uniform(0.5, 1.75, (n, d)) * size).astype(np.float32)
        y[:, ::3] *= -1
        x = (0.1 * rng.standard_normal((n, d))).astype(np.float32)
        x[n // 2:] *= 30  # logits that rise along the context: weights above 1
        k.append(0, x)
        v.append(0, y)
        kv = _one_head(C, 2, k, v)
        q = torch.randn((1, 2, 2, d), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").to(dtype)
        K, V = k.values(n)[:, None], v.values(n)[:, None]
        for limit in (40, n):
            out, lse = _attend(C, kv, n, q, limit)
            wo, wl, A, big = R.attend(q[0].double().cpu().numpy(), K, V, np.full(2, limit), d ** -0.5)
            e = (d + 4) * 2.0 ** -23 * A
            tol = ((np.expm1(2 * e) + (limit + 16) * 2.0 ** -23) * big)[..., None]
            tol = tol + (2.0 ** -8 if dtype == BF else 2.0 ** -22) * np.abs(wo)
            assert np.all(np.abs(out[0].double().cpu().numpy() - wo) <= tol), (size, limit)
            off = np.abs(lse[0].double().cpu().numpy() - wl)
            assert np.all(off <= e.T + 2.0 ** -22 * np.abs(wl) + limit * 2.0 ** -23 + 2.0 ** -21), (size, limit)


@pytest.mark.parametrize("rows", [1, 40])
def test_small_weights_beside_large_values(C, rows):
    """Values of 2^100 whose weights are 2^-30 of those of zeros, and the other way round."""
    n, d = 2048, 128
    for high in (0, 1):  # which blocks have the large logits: the zeros', the values'
        k, v = F.Blocks(n, d), F.Blocks(n, d)
        x, y = np.zeros((n, d), dtype=np.float32), np.zeros((n, d), dtype=np.float32)
        for b in range(n // 16):
            x[16 * b:16 * b + 16, 0] = 1.0 if b % 2 == high else 0.0
            y[16 * b:16 * b + 16] = 2.0 ** 100 if b % 2 else 0.0
        k.append(0, x)
        v.append(0, y)
        kv = _one_head(C, 1, k, v)
        q = torch.zeros((1, rows, 1, d), device="cuda", dtype=BF)
        q[..., 0] = 30.0
        seqs = C.Seqs([0, rows], torch.tensor([n], dtype=torch.int32, device="cuda"), n)
        lse = torch.zeros((1, 1, rows), device="cuda")
        scale = float(np.float32(np.log(2.0)))
        out = C.conduit_fp8_attn(kv, seqs, q, scale=scale, limits=torch.full((rows,), n, dtype=torch.int32, device="cuda"), lse=lse)
        w = np.exp(30.0 * scale)
        share, total = (1.0, 1.0 + w) if high == 0 else (w, 1.0 + w)
        want = share / total * 2.0 ** 100
        e = (d + 4) * 2.0 ** -23 * 30 * scale + 3 * (160 + 60) * np.log(2) * 2.0 ** -24
        assert torch.all((out.double() - want).abs() <= want * (np.expm1(2 * e) + n * 2.0 ** -23 + 2.0 ** -11 + 2.0 ** -8))
        assert np.all(np.abs(lse.double().cpu().numpy() - np.log(n / 2 * total)) <= e + n * 2.0 ** -23 + 2.0 ** -17)
