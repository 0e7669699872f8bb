"""Attention on the tensor cores with bf16 queries whose elements lie far apart in size, against 64 bits.

A row's queries are scaled by a power of two to fp16's range: the largest to [2^15, 2^16) over the 8-bit cache, to [2^8, 2^9) over the
4-bit one. fp16 holds bf16's eight bits down to 2^-17 and rounds what is smaller to multiples of 2^-24. So an
element is exact down to 2^-32 (2^-25) of its row's largest and off by 2^-25, that is 2^-40 (2^-33) of the largest, at most
below. A logit is then off by scale sum |k| times that over the dims concerned, beside the rounding of its fp32 sum,
(d + 4) 2^-23 of A = scale sum |q||k|. The rest as in test_gpu_fp8_attn.py.
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


def _eight_bits(C, k, v, hq):
    n, d = k.shape
    kb, vb = F.Blocks(n, d), F.Blocks(n, d)
    kb.append(0, k.astype(np.float32))
    vb.append(0, v.astype(np.float32))
    pool = np.full((1, n // 16, 1, 32 * d + 16), 0xFF, dtype=np.uint8)
    for b in range(n // 16):
        F.put_block(pool[0, b, 0], kb, vb, b)
    kv = C.Fp8Kv(torch.from_numpy(pool).cuda(), hq, d, 16, torch.arange(n // 16, dtype=torch.int32)[None])
    return kv, kb.values(n), vb.values(n)


def _check(C, attn, kv, k, v, q, scale, below, step):
    """below: elements under it times their row's largest are off by step times the largest."""
    n, d = k.shape
    rows = q.shape[1]
    seqs = C.Seqs([0, rows], torch.tensor([n], dtype=torch.int32, device="cuda"), n)
    lse = torch.zeros((1, q.shape[2], rows), device="cuda")
    limits = torch.full((rows,), n, dtype=torch.int32, device="cuda")
    out = attn(kv, seqs, q, scale=scale, limits=limits, lse=lse)
    qd = q[0].double().cpu().numpy()
    wo, wl, A, big = R.attend(qd, k[:, None], v[:, None], np.full(rows, n), scale)
    most = np.abs(qd).max(-1, keepdims=True)
    small = (np.abs(qd) < below * most) & (qd != 0)
    extra = scale * step * most[..., 0] * np.einsum("thd,nd->thn", small.astype(float), np.abs(k)).max(-1)
    e = (d + 4) * 2.0 ** -23 * A + (extra if q.dtype == BF else 0.0)
    tol = (np.expm1(2 * e) + (n + 16) * 2.0 ** -23 + (2.0 ** -11 if q.dtype == BF else 0.0)) * big
    tol = tol[..., None] + (2.0 ** -8 if q.dtype == BF else 2.0 ** -22) * np.abs(wo)
    assert np.all(np.abs(out[0].double().cpu().numpy() - wo) <= tol)
    off = np.abs(lse[0].double().cpu().numpy() - wl)
    assert np.all(off <= e.T + 2.0 ** -22 * np.abs(wl) + n * 2.0 ** -23 + 2.0 ** -21), (off.max(), e.max())


@pytest.mark.parametrize("dtype,d,rows,power", [(BF, d, rows, power) for d in (64, 96, 128) for rows in (1, 5, 40, 150)
                                                for power in (20, 30, 34, 38, 44)] +
                         [(F32, 128, rows, power) for rows in (1, 5) for power in (20, 38, 80)])
def test_unequal_queries_over_8_bits(C, dtype, d, rows, power):
    """A dim 2^power larger than the others meets zero keys, so that the logits come from the small dims alone."""
    n, hq = 208, 2
    rng = np.random.default_rng(power)
    k = rng.standard_normal((n, d))
    k[:, 7] = 0.0
    kv, k, v = _eight_bits(C, k, rng.standard_normal((n, d)), hq)
    q = torch.from_numpy(rng.standard_normal((1, rows, hq, d)))
    q[..., 7] = 1.9 * 2.0 ** power
    q[:, :, 1] *= 2.0 ** -30  # a head of its own size, whose scale does not follow
    _check(C, C.conduit_fp8_attn, kv, k, v, q.to("cuda", dtype), d ** -0.5, 2.0 ** -32, 2.0 ** -40)


@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("size", [-126, -100, 96])
def test_elements_of_every_size_over_8_bits(C, rows, size):
    """Rows whose elements are spread over 2^40, near the least and the largest bf16 numbers too."""
    n, d, hq = 208, 128, 2
    rng = np.random.default_rng(7)
    k = rng.standard_normal((n, d)) * 2.0 ** rng.integers(-8, 1, (1, d))
    kv, k, v = _eight_bits(C, k, rng.standard_normal((n, d)), hq)
    q = rng.standard_normal((1, rows, hq, d)) * 2.0 ** rng.integers(-40, 1, (1, rows, hq, d))
    q = torch.from_numpy(q * 2.0 ** size).to("cuda", BF)
    _check(C, C.conduit_fp8_attn, kv, k, v, q, float(np.float32(2.0 ** -size / 8)) if size > -120 else 2.0 ** 120, 2.0 ** -32, 2.0 ** -40)


@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("power", [20, 24, 30, 36])
def test_unequal_queries_over_4_bits(C, rows, power):
    n, d, hq = 208, 128, 7
    rng = np.random.default_rng(power)
    k = np.repeat(rng.integers(-4, 5, (n, 4)) / 4.0, 32, axis=1)  # a group of 32 dims is held exactly
    k[:, :32] = 0.0
    v = np.repeat(rng.integers(-8, 9, (n, 4)) / 8.0, 32, axis=1)
    kv = C.PackedKv.empty(1, n // 16, hq, 1, d, 16, torch.arange(n // 16, dtype=torch.int32)[None])
    seqs = C.Seqs([0, n], torch.tensor([n], dtype=torch.int32, device="cuda"), n)
    C.conduit_packed_append(kv, seqs, *(torch.from_numpy(x).float().cuda()[None, :, None] for x in (k, v)))
    q = torch.from_numpy(rng.standard_normal((1, rows, hq, d)))
    q[..., 7] = 1.9 * 2.0 ** power
    _check(C, C.conduit_packed_attn, kv, k, v, q.to("cuda", BF), d ** -0.5, 2.0 ** -25, 2.0 ** -33)
