"""Attention over the 8-bit cache dim by dim: what stays finite beside NaN values, and small values beside large ones.

Tolerances as in test_gpu_fp8_attn.py, but a dim is held to its own values: with big the largest |V| of the dim among the keys seen, it is
off by (e^(2 e) - 1 + (n + 16) 2^-23 + 2^-11) big, the rounding of the output, and what weights of the tensor cores may lose
beside the row's largest: 2^-32 of a key whose value's scale is the largest, 2^v, times a code of 448 at most, for each key:
n 2^-32 448 2^v.
"""

import numpy as np
import pytest
import torch

from tests import cache_reference as R
from tests import fp8_reference as F
from tests.test_gpu_fp8_attn import _cache, _seqs

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def C():
    from paper_2609_05821_gb300 import _build
    _build.build()
    from paper_2609_05821_gb300 import conduit
    return conduit


def _check_dims(heads, q, limits, out, lse, scale, bf16):
    """One layer and request: heads [(K, V) Blocks]; every dim that is not NaN."""
    n, d = len(heads[0][0].held), q.shape[-1]
    G = q.shape[2] // len(heads)
    compared = 0
    for g, (kb, vb) in enumerate(heads):
        k, v = kb.values(n), vb.values(n)
        for i in range(q.shape[1]):
            seen = int(limits[i])
            if not seen:
                assert not out[0, i, g * G:(g + 1) * G].any()
                continue
            rows = q[0, i, g * G:(g + 1) * G].double().cpu().numpy()
            wo, wl, A, _ = R.attend(rows[None], k[:, None], v[:, None], np.array([seen]), scale)
            got = out[0, i, g * G:(g + 1) * G].double().cpu().numpy()
            wo, A = wo[0], A[0][:, None]
            clean = ~np.isnan(v[:seen]).any(0)
            assert np.array_equal(np.isnan(got), np.isnan(wo)) and np.array_equal(np.isnan(wo), np.tile(~clean, (G, 1)))
            big = np.nanmax(np.where(np.isnan(v[:seen]), -1.0, np.abs(v[:seen])), axis=0)
            e = (d + 4) * 2.0 ** -23 * A
            top = max(x for x in vb.exp[:-(-seen // 16)])
            tol = (np.expm1(2 * e) + (seen + 16) * 2.0 ** -23 + (2.0 ** -11 if bf16 else 0.0)) * big
            tol = tol + (2.0 ** -8 if bf16 else 2.0 ** -22) * np.abs(wo) + (seen * 448 * 2.0 ** (top - 32) if bf16 else 0.0)
            off = np.abs(got - wo)[:, clean]
            assert np.all(off <= tol[:, clean]), (i, g, float((off / tol[:, clean]).max()))
            compared += off.size
            if lse is not None:
                gl = lse[0, g * G:(g + 1) * G, i].double().cpu().numpy()
                assert np.all(np.abs(gl - wl[:, 0]) <= e[:, 0] + 2.0 ** -22 * np.abs(wl[:, 0]) + seen * 2.0 ** -23 + 2.0 ** -21)
    return compared


@pytest.mark.parametrize("d,page", [(64, 16), (96, 32), (128, 16)])
@pytest.mark.parametrize("dtype,n,rows", [(BF, n, rows) for n, rows in ((17, 1), (17, 17), (40, 4), (40, 60), (345, 1), (345, 19),
                                                                        (345, 60), (345, 300))] +
                         [(F32, n, rows) for n, rows in ((17, 1), (17, 17), (40, 4), (345, 19))])
def test_finite_dims_beside_nan_values(C, dtype, d, page, n, rows):
    """NaN values in blocks that every row sees, in those that some see and in the last one, neighbours in tokens and in dims
    among them: the other dims of the rows that see them are as without. (In the short contexts each value is a share of the output
    well above the tolerance.)"""
    hq, hkv, seen_first = 6, 2, max(n - rows, 0)
    places = [
        [(0, 0, 3)],
        [(5, 0, d - 1), (5, 0, d - 2), (6, 0, d - 1), (13, 1, 0)],
        [(n - 1, 0, 7), (n - 1, 1, 8), (n - 2, 0, 40)],
        [(seen_first, 0, 3), (max(seen_first - 1, 0), 0, 4), (n - 1, 0, 33), (n - 1, 0, 34)],
        [(j, 0, (7 * j) % d) for j in range(n // 3, 2 * n // 3, 3)],
        [(j, g, j % 16) for j in range(max(0, n - rows - 20), n) for g in range(2)],
    ]
    q = torch.randn((1, rows, hq, d), generator=torch.Generator(device="cuda").manual_seed(rows), device="cuda").to(dtype)
    for at, v_nan in enumerate(places):
        kv, groups = _cache(C, 30 + at, 1, hq, hkv, d, page, (n,), v_nan=v_nan)
        for limits in (None, torch.arange(rows, dtype=torch.int32, device="cuda") * n // rows):
            lse = torch.zeros((1, hq, rows), device="cuda")
            status = torch.zeros(1, dtype=torch.int32, device="cuda")
            out = C.conduit_fp8_attn(kv, _seqs(C, (n,), (rows,)), q, limits=limits, lse=lse, status=status)
            assert C.conduit_read_status(status) == C.OK
            seen = np.maximum(np.arange(n - rows + 1, n + 1), 0) if limits is None else limits.cpu().numpy()
            assert _check_dims(groups[0][0], q, seen, out, lse, d ** -0.5, dtype == BF) > 0 or not seen.any()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("rows", [1, 40])
def test_small_blocks_beside_zeros(C, dtype, rows):
    """Contexts of small blocks and zeros alone, and small dims beside blocks that are large in other dims: the small values' share
    is there at its size."""
    n, d, hq = 400, 64, 2
    rng = np.random.default_rng(4)
    q = torch.randn((1, rows, hq, d), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").to(dtype)
    x = rng.standard_normal((n, d)).astype(np.float32)
    y = rng.standard_normal((n, d)).astype(np.float32)
    for kind in range(3):
        z = y.copy()
        for b in range(n // 16):
            at = slice(16 * b, 16 * b + 16)
            if kind == 0:
                z[at] *= (0.0, 2.0 ** -20, 2.0 ** -26)[b % 3]
            elif kind == 1:
                z[at] *= (2.0 ** -20, 0.0, 2.0 ** -30)[b % 3]
            elif b % 2:
                z[at, d // 2:] = 0.0       # large, in the first dims alone
            else:
                z[at] *= 2.0 ** -12
        k, v = F.Blocks(n, d), F.Blocks(n, d)
        k.append(0, x)
        v.append(0, z)
        pool = np.full((1, n // 16, 1, 32 * d + 16), 0xFF, dtype=np.uint8)
        for b in range(n // 16):
            F.put_block(pool[0, b, 0], k, v, b)
        kv = C.Fp8Kv(torch.from_numpy(pool).cuda(), hq, d, 16, torch.arange(n // 16, dtype=torch.int32)[None])
        for limit in (20, 33, 48, 400):
            lim = torch.full((rows,), limit, dtype=torch.int32, device="cuda")
            lse = torch.zeros((1, hq, rows), device="cuda")
            out = C.conduit_fp8_attn(kv, _seqs(C, (n,), (rows,)), q, limits=lim, lse=lse)
            _check_dims([(k, v)], q, np.full(rows, limit), out, lse, d ** -0.5, dtype == BF)
