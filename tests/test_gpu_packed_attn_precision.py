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
