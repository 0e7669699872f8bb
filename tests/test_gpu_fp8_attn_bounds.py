"""8-bit attention whose max_len lies far above its lengths: chunks that most contexts do not reach, on every kernel."""

import numpy as np
import pytest
import torch

from tests.test_gpu_fp8_attn import _cache, _check, _seqs

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def C():
    from paper_2609_05821_gb300 import _build
    _build.build()
    from paper_2609_05821_gb300 import conduit
    return conduit


@pytest.mark.parametrize("dtype,hq,hkv,d,lens,rows", [
    (BF, 4, 2, 128, (130, 0, 1, 700), (1, 1, 1, 1)),                # few rows
    (BF, 8, 1, 64, (33, 257), (3, 2)),
    (BF, 28, 4, 128, (130, 0, 1, 700), (40, 3, 1, 100)),            # many rows: one column tile, pairs, and rows without keys
    (BF, 28, 4, 96, (5, 2500), (60, 37)),
    (BF, 6, 2, 64, (900,), (300,)),
    (F32, 4, 2, 64, (130, 0, 1, 700), (1, 2, 1, 3)),
])
@pytest.mark.parametrize("most", [4096, 200000])
def test_lengths_far_below_the_bound(C, dtype, hq, hkv, d, lens, rows, most):
    kv, groups = _cache(C, len(lens), 1, hq, hkv, d, 16, lens)
    wide = torch.full((len(lens), most // 16), 10 ** 6, dtype=torch.int32)  # pages that no token has do not exist
    wide[:, :kv.page_table.shape[1]] = kv.page_table.cpu()
    kv = C.Fp8Kv(kv.pool, hq, d, 16, wide)
    T = sum(rows)
    q = torch.randn((1, T, hq, d), generator=torch.Generator(device="cuda").manual_seed(T), device="cuda").to(dtype)
    seqs = _seqs(C, lens, rows, most=most)
    status, lse = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros((1, hq, T), device="cuda")
    ws = torch.full((max(C.conduit_fp8_attn_workspace_size(kv, seqs, dtype), 1),), 0xFF, dtype=torch.uint8, device="cuda")
    for limits in (None, torch.from_numpy(np.random.default_rng(T).integers(0, most, T)).int().cuda()):
        out = C.conduit_fp8_attn(kv, seqs, q, limits=limits, lse=lse, workspace=ws, status=status)
        assert C.conduit_read_status(status) == C.OK
        _check(groups, lens, rows, q, limits, out, lse, d ** -0.5, dtype == BF)
