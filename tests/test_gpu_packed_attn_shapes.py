"""Attention over the 4-bit cache: head and page sizes on every kernel, precise log-sum-exps, and their use in scoring.

Outputs as in test_gpu_packed_attn.py. A log-sum-exp of rows with few columns a KV head, or
that see fewer than 2,048 keys, has no term for rounded keys: it is off by d 2^-23 of the largest scale sum |q||k|.
"""

import numpy as np
import pytest
import torch

from tests import cache_reference as R
from tests import test_gpu_variants as TV
from tests.test_gpu_packed_attn import BF, C, F, _cache, _check  # noqa: F401 (C is a fixture)

pytestmark = pytest.mark.gpu


def _limits(rng, lens, rows):
    """Keys that each row sees: none, one, all, past the context, and numbers in between."""
    got = []
    for n, c in zip(lens, rows):
        x = rng.integers(0, n + 1, c)
        x[::7], x[1::7], x[2::7], x[3::7] = 0, min(n, 1), n, n + 100
        got.append(x)
    return torch.from_numpy(np.concatenate(got).astype(np.int32)).cuda()


def _run(C, dtype, L, hq, hkv, d, ps, lens, rows, limits, nan_at, max_len=None):
    kv, groups = _cache(C, 7 * d + ps, L, hq, hkv, d, ps, lens, nan_at=nan_at)
    T = sum(rows)
    gen = torch.Generator(device="cuda").manual_seed(T + d)
    q = torch.randn((L, T, hq, d), generator=gen, device="cuda").to(dtype)
    lim = _limits(np.random.default_rng(T), lens, rows) if limits else None
    dev_lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    seqs = C.Seqs(np.concatenate([[0], np.cumsum(rows)]), dev_lens, max_len or max(lens))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    lse = torch.zeros((L, hq, T), device="cuda")
    out = C.conduit_packed_attn(kv, seqs, q, limits=lim, lse=lse, status=status)
    assert C.conduit_read_status(status) == C.OK
    _check(C, kv, groups, lens, rows, q, lim, out, None, d ** -0.5, dtype == BF)
    # log-sum-exps, with the keys' rounding only where the call may round them
    t, few_columns = 0, max(rows) * (hq // hkv) <= 8
    for r, (n, c) in enumerate(zip(lens, rows)):
        seen = np.arange(n - c + 1, n + 1) if lim is None else lim[t:t + c].cpu().numpy()
        seen = np.clip(seen, 0, n)
        for l in range(L if c else 0):
            k, v = (R.values(*part) for part in groups[r][l])
            _, wl, A, _ = R.attend(q[l, t:t + c].double().cpu().numpy(), k, v, seen, d ** -0.5)
            gl = lse[l, :, t:t + c].double().cpu().numpy()
            assert np.array_equal(np.isneginf(gl), np.isneginf(wl)) and np.array_equal(np.isnan(gl), np.isnan(wl))
            rounded = dtype == BF and not few_columns and (seen >= 2048)
            e = (d * 2.0 ** -23 + np.where(rounded, 2.0 ** -11, 0.0))[None] * A.T if np.ndim(rounded) else d * 2.0 ** -23 * A.T
            room = e + 2.0 ** -22 * np.abs(wl) + n * 2.0 ** -24 + 2.0 ** -21
            fin = np.isfinite(wl)
            assert np.all(np.abs(gl[fin] - wl[fin]) <= room[fin]), (r, l)
        t += c


# (L, hq, hkv, d, page, cached tokens, rows, limits, token packed from NaN, max_len or None)
MANY = [
    (1, 6, 2, 96, 8, (2300, 61, 700), (70, 61, 33), False, None, None),
    (1, 18, 2, 96, 64, (900, 129), (40, 9), True, None, None),       # three column tiles and one; keys in two parts
    (2, 3, 1, 96, 128, (2100, 333), (100, 43), True, None, None),
    (1, 6, 2, 96, 16, (400,), (90,), False, 350, None),
    (1, 6, 2, 96, 32, (2500,), (90,), True, 2050, None),
    (1, 4, 4, 64, 8, (2051, 130), (130, 129), True, None, None),
    (1, 8, 2, 64, 128, (300, 1, 2600), (70, 1, 33), False, None, None),
    (1, 8, 2, 64, 1024, (1500,), (129,), True, 1400, None),
    (1, 14, 2, 128, 8, (515,), (40,), True, None, 4096),
    (1, 14, 2, 128, 64, (2500, 64, 65), (20, 64, 37), False, None, None),
    (1, 14, 2, 128, 128, (777, 127), (37, 20), True, 100, 4096),
    (1, 7, 1, 128, 1024, (2200, 90), (33, 40), True, None, None),
]


@pytest.mark.parametrize("L,hq,hkv,d,ps,lens,rows,limits,nan_at,max_len", MANY)
def test_many_rows(C, L, hq, hkv, d, ps, lens, rows, limits, nan_at, max_len):
    if nan_at is not None:
        lens = tuple(max(n, nan_at + 1) for n in lens)
    _run(C, BF, L, hq, hkv, d, ps, lens, rows, limits, nan_at, max_len)


FEW = [(d, ps) for d in (64, 96, 128) for ps in (8, 16, 32, 64, 1024)]


@pytest.mark.parametrize("d,ps", FEW)
def test_one_row(C, d, ps):
    _run(C, BF, 2, 14, 2, d, ps, (5000, 1, 31, 257), (1, 1, 1, 1), False, None)


@pytest.mark.parametrize("d,ps", [(96, 64), (128, 8), (64, 128)])
def test_few_rows_with_limits_and_nan(C, d, ps):
    _run(C, BF, 1, 4, 2, d, ps, (700, 300), (4, 3), True, 290)


@pytest.mark.parametrize("d,ps,rows", [(32, 16, 40), (160, 64, 3), (256, 8, 9)])
def test_other_head_sizes(C, d, ps, rows):
    """On the CUDA cores: bf16 rows, fp32 arithmetic (and so log-sum-exps without any rounding of keys)."""
    _run(C, BF, 1, 4, 2, d, ps, (300, 77), (rows, 2), True, 70)


def test_many_rows_in_fp32(C):
    _run(C, F, 1, 4, 2, 64, 32, (900, 66), (70, 5), True, None)


def test_log_sum_exps_in_scoring(C):
    """Visual tokens in a plain cache, the text around them in 4 bits: the log-sum-exps of the scoring queries over
    the text are what conduit_score takes for the full context. Against the oracle with 64-bit log-sum-exps."""
    from paper_2609_05821_gb300 import pipeline
    inputs, pipe, layers = TV._setup(pipeline, "ragged_bf16_d64")
    q = inputs["q"]  # [L, Hq, Q, d]
    L, hq, _, d = q.shape
    hkv, qo = inputs["k"].shape[1], inputs["q_off"].tolist()
    rows = [b - a for a, b in zip(qo[:-1], qo[1:])]
    lens = [45, 0, 700][:len(rows)]
    kv, groups = _cache(C, 5, L, hq, hkv, d, 16, lens)
    seqs = C.Seqs(qo, torch.tensor(lens, dtype=torch.int32, device="cuda"), 700)
    limits = torch.repeat_interleave(torch.tensor(lens), torch.tensor(rows)).int().cuda()
    lse = torch.zeros((L, hq, qo[-1]), device="cuda")
    C.conduit_packed_attn(kv, seqs, q.transpose(1, 2), limits=limits, lse=lse)
    want = torch.zeros((L, hq, qo[-1]), dtype=torch.float64)
    for r, n in enumerate(lens):
        for l in range(L):
            k, v = (R.values(*part) for part in groups[r][l])
            x = q[l, :, qo[r]:qo[r + 1]].transpose(0, 1).double().cpu().numpy()
            want[l, :, qo[r]:qo[r + 1]] = torch.from_numpy(R.attend(x, k, v, [n] * rows[r], d ** -0.5)[1])
    got = C.conduit_score_ex(pipe.kv, pipe.batch, pipe.q, layers, extra_lse=lse)
    torch.cuda.synchronize()
    TV._compare(pipe, inputs, got, layers, TV._rtol(inputs), extra_lse=want)
