"""Appends whose rotation pairs neighbouring dims: plain and 4-bit pages, in 16-byte chunks and element by element.

Bounds and the rotation in fp32 as in test_gpu_rope_append.py.
"""

import numpy as np
import pytest
import torch

from tests import cache_reference as R
from tests.test_gpu_rope_append import C, _axis, _close, _draw, _table_of  # noqa: F401 (C is a fixture)

pytestmark = pytest.mark.gpu

# (dtype, L, hq, hkv, d, rot, page, cached tokens, rows of the call)
CASES = [
    (torch.bfloat16, 2, 8, 2, 128, 128, 16, (40, 17, 300), (1, 17, 47)),
    (torch.bfloat16, 1, 4, 2, 64, 32, 8, (100, 9), (100, 2)),
    (torch.bfloat16, 1, 6, 3, 96, 36, 32, (33, 70), (33, 5)),     # 18 pairs, rows of 36 and 60 dims: no whole chunks
    (torch.bfloat16, 1, 2, 1, 32, 6, 16, (20,), (7,)),
    (torch.float32, 2, 6, 2, 96, 96, 64, (70, 1), (65, 1)),
    (torch.float32, 1, 3, 3, 64, 44, 16, (5, 60), (5, 3)),
]


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("strided", [False, True])
@pytest.mark.parametrize("dtype,L,hq,hkv,d,rot,ps,lens,rows", CASES)
def test_append(C, dtype, L, hq, hkv, d, rot, ps, lens, rows, strided, packed):
    T, axis = sum(rows), _axis("thw", rot // 2)
    x = _draw(T + rot)(L, T, hq + 2 * hkv + 1, d, dtype=dtype)[:, :, 1:]
    q, k, v = x[:, :, :hq], x[:, :, hq:hq + hkv], x[:, :, hq + hkv:]
    if not strided:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    table = C.rope_table(10000.0, rot, 700)
    pos = torch.randint(0, 700, (max(axis) + 1, T), dtype=torch.int32, device="cuda")
    rope = C.Rope(table, axis, "pairs")
    seqs = C.Seqs(np.concatenate([[0], np.cumsum(rows)]), torch.tensor(lens, dtype=torch.int32, device="cuda"), max(lens))
    pages, P = _table_of(lens, ps)
    slot = [(int(pages[r, j // ps]), j % ps) for r, (n, c) in enumerate(zip(lens, rows)) for j in range(n - c, n)]
    at = [torch.tensor(s, device="cuda") for s in zip(*slot)]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    turn = lambda y: R.rotate(y, pos, table, axis, "pairs")
    if packed:
        kv = C.PackedKv.empty(L, P, hq, hkv, d, ps, torch.from_numpy(pages))
        kv.pool.zero_()
        q_out = C.conduit_packed_append(kv, seqs, k, v, rope, pos, q, status=status)
        # all pages back, as one request whose pages are in order
        every = C.PackedKv(kv.pool, hq, d, ps, torch.arange(P, dtype=torch.int32)[None])
        dst = C.KvCache(*[torch.zeros((L, hkv, P * ps, d), device="cuda") for _ in range(2)], hq)
        C.conduit_packed_read(every, C.Batch([0, P * ps], [0, P * ps], [0, 1], [0, 1]), dst)
        got = [y.view(L, hkv, P, ps, d)[:, :, at[0], at[1]].transpose(1, 2) for y in (dst.k, dst.v)]
        cs = table[pos.long()[torch.as_tensor(axis, device="cuda")].T, torch.arange(rot // 2, device="cuda")][:, None]
        f, kk = k.float(), k.float().clone()
        kk[..., 0:rot:2] = f[..., 0:rot:2] * cs[..., 0] - f[..., 1:rot:2] * cs[..., 1]
        kk[..., 1:rot:2] = f[..., 1:rot:2] * cs[..., 0] + f[..., 0:rot:2] * cs[..., 1]
        for y, rows32 in zip(got, (kk, v.float())):
            assert np.array_equal(y.cpu().numpy(), R.values(*R.pack_groups(rows32.cpu().numpy())).astype(np.float32))
    else:
        pool = [torch.zeros((L, P, hkv, ps, d), dtype=dtype, device="cuda") for _ in range(2)]
        kv = C.KvCache(*pool, hq, ps, torch.from_numpy(pages))
        q_out = C.conduit_kv_append(kv, seqs, k, v, rope, pos, q, status=status)
        got = [y.transpose(2, 3)[:, at[0], at[1]] for y in pool]
        _close(got[0], k, turn(k), dtype, rot // 2, "pairs")
        assert torch.equal(got[1], v)
    assert C.conduit_read_status(status) == C.OK
    _close(q_out, q, turn(q), dtype, rot // 2, "pairs")
