"""PackedContexts at its capacity: a request whose new rows do not fit keeps what it had.

Attention tolerances as in test_gpu_packed_attn.py (fp32 rows).
"""

import numpy as np
import pytest
import torch

from tests import cache_reference as R

pytestmark = pytest.mark.gpu

HQ, HKV, D, MAX = 4, 2, 64, 40


@pytest.fixture(scope="module")
def C():
    from paper_2609_05821_gb300 import _build
    _build.build()
    from paper_2609_05821_gb300 import conduit
    return conduit


def _draw(gen, T):
    x = torch.randn((1, T, HQ + 2 * HKV, D), generator=gen, device="cuda")
    return x[:, :, :HQ], x[:, :, HQ:HQ + HKV], x[:, :, HQ + HKV:]


def _attends_as(k, v, q, out, seen):
    """out of rows q [n, HQ, D] over the packed rows k, v [N, HKV, D]."""
    pack = lambda x: R.values(*R.pack_groups(x.float().cpu().numpy()))
    n = k.shape[0]
    want, _, A, big = R.attend(q.double().cpu().numpy(), pack(k), pack(v), np.asarray(seen), D ** -0.5)
    e = D * 2.0 ** -23 * A
    tol = ((np.expm1(2 * e) + (n + 16) * 2.0 ** -24) * big)[..., None] + 2.0 ** -22 * np.abs(want)
    assert np.all(np.abs(out.double().cpu().numpy() - want) <= tol)


def test_rows_that_do_not_fit(C):
    """Three rows for a context with room for one: none is written and its length stays, the other request
    goes on, and what comes later is right and not flagged."""
    from paper_2609_05821_gb300 import context
    gen = torch.Generator(device="cuda").manual_seed(1)
    ctx = context.PackedContexts(2, MAX, 1, HQ, HKV, D)
    q, k, v = _draw(gen, MAX - 1 + 5)
    ctx.append([MAX - 1, 5], k, v)
    assert ctx.check() == C.OK
    before = ctx.kv.pool.clone()
    q2, k2, v2 = _draw(gen, 5)
    ctx.append([3, 2], k2, v2)
    assert ctx.check() == C.ERR_INDEX and ctx.lens.tolist() == [MAX - 1, 7]
    own = ctx.kv.page_table[0].long()
    assert torch.equal(ctx.kv.pool[:, own], before[:, own])
    q3, k3, v3 = _draw(gen, 3)
    ctx.append([1, 2], k3, v3)
    out = ctx.attend([1, 2], q3)
    assert ctx.check() == C.OK and ctx.lens.tolist() == [MAX, 9]
    one = lambda *parts: torch.cat(parts)
    _attends_as(one(k[0, :MAX - 1], k3[0, :1]), one(v[0, :MAX - 1], v3[0, :1]), q3[0, :1], out[0, :1], [MAX])
    _attends_as(one(k[0, MAX - 1:], k2[0, 3:], k3[0, 1:]), one(v[0, MAX - 1:], v2[0, 3:], v3[0, 1:]), q3[0, 1:],
                out[0, 1:], [8, 9])
    # rows of the whole context: each sees the tokens up to its own
    q4 = _draw(gen, MAX + 9)[0]
    out = ctx.attend([MAX, 9], q4)
    assert ctx.check() == C.OK
    _attends_as(one(k[0, :MAX - 1], k3[0, :1]), one(v[0, :MAX - 1], v3[0, :1]), q4[0, :MAX], out[0, :MAX],
                np.arange(1, MAX + 1))


def test_steps_past_the_capacity(C):
    """Steps on a full context are flagged, write nothing and do not move its length; the other goes on."""
    from paper_2609_05821_gb300 import context
    gen = torch.Generator(device="cuda").manual_seed(2)
    ctx = context.PackedContexts(2, MAX, 1, HQ, HKV, D)
    q, k, v = _draw(gen, MAX + 3)
    ctx.append([MAX, 3], k, v)
    step = ctx.decoder(torch.float32)
    before = ctx.kv.pool.clone()
    rows = []
    for i in range(3):
        q2, k2, v2 = _draw(gen, 2)
        out = step(q2, k2, v2).clone()
        rows.append((q2, k2, v2, out))
        assert ctx.check() == C.ERR_INDEX and ctx.lens.tolist() == [MAX, 4 + i]
    own = ctx.kv.page_table[0].long()
    assert torch.equal(ctx.kv.pool[:, own], before[:, own])
    for i, (q2, _, _, out) in enumerate(rows):
        kk, vv = (torch.cat([x[0, MAX:]] + [r[at][0, 1:] for r in rows[:i + 1]]) for x, at in ((k, 1), (v, 2)))
        _attends_as(kk, vv, q2[0, 1:], out[0, 1:], [4 + i])
    # the caller ends a context by setting its length
    ctx.lens[0] = 0
    q2, k2, v2 = _draw(gen, 2)
    out = step(q2, k2, v2)
    assert ctx.check() == C.OK and ctx.lens.tolist() == [1, 7]
    _attends_as(k2[0, :1], v2[0, :1], q2[0, :1], out[0, :1], [1])
