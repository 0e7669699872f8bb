"""PackedContexts: prompts, decoding steps in a CUDA graph, and a context taken up for scoring.

The attention of a step is compared with softmax attention in 64 bits over the values that
the cache stands for (read back with conduit_packed_read); tolerances as in
test_gpu_packed_attn.py.
"""

import numpy as np
import pytest
import torch

from tests import cache_reference as R

pytestmark = pytest.mark.gpu

L, HQ, HKV, D, REQ, MAX = 2, 14, 2, 64, 3, 400
PROMPTS = (100, 37, 250)


@pytest.fixture(scope="module")
def C():
    from paper_2609_05821_gb300 import _build
    _build.build()
    from paper_2609_05821_gb300 import conduit
    return conduit


def _rows(gen, T):
    x = torch.randn((L, T, HQ + 2 * HKV, D), generator=gen, device="cuda").to(torch.bfloat16)
    return x[:, :, :HQ], x[:, :, HQ:HQ + HKV], x[:, :, HQ + HKV:]


def _positions(start, rows):
    """Patches of a 16-wide grid: time, height, width."""
    slot = np.concatenate([np.arange(s, s + n) for s, n in zip(start, rows)])
    return torch.tensor(np.stack([slot // 256, slot % 256 // 16, slot % 16]), dtype=torch.int32, device="cuda")


def _values(C, ctx, lens):
    """What the cache stands for, float64 [L, N, Hkv, d] per request."""
    off = np.concatenate([[0], np.cumsum(lens)]).tolist()
    batch = C.Batch(off, off, list(range(REQ + 1)), list(range(REQ + 1)))
    dst = C.KvCache(*[torch.zeros((L, HKV, off[-1], D), device="cuda") for _ in range(2)], HQ)
    ctx.take_up(batch, dst)
    return [tuple(x[:, :, a:b].transpose(1, 2).double().cpu().numpy() for x in (dst.k, dst.v))
            for a, b in zip(off[:-1], off[1:])]


def _check(values, lens, rows, q, out):
    t = 0
    for r, (n, c) in enumerate(zip(lens, rows)):
        for l in range(L):
            k, v = values[r][0][l], values[r][1][l]
            seen = np.arange(n - c + 1, n + 1)
            wo, _, A, big = R.attend(q[l, t:t + c].double().cpu().numpy(), k, v, seen, D ** -0.5)
            e = (D * 2.0 ** -23 + 2.0 ** -11) * A
            tol = ((np.expm1(2 * e) + (n + 16) * 2.0 ** -24 + 2.0 ** -10) * big)[..., None] + 2.0 ** -8 * np.abs(wo)
            assert np.all(np.abs(out[l, t:t + c].double().cpu().numpy() - wo) <= tol)
        t += c


def test_prompts_then_decoding_in_a_graph(C):
    from paper_2609_05821_gb300 import context
    gen = torch.Generator(device="cuda").manual_seed(3)
    rope = C.Rope(C.rope_table(10000.0, D, 64), [i % 3 for i in range(D // 2)])
    ctx = context.PackedContexts(REQ, MAX, L, HQ, HKV, D, rope, page_size=16)
    q, k, v = _rows(gen, sum(PROMPTS))
    pos = _positions([0] * REQ, PROMPTS)
    q_rot = ctx.append(PROMPTS, k, v, pos, q)
    assert torch.equal(q_rot, C.conduit_rope(rope, q, pos))
    out = ctx.attend(PROMPTS, q_rot)
    assert ctx.check() == C.OK
    lens = list(PROMPTS)
    _check(_values(C, ctx, lens), lens, lens, q_rot, out)

    step = ctx.decoder()
    held = [torch.empty((L, REQ, h, D), dtype=torch.bfloat16, device="cuda") for h in (HQ, HKV, HKV)]
    at = torch.zeros((3, REQ), dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        before = ctx.lens.clone()
        with torch.cuda.graph(graph, stream=side):
            out = step(*held, at)
        ctx.lens.copy_(before)
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(4):
        for dst, src in zip(held, _rows(gen, REQ)):
            dst.copy_(src)
        at.copy_(_positions(lens, [1] * REQ))
        graph.replay()
        lens = [n + 1 for n in lens]
        assert ctx.check() == C.OK and ctx.lens.tolist() == lens
        _check(_values(C, ctx, lens), lens, [1] * REQ, C.conduit_rope(rope, held[0], at), out)


def test_context_taken_up_for_scoring(C):
    """Scores of a taken-up context are those of a cache filled with the same values."""
    from paper_2609_05821_gb300 import context
    gen = torch.Generator(device="cuda").manual_seed(4)
    ctx = context.PackedContexts(REQ, MAX, L, HQ, HKV, D)
    q, k, v = _rows(gen, sum(PROMPTS))
    ctx.append(PROMPTS, k, v)
    off = np.concatenate([[0], np.cumsum(PROMPTS)]).tolist()
    batch = C.Batch(off, off, list(range(REQ + 1)), [0, 4, 8, 12])
    zeros = lambda: torch.zeros((L, HKV, off[-1], D), dtype=torch.bfloat16, device="cuda")
    taken = ctx.take_up(batch, C.KvCache(zeros(), zeros(), HQ))
    assert ctx.check() == C.OK
    own = []
    for x in (k, v):
        y = torch.from_numpy(R.values(*R.pack_groups(x.float().cpu().numpy()))).to(torch.bfloat16)
        own.append(y.transpose(1, 2).contiguous().cuda())
    query = torch.randn((L, HQ, 12, D), generator=gen, device="cuda").to(torch.bfloat16)
    for a, b in zip(C.conduit_score(taken, batch, query), C.conduit_score(C.KvCache(*own, HQ), batch, query)):
        assert torch.equal(a, b)


def test_context_that_is_full(C):
    """A step past max_len is flagged and writes nothing."""
    from paper_2609_05821_gb300 import context
    ctx = context.PackedContexts(1, 16, 1, 2, 1, D)
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn((1, 16, 3, D), generator=gen, device="cuda").to(torch.bfloat16)
    ctx.append([16], x[:, :, 2:], x[:, :, 2:])
    assert ctx.check() == C.OK
    before = ctx.kv.pool.clone()
    ctx.append([1], x[:, :1, 2:], x[:, :1, 2:])
    assert ctx.check() == C.ERR_INDEX and torch.equal(ctx.kv.pool, before)
