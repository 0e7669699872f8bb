"""Beam search over contexts in 8 and 4 bits, as a serving loop runs it: a prompt in the first beam of each group, children,
steps of attention, selection and reordering replayed from a graph, a restart.

Each beam's history is kept apart from the library, as the values that an 8-bit cache would hold for it alone; a
step's attention is compared with softmax attention in 64 bits over them (tolerances as in test_gpu_fp8_attn.py), its selection
with the ranking of the step's own logits. In 4 bits, whose values depend on a token alone, a beam's attention has the
bits of the same history in contexts of its own.
"""

import copy

import numpy as np
import pytest
import torch

from tests import cache_reference as R
from tests import fp8_reference as F
from tests.test_gpu_beam import EPS, _scores

pytestmark = pytest.mark.gpu
BF = torch.bfloat16

L, HQ, HKV, D, W, G, MAX, VOCAB = 2, 6, 2, 64, 3, 2, 96, 500
N = W * G
PROMPTS = (21, 40)


@pytest.fixture(scope="module")
def C():
    from paper_2609_05821_gb300 import _build
    _build.build()
    from paper_2609_05821_gb300 import conduit
    return conduit


class Model:
    """Tokens to rows, attention to logits: fixed random weights."""

    def __init__(self, seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        draw = lambda *s: torch.randn(s, generator=gen, device="cuda")
        size = torch.exp(draw(VOCAB, 1, 1))  # tokens of unequal size: scales that grow over a block
        self.rows = [(draw(VOCAB, L, h * D) * size).view(VOCAB, L, h, D).to(BF) for h in (HQ, HKV, HKV)]
        self.out = draw(L * HQ * D, VOCAB) / 4

    def qkv(self, token):
        return [r[token].transpose(0, 1) for r in self.rows]  # [L, T, h, D]

    def logits(self, out):
        return out.transpose(0, 1).reshape(out.shape[1], -1).float() @ self.out


def _check_attention(beams, out, q):
    for b, (heads, n) in enumerate(beams):
        for l in range(L):
            k, v = (np.stack([heads[l][g][w].values(n) for g in range(HKV)], axis=1) for w in (0, 1))
            wo, _, A, big = R.attend(q[l, b:b + 1].double().cpu().numpy(), k, v, [n], D ** -0.5)
            e = (D + 4) * 2.0 ** -23 * A
            tol = ((np.expm1(2 * e) + (n + 16) * 2.0 ** -23 + 2.0 ** -11) * big)[..., None] + 2.0 ** -8 * np.abs(wo)
            assert np.all(np.abs(out[l, b:b + 1].double().cpu().numpy() - wo) <= tol), (b, l)


def _new_beam():
    return [[(F.Blocks(MAX, D), F.Blocks(MAX, D)) for _ in range(HKV)] for _ in range(L)]


def _extend(beam, k, v):
    """Rows k, v [L, T, HKV, D] to the end of a beam (heads, length)."""
    heads, n = beam
    for l in range(L):
        for g in range(HKV):
            heads[l][g][0].append(n, k[l, :, g].float().cpu().numpy())
            heads[l][g][1].append(n, v[l, :, g].float().cpu().numpy())
    return heads, n + k.shape[1]


def test_search_in_8_bits(C):
    from paper_2609_05821_gb300 import context
    model = Model(1)
    ctx = context.PackedContexts(N, MAX, L, HQ, HKV, D, bits=8)
    step = ctx.decoder()
    first = torch.arange(N, dtype=torch.int32, device="cuda") // W * W
    score = torch.zeros((G, W), device="cuda")
    parent, token = (torch.zeros((G, W), dtype=torch.int32, device="cuda") for _ in range(2))
    logits = torch.zeros((N, VOCAB), device="cuda")
    held = {}

    def one():
        ctx.reorder(parent.view(-1), W)
        q, k, v = model.qkv(token.view(-1).long())
        held["q"] = q.contiguous()
        held["out"] = step(held["q"], k.contiguous(), v.contiguous())
        logits.copy_(model.logits(held["out"]))
        C.conduit_beam_select(logits, score.view(-1), W, W, score_out, parent, token, status=ctx.status)
        score.copy_(score_out)

    score_out = torch.zeros_like(score)
    graph = None
    for search in range(2):
        ctx.restart()
        gen = torch.Generator(device="cuda").manual_seed(search)
        rows = [0] * N
        for g, n in enumerate(PROMPTS):
            rows[g * W] = n
        prompt = torch.randint(VOCAB, (sum(PROMPTS),), generator=gen, device="cuda")
        q, k, v = model.qkv(prompt)
        ctx.append(rows, k, v)
        beams, at = [None] * N, 0
        for g, n in enumerate(PROMPTS):
            beams[g * W] = _extend((_new_beam(), 0), k[:, at:at + n], v[:, at:at + n])
            at += n
        # the first step continues one beam of each group: every beam's parent is the first, with its own first token
        parent.copy_(first.view(G, W))
        token.copy_(torch.randint(VOCAB, (G, W), generator=gen, device="cuda", dtype=torch.int32))
        score.copy_(-torch.rand((G, W), generator=gen, device="cuda"))
        if graph is None:
            stream = torch.cuda.Stream()
            stream.wait_stream(torch.cuda.current_stream())
            keep = [x.clone() for x in (ctx.kv.pool, ctx.kv.page_table, ctx.lens, score, parent, token)]
            with torch.cuda.stream(stream):
                one()
                graph = torch.cuda.CUDAGraph()
                for x, y in zip((ctx.kv.pool, ctx.kv.page_table, ctx.lens, score, parent, token), keep):
                    x.copy_(y)
                with torch.cuda.graph(graph, stream=stream):
                    one()
            torch.cuda.current_stream().wait_stream(stream)
        for _ in range(30):
            was, chosen, sums = parent.view(-1).tolist(), token.view(-1).long(), score.view(-1).clone()
            beams = [copy.deepcopy(beams[p]) for p in was]
            _, k, v = model.qkv(chosen)
            beams = [_extend(b, k[:, i:i + 1], v[:, i:i + 1]) for i, b in enumerate(beams)]
            graph.replay()
            assert ctx.check() == C.OK
            assert ctx.lens.tolist() == [n for _, n in beams]
            _check_attention(beams, held["out"], held["q"])
            want, _ = _scores(logits, sums)
            for g in range(G):
                s = want[g * W:(g + 1) * W]
                best = np.sort(s.ravel())[::-1][:W]
                got = s[parent[g].cpu().numpy() - g * W, token[g].cpu().numpy()]
                assert np.all(np.abs(got - best) <= 2 * EPS)
                assert np.all(np.abs(score[g].double().cpu().numpy() - best) <= EPS + 2.0 ** -24 * np.abs(best))


def test_search_in_4_bits_has_the_bits_of_contexts_of_their_own(C):
    from paper_2609_05821_gb300 import context
    model = Model(2)
    ctx = context.PackedContexts(N, MAX, L, HQ, HKV, D, page_size=8)
    own = context.PackedContexts(N, MAX, L, HQ, HKV, D, page_size=8)
    rng = np.random.default_rng(3)
    tokens = [rng.integers(0, VOCAB, PROMPTS[b // W]).tolist() for b in range(N)]
    rows = [0] * N
    for g in range(G):
        rows[g * W] = PROMPTS[g]
        for b in range(W):
            tokens[g * W + b] = tokens[g * W]
    _, k, v = model.qkv(torch.tensor(sum((tokens[g * W] for g in range(G)), []), device="cuda"))
    ctx.append(rows, k, v)
    parent = np.arange(N) // W * W
    step = ctx.decoder()
    for _ in range(20):
        ctx.reorder(torch.tensor(parent, dtype=torch.int32, device="cuda"), W)
        new = rng.integers(0, VOCAB, N)
        tokens = [tokens[p] + [int(t)] for p, t in zip(parent, new)]
        q, k, v = (x.contiguous() for x in model.qkv(torch.tensor(new, device="cuda")))
        out = step(q, k, v)
        assert ctx.check() == C.OK
        own.restart()
        _, k, v = model.qkv(torch.tensor(sum(tokens, []), device="cuda"))
        own.append([len(t) for t in tokens], k, v)
        assert torch.equal(out, own.attend([1] * N, q))
        parent = np.arange(N) // W * W + rng.integers(0, W, N)


def test_a_context_in_8_bits_taken_up_and_full(C):
    """Prompts and steps as in 4 bits: values read back, a request past its length flagged and left as it was."""
    from paper_2609_05821_gb300 import context
    ctx = context.PackedContexts(2, 20, L, HQ, HKV, D, bits=8)
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn((L, 30, HQ + 2 * HKV, D), generator=gen, device="cuda").to(BF)
    q, k, v = x[:, :, :HQ], x[:, :, HQ:HQ + HKV], x[:, :, HQ + HKV:]
    ctx.append([19, 11], k, v)
    step = ctx.decoder()
    one = [x[:, :2].contiguous() for x in (q, k, v)]
    step(*one)
    assert ctx.check() == C.OK and ctx.lens.tolist() == [20, 12]
    before = ctx.kv.pool.clone()
    step(*one)
    assert ctx.check() == C.ERR_INDEX and ctx.lens.tolist() == [20, 13]
    assert torch.equal(ctx.kv.pool[:, :2], before[:, :2])
    batch = C.Batch([0, 20, 33], [0, 20, 33], [0, 1, 2], [0, 1, 2])
    dst = ctx.take_up(batch, C.KvCache(*[torch.zeros((L, HKV, 33, D), device="cuda") for _ in range(2)], HQ))
    b = F.Blocks(20, D)
    b.append(0, k[1, :19, 1].float().cpu().numpy())
    b.append(19, k[1, :1, 1].float().cpu().numpy())
    assert np.array_equal(dst.k[1, 1, :20].cpu().numpy(), b.values(20).astype(np.float32))
    with pytest.raises(C.ConduitError):
        context.PackedContexts(1, 16, 1, 2, 1, D, bits=6)
