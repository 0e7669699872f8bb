"""Beam selection and reordering at the ends of their ranges."""

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
INF = float("inf")


@pytest.fixture(scope="module")
def C():
    from paper_2609_05821_gb300 import _build
    _build.build()
    from paper_2609_05821_gb300 import conduit
    return conduit


@pytest.mark.parametrize("vocab", [2 ** 31 - 1, 2 ** 31 - 8, 2 ** 31 - 25])
def test_select_over_the_longest_rows(C, vocab):
    """A row whose last indexes and one load more pass 2^31. All but four logits are -inf, so that the scores are
    z - ln(sum of four exponentials), whose sum and logarithm are off by a few 2^-24."""
    z = torch.full((1, vocab), -INF, dtype=BF, device="cuda")
    at = {vocab - 1: 1.5, 0: 1.0, vocab // 2: 0.5, vocab - 9: -2.0}
    for i, x in at.items():
        z[0, i] = x
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    score, parent, token = C.conduit_beam_select(z, torch.full((1,), -1.0, device="cuda"), 1, 6, status=status)
    assert C.conduit_read_status(status) == C.OK
    lse = np.log(sum(np.exp(x) for x in at.values()))
    assert token[0].tolist() == list(at) + [0, 0] and parent[0].tolist() == [0] * 6
    want = np.array([x - lse - 1.0 for x in at.values()])
    assert np.all(np.abs(score[0, :4].double().cpu().numpy() - want) <= 8 * 2.0 ** -24 * np.abs(want) + 8 * 2.0 ** -24)
    assert score[0, 4:].tolist() == [-INF] * 2


def _check_sums(C, z, width):
    """The best score of every beam of one group shape against 64 bits: a log-sum-exp within (21 + ln vocab) 2^-22, the score
    rounded to fp32."""
    n, vocab = z.shape
    sums = torch.zeros(n, device="cuda")
    top = z.double().amax(-1)
    want = torch.cat([-(row.double() - m).exp().sum().log()[None] for row, m in zip(z[:width], top)])
    for b in range(width):  # each beam of the first group alone is chosen from
        only = torch.full((n,), -INF, device="cuda")
        only[b::width] = sums[b::width]
        score, parent, token = C.conduit_beam_select(z, only, width, 1)
        assert torch.equal(score, score[:1].expand_as(score)) and parent[0, 0] == b
        tol = (21 + np.log(vocab)) * 2.0 ** -22 + 2.0 ** -24 * abs(float(want[b]))
        assert abs(float(score[0, 0]) - float(want[b])) <= tol, (b, float(score[0, 0]) - float(want[b]), tol)


@pytest.mark.parametrize("dtype", [F32, BF])
@pytest.mark.parametrize("width,vocab", [(32, 200000), (20, 128000), (1, 3000000)])
def test_select_adds_up_long_rows(C, dtype, width, vocab):
    """Rows whose sum is a peak and a flat level far below it, which every lane adds up one load after another; rows that rise
    or fall slowly from end to end; one segment a row (more than 38 groups of more than 16 beams) and many."""
    groups = 40 if width > 1 else 2
    rows = []
    per = 32 * 16 // torch.empty((), dtype=dtype).element_size()  # one load of a warp's lanes
    for level in (-6.3, -8.0, -9.7, -11.1, -13.0):
        z = torch.full((vocab,), level, device="cuda")
        z[:per] = 0.0
        rows.append(z)
    up = torch.arange(vocab, device="cuda", dtype=torch.float64)
    for span in (2.0, 12.0, 40.0):
        rows += [(up * (span / vocab)).float(), (up.flip(0) * (span / vocab)).float()]
    rows = torch.stack([rows[i % len(rows)] for i in range(min(width, len(rows)))] * (-(-width // len(rows))))[:width].to(dtype)
    _check_sums(C, rows.repeat(groups, 1), width)


@pytest.mark.parametrize("dtype,groups,width,vocab,n,pad", [(F32, 39, 17, 5003, 32, 0), (BF, 77, 32, 2500, 32, 6),
                                                            (BF, 41, 24, 9001, 5, 7), (F32, 160, 31, 333, 31, 2)])
def test_select_with_one_segment_a_row(C, dtype, groups, width, vocab, n, pad):
    """More beams than half of a cluster's warps: a row is one warp's."""
    from tests.test_gpu_beam import _check_select
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    z = 3 * torch.randn((groups * width, vocab + pad), generator=gen, device="cuda")
    z[:, vocab:] = 1e4
    sums = -5 * torch.rand(groups * width, generator=gen, device="cuda")
    _check_select(C, z.to(dtype)[:, :vocab], sums, width, n)


def test_equal_rows_come_in_their_order(C):
    """Odd vocabularies whose rows begin at multiples of 16 bytes: equal rows have equal scores to the last bit."""
    for dtype, vocab, stride in ((BF, 50021, 50024), (F32, 30001, 30004)):
        row = 3 * torch.randn(vocab, generator=torch.Generator().manual_seed(5)).cuda()
        z = torch.zeros((8, stride), device="cuda", dtype=dtype)[:, :vocab]
        z[:] = row.to(dtype)
        score, parent, token = C.conduit_beam_select(z, torch.full((8,), -1.5, device="cuda"), 8, 8)
        assert parent[0].tolist() == list(range(8)) and len(set(token[0].tolist())) == 1 and len(set(score[0].tolist())) == 1


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("L,hkv,d,ps,G,width,lens", [
    (2, 3, 8, 5, 3, 3, (13, 0, 99)),
    (1, 1, 8, 1, 2, 4, (7, 1)),
    (3, 2, 24, 12, 2, 17, (1, 47)),
    (1, 5, 40, 100, 4, 2, (99, 100, 101, 3)),
])
def test_reorder_over_odd_heads_and_pages(C, kind, L, hkv, d, ps, G, width, lens):
    """Heads of 8 dims, whose rows are 16 bytes, and pages of any number of tokens."""
    from tests import test_gpu_beam
    test_gpu_beam.test_reorder(C, kind, L, hkv, d, ps, G, width, lens)
