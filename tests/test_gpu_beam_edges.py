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
