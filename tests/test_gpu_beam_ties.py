"""nacl_beam_select where values are equal: the lowest beam is taken, of it the largest
logits, of equal ones the lowest tokens."""

import math

import pytest
import torch

nacl = pytest.importorskip("paper_2408_03675_amd.nacl")
from test_gpu_paged import DEV, DT

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K", [1, 2, 3])
@pytest.mark.parametrize("kind", ["ended", "one token", "infinite"])
def test_zero_scores_of_both_signs_are_equal(kind, K, dtype):
    """Values of 0 by beams whose scores are -0 and 0, in both orders: an ended
    beam's, a certain token's, an infinite logit's."""
    V = 1 if kind == "one token" else 300
    scores = torch.tensor([[-0.0, 0.0, -0.0], [0.0, -0.0, 0.0]], device=DEV)
    logits = torch.zeros((6, V), dtype=DT[dtype], device=DEV)
    kw = {}
    if kind == "ended":
        kw = dict(ended=torch.ones((2, 3), dtype=torch.int32, device=DEV), end_token=17)
    elif kind == "infinite":
        logits[:, 17] = math.inf
    parents, tokens, out = nacl.beam_select(logits, scores, K, **kw)
    token = 0 if kind == "one token" else 17
    assert parents.tolist() == [list(range(K))] * 2 and tokens.tolist() == [[token] * K] * 2
    assert (out == 0).all()


def _by_logit(row, K):
    """A beam's K first tokens: the largest logits first, equal ones by token."""
    return torch.sort(row.double().cpu(), descending=True, stable=True).indices[:K].tolist()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("score", [-1e30, torch.finfo(torch.float32).min, 1e30, -1e15, -3.0])
@pytest.mark.parametrize("V", [7, 9000, 30000, 70001])
def test_a_beam_s_order_is_that_of_its_logits(V, score, dtype):
    """Also where the differences vanish beside the score, so that the values are equal."""
    g = torch.Generator().manual_seed(V)
    for spread in (2.0, 1e-20):
        logits = (spread * torch.randn((1, V), generator=g)).to(DT[dtype]).to(DEV)
        scores = torch.tensor([[score]], device=DEV)
        for K in (1, 4, 33, 64):
            parents, tokens, out = nacl.beam_select(logits, scores, K)
            n, pad = min(K, V), max(0, K - V)
            assert tokens[0].tolist() == _by_logit(logits[0], K) + [-1] * pad
            assert parents[0].tolist() == [0] * n + [-1] * pad
            if abs(score) >= 1e15:
                assert (out[0, :n] == scores[0, 0]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("W,V,K", [(2, 9000, 64), (4, 5, 12), (8, 30000, 16), (8, 30000, 64), (33, 20000, 1), (64, 40000, 64),
                                   (64, 131000, 50)])
def test_equal_values_of_many_beams(W, V, K, dtype):
    """The first beam's continuations by their logits, then the next one's: scores beside
    which every difference vanishes, and logits whose differences vanish beside scores of
    ordinary size."""
    g = torch.Generator().manual_seed(W)
    for spread, score in ((2.0, -1e30), (1e-20, -20.0)):
        logits = (spread * torch.randn((W, V), generator=g)).to(DT[dtype]).to(DEV)
        parents, tokens, _ = nacl.beam_select(logits, torch.full((1, W), score, device=DEV), K)
        want = [(w, t) for w in range(-(-K // V)) for t in _by_logit(logits[w], V)][:K]
        assert list(zip(parents[0].tolist(), tokens[0].tolist())) == want
