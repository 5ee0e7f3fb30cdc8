"""nacl_beam_select where values are equal: the lowest beam and token are taken."""

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
