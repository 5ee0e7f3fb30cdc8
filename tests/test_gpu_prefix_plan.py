"""nacl_prefix_attention on both sides of the lines of its plan: rows per
work-group, chunks, waves and batches of the merge."""

import math

import pytest
import torch

nacl = pytest.importorskip("paper_2408_03675_amd.nacl")
from test_gpu_prefix import _make

pytestmark = pytest.mark.gpu


#        B  H  G  T  L  D  dtype  Lp
EMPTY = [
    (2, 2, 2, 1, 50, 128, "bf16", 0),      # one chunk in all: no merge
    (2, 2, 2, 1, 700, 128, "bf16", 0),     # several chunks
    (2, 2, 2, 1, 700, 64, "f32", 0),
    (3, 2, 4, 1, 40, 128, "bf16", 300),    # a prefix by 32 rows
    (3, 1, 4, 2, 40, 64, "f32", 300),
    (60, 1, 2, 1, 40, 128, "bf16", 600),   # a prefix by tiles of 128 rows
    (70, 1, 4, 1, 40, 64, "bf16", 600),    # of 256 rows
    (2, 1, 8, 20, 400, 128, "bf16", 0),    # own caches by tiles
    (1, 1, 64, 33, 1000, 64, "bf16", 0),   # more than 2048 rows
]


@pytest.mark.parametrize("case", EMPTY, ids=str)
def test_rows_without_weight_are_empty(case):
    """Every visible logit -infinity: zeros and a log-sum-exp of -infinity,
    whatever the visible values are and however the keys are shared out."""
    B, H, G, T, L, D, dtype, Lp = case
    q, k, v, kp, vp, _, _ = _make(B, H, G, T, L, D, dtype, 1, Lp)
    q.copy_(q.abs() + 0.5)
    k.fill_(float("-inf"))
    v[:, :, 1] = float("inf")
    v[:, :, L - 1, 3] = float("nan")
    if Lp:
        kp.fill_(float("-inf"))
        vp[:, :, Lp // 2] = float("nan")
        vp[:, :, 0, 5] = float("-inf")
    prob = nacl.Problem(B, H, L, D, dtype, [L - 1], q_group=G)
    step = nacl.Step(prob, T, row0=L - T)
    out, lse = nacl.prefix_attention(prob, step, q, k, v, prefix=nacl.Prefix(prob, kp, vp) if Lp else None)
    torch.cuda.synchronize()
    assert (out == 0).all() and (lse == -math.inf).all()
