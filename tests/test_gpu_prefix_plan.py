"""nacl_prefix_attention on both sides of the lines of its plan (rows per
work-group, waves and batches of the merge), padding in every size of block, rows
without any weight, and the accuracy of the few-row path's probabilities."""

import math

import numpy as np
import pytest
import torch

nacl = pytest.importorskip("paper_2408_03675_amd.nacl")
from test_gpu_prefix import DEV, _f64, _make, _rows, check_rows
from test_prefix_rules import excess

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


def _run(case, n_new=None, most=150):
    """A call with a workspace full of NaN against the definition."""
    B, H, G, T, L, D, dtype, groups, Lp = case
    q, k, v, kp, vp, lens, plens = _make(B, H, G, T, L, D, dtype, groups, Lp, seed=B + T)
    prob = nacl.Problem(B, H, L, D, dtype, [L - 1], q_group=G)
    new = None if n_new is None else torch.tensor(n_new, dtype=torch.int32, device=DEV)
    step = nacl.Step(prob, T, lens=lens.to(DEV), n_new=new)
    prefix = nacl.Prefix(prob, kp, vp, lens=plens.to(DEV)) if Lp else None
    ws = nacl.prefix_workspace(prob, step, prefix, DEV)
    ws.view(torch.float32).fill_(float("nan"))
    out, lse = nacl.prefix_attention(prob, step, q, k, v, prefix=prefix, ws=ws)
    torch.cuda.synchronize()
    rows = _rows(B, H * G, T, most)
    if n_new is not None:  # each sequence's last real tokens and first padding ones
        rows += [(b, h, t) for b in range(B) for h in (0, H * G - 1) for t in range(n_new[b] - 2, n_new[b] + 2) if 0 <= t < T]
    check_rows(q, k, v, kp, vp, lens, plens, out, lse, prob.c.sm_scale, rows, n_new=n_new)
    if n_new is not None:
        for b in range(B):
            assert (out[b, :, n_new[b]:] == 0).all() and (lse[b, :, n_new[b]:] == -math.inf).all()


#        B   H  G   T  L     D    dtype  groups Lp
MANY = [
    (64, 1, 40, 1, 20, 128, "bf16", 1, 10000),   # 2560 rows, 27 chunks of D = 128
    (63, 1, 33, 1, 600, 64, "bf16", 1, 10000),   # 2079 rows, more than 32 chunks of D = 64
    (1, 1, 64, 40, 8000, 64, "bf16", 1, 0),      # the same of an own cache
    (1, 1, 64, 40, 8000, 128, "bf16", 1, 0),
    (4, 1, 64, 9, 6000, 128, "f32", 1, 4000),
    (2, 1, 64, 16, 4000, 128, "bf16", 1, 0),     # exactly 2048 rows, 32 chunks
]


@pytest.mark.parametrize("case", MANY, ids=str)
def test_many_rows_of_many_chunks(case):
    _run(case, most=60)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("Lp", [0, 700])
@pytest.mark.parametrize("G,T,L", [(4, 50, 1000), (1, 300, 1000), (3, 12, 1000), (64, 3, 1000), (2, 5, 1000), (2, 5, 4000),
                                   (4, 6, 1000)])
def test_padding_in_every_block(G, T, L, Lp, D, dtype):
    """Sequences with none, one, some and all of the step's tokens, in blocks of
    16 to 256 rows and several chunks, joined by one wave a row and by four."""
    _run((5, 1, G, T, L, D, dtype, 1, Lp), n_new=[T, 0, 1, T // 2 + 1, T - 1], most=60)


@pytest.mark.parametrize("n", [15, 16, 17, 31, 32, 33, 127, 128, 129, 255, 256, 257])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_at_the_plan_s_lines(n, dtype):
    """n rows of one sequence over its cache and of one group over its prefix."""
    _run((1, 2, 1, n, n + 400, 64, dtype, 1, 0), most=80)
    _run((n, 1, 1, 1, 150, 128, dtype, 1, 333), most=80)
    _run((2, 1, 1, n, n + 40, 128, dtype, 2, 333), most=80)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,G,L,Lp", [(4, 2, 12, 0), (3, 16, 24, 0), (4, 4, 9, 14), (2, 16, 9, 30)])
def test_few_rows_keep_their_probabilities(B, G, L, Lp, D):
    """Up to 32 rows per key: the probabilities are two bf16, of which 2^-17 is
    lost (the rounding of what a first rounding by half a step, 2^-8, leaves).
    Small logits and few keys, so that a single bf16's loss would stand out."""
    H = 2
    q, k, v, kp, vp, _, _ = _make(B, H, G, 1, L, D, "bf16", 1, Lp, scale=0.25)
    prob = nacl.Problem(B, H, L, D, "bf16", [L - 1], q_group=G)
    prefix = nacl.Prefix(prob, kp, vp) if Lp else None
    out, lse = nacl.prefix_attention(prob, nacl.Step(prob, 1, row0=L - 1), q, k, v, prefix=prefix)
    torch.cuda.synchronize()
    for b in range(B):
        for hq in range(H * G):
            kk, vv = _f64(k[b, hq // G]), _f64(v[b, hq // G])
            if Lp:
                kk, vv = np.concatenate((_f64(kp[0, hq // G]), kk)), np.concatenate((_f64(vp[0, hq // G]), vv))
            assert excess(_f64(out[b, hq, 0]), _f64(q[b, hq, 0]), kk, vv, prob.c.sm_scale, 2.0 ** -17) <= 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B", [2, 20, 90])
def test_prefix_lengths_are_clamped(B, dtype):
    """Lengths below 0 count as 0, past the buffers as all of their rows."""
    H, G, T, L, D, Lp = 1, 2, 2, 30, 64, 210
    q, k, v, kp, vp, lens, _ = _make(B, H, G, T, L, D, dtype, 2, Lp)
    prob = nacl.Problem(B, H, L, D, dtype, [L - 1], q_group=G)
    given = torch.tensor([-5, Lp + 1000], dtype=torch.int32, device=DEV)
    out, lse = nacl.prefix_attention(prob, nacl.Step(prob, T, lens=lens.to(DEV)), q, k, v, prefix=nacl.Prefix(prob, kp, vp, lens=given))
    torch.cuda.synchronize()
    check_rows(q, k, v, kp, vp, lens, torch.tensor([0, Lp]), out, lse, prob.c.sm_scale, _rows(B, H * G, T))
