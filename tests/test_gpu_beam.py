"""nacl_beam_select against the float64 continuations of every group, and
nacl_beam_reorder against its reference."""

import math

import numpy as np
import pytest
import torch

nacl = pytest.importorskip("paper_2408_03675_amd.nacl")
from oracle.paged import beam_values, best, take_over
from test_gpu_paged import DEV, DT, _i32, _pool

pytestmark = pytest.mark.gpu


def _check(logits, scores, K, got, ended=None, end_token=0):
    """Every chosen continuation is a group's, once, with its value, and in an order
    that values within the arithmetic's error of each other explain; where no two
    are that close, the reference's."""
    B, W = scores.shape
    x = logits.detach().double().cpu().numpy().reshape(B, W, -1)
    parents, tokens, out = (t.cpu().numpy() for t in got)
    for b in range(B):
        made = [beam_values(x[b, w], float(scores[b, w]), bool(ended is not None and ended[b, w]), end_token) for w in range(W)]
        values, err = np.stack([m[0] for m in made]), max(m[1] for m in made)
        rp, rt, rv = best(values, K + 1)
        at = [(int(p), int(t)) for p, t in zip(parents[b], tokens[b])]
        n = int((np.array(rv[:K]) > -math.inf).sum())
        assert all(a == (-1, -1) for a in at[n:]) and (out[b, n:] == -math.inf).all()
        assert len(set(at[:n])) == n
        for i in range(n):
            mine = values[at[i]]
            assert abs(mine - rv[i]) <= 2 * err, (b, i, at[i], mine, rv[i])
            if abs(mine) >= 2.0 ** 128:  # rounds to an infinity of fp32, whose largest number is below 2^128
                assert out[b, i] == math.copysign(math.inf, mine)
                continue
            assert abs(out[b, i] - mine) <= err + 2.0 ** -24 * abs(mine) + 1e-45, (b, i, out[b, i], mine)
        # Of one beam the order is that of the logits, exactly; equal ones by token.
        for i in range(n - 1):
            if at[i][0] == at[i + 1][0]:
                a, c = values[at[i]], values[at[i + 1]]
                assert a > c or (a == c and at[i][1] < at[i + 1][1])
        close = any(rv[i] != rv[i + 1] and rv[i] - rv[i + 1] <= 2 * err for i in range(n) if rv[i + 1] > -math.inf)
        if not close:
            assert at[:n] == list(zip(rp[:n], rt[:n])), b


def _make(B, W, V, dtype, seed=0, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    x = spread * torch.randn((B * W, V), generator=g)
    scores = -20 - 3 * torch.rand((B, W), generator=g)
    return x.to(DT[dtype]).to(DEV), scores.to(DEV)


CASES = [
    (1, 1, 1, 1), (1, 1, 1, 5), (2, 3, 2, 64), (1, 4, 32000, 4), (3, 5, 1000, 10), (2, 8, 8192, 16), (2, 8, 8193, 16),
    (1, 2, 131072, 64), (4, 1, 50257, 1), (1, 32, 40001, 64), (2, 64, 300, 64), (1, 64, 131000, 20), (1, 1, 1 << 20, 33),
    (9, 3, 7, 21), (1, 33, 200000, 64),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,W,V,K", CASES)
def test_select(B, W, V, K, dtype):
    logits, scores = _make(B, W, V, dtype, seed=V)
    _check(logits, scores, K, nacl.beam_select(logits, scores, K))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_select_ended_and_dead_beams(dtype):
    logits, scores = _make(6, 4, 9000, dtype)
    ended = torch.zeros((6, 4), dtype=torch.int32)
    ended[0, 1] = ended[1] = ended[2, 3] = 7
    scores[2, 3], scores[3, 1:], scores[4] = -math.inf, -math.inf, math.nan
    scores[5, 0], scores[5, 1] = math.inf, -1e30
    logits[0 * 4 + 1] = math.nan  # of a beam that has ended, not read
    got = nacl.beam_select(logits, scores, 8, ended=ended.to(DEV), end_token=8999)
    _check(logits, scores.cpu(), 8, got, ended, 8999)
    assert (got[0][3].cpu() == 0).all() and (got[0][4].cpu() == -1).all()
    assert got[0][1].cpu().tolist()[4:] == [-1] * 4 and set(got[0][1].cpu().tolist()[:4]) == {0, 1, 2, 3}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [100, 20000])
def test_select_odd_logits(dtype, V):
    """NaN, infinities, the type's lowest value, rows without a logit, zeros of both
    signs, all equal."""
    low = torch.finfo(DT[dtype]).min
    logits, scores = _make(1, 12, V, dtype, seed=1)
    logits[0, ::2] = math.nan
    logits[1] = -math.inf
    logits[2] = math.nan
    logits[3, [5, V - 1, 17]] = math.inf
    logits[4, :-2] = -math.inf
    logits[5] = low
    logits[6] = 0.0
    logits[6, 1::2] = -0.0
    logits[7], logits[7, 3] = low, torch.finfo(DT[dtype]).max
    logits[8, 1:] = -math.inf
    logits[9] = logits[10]
    scores[0, 9] = scores[0, 10]
    for w in range(12):
        one = logits[w:w + 1].contiguous()
        _check(one, scores[:, w:w + 1], 20, nacl.beam_select(one, scores[:, w:w + 1].contiguous(), 20))
    _check(logits, scores, 64, nacl.beam_select(logits, scores, 64))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("W,V,K", [(1, 30000, 64), (8, 30000, 64), (32, 30000, 64), (64, 20000, 3)])
def test_select_ties(dtype, W, V, K):
    """Equal logits and equal beams go to the lowest beam and token, exactly: all
    equal, few values, a run of equal ones in few threads, the same row in every
    beam."""
    g = torch.Generator().manual_seed(W)
    scores = torch.full((1, W), -3.0, device=DEV)
    rows = [torch.zeros(V), torch.randint(0, 3, (V,), generator=g).float(), torch.arange(V) / 7.0, -torch.arange(V) / 7.0,
            torch.where(torch.arange(V) // 100 == 151, 9.0, torch.randn(V, generator=g))]
    for row in rows:
        x = row.to(DT[dtype])
        logits = x.expand(W, V).contiguous().to(DEV)
        parents, tokens, out = nacl.beam_select(logits, scores, K)
        rp, rt, _ = best(np.broadcast_to(x.double().numpy(), (W, V)), K)
        assert parents[0].tolist() == rp and tokens[0].tolist() == rt
        _check(logits, scores, K, (parents, tokens, out))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_select_from_strided_rows(dtype):
    """Rows that start at any element, by a row stride and from the middle of a
    buffer whose ends hold larger numbers; results that the row alone decides."""
    B, W, V, K = 2, 3, 16384, 12
    logits, scores = _make(B, W, V, dtype)
    want = nacl.beam_select(logits, scores, K)
    _check(logits, scores, K, want)
    for lead, gap in ((1, 0), (3, 1), (7, 9), (0, 5), (8, 8)):
        wide = torch.full((B * W * (V + gap) + lead + 16,), 1e4, dtype=DT[dtype], device=DEV)
        rows = wide[lead:lead + B * W * (V + gap)].view(B * W, V + gap)[:, :V]
        rows.copy_(logits)
        for x, y in zip(nacl.beam_select(rows, scores, K), want):
            assert torch.equal(x, y)


def test_select_again_and_in_halves():
    """The same call gives the same bits, and a group's result does not depend on the
    others."""
    logits, scores = _make(40, 5, 70001, "f32")
    a, b = nacl.beam_select(logits, scores, 10), nacl.beam_select(logits, scores, 10)
    half = nacl.beam_select(logits[75:].clone(), scores[15:].contiguous(), 10)
    for x, y, z in zip(a, b, half):
        assert torch.equal(x, y) and torch.equal(x[15:], z)


# --------------------------------------------------------------------------
# Reordering

@pytest.mark.parametrize("layout", ["heads", "rows", "one", "side"])
@pytest.mark.parametrize("groups,W,H,D,page,entries,dtype", [
    (1, 1, 1, 64, 16, 1, "bf16"), (1, 4, 8, 128, 16, 9, "bf16"), (3, 5, 2, 64, 7, 6, "f32"), (2, 64, 1, 64, 3, 4, "bf16"),
    (5, 8, 3, 128, 33, 3, "f32"), (1, 2, 2, 128, 1000, 2, "bf16"),
])
def test_reorder(layout, groups, W, H, D, page, entries, dtype):
    g = torch.Generator().manual_seed(W + page)
    B, own = groups * W, entries
    shared = 2
    n = groups * shared + B * own + 1
    k, v = _pool(g, n, H, page, D, dtype, layout)
    perm = torch.randperm(n, generator=g)
    table = torch.cat((perm[:groups * shared].view(groups, 1, shared).expand(groups, W, shared).reshape(B, shared),
                       perm[groups * shared:groups * shared + B * own].view(B, own)), dim=1).int()
    L = (shared + own) * page
    for trial in range(3):
        parents = torch.randint(0, W, (groups, W), generator=g, dtype=torch.int32)
        if trial == 1:
            parents[:] = torch.arange(W)  # nothing to copy
        if trial == 2:
            parents[0, 0], parents[-1, -1] = -1, W
        lens = torch.randint(0, L + 1, (B,), generator=g, dtype=torch.int32)
        lens[0] = L + 5
        held = torch.randint(0, shared + own + 1, (B,), generator=g, dtype=torch.int32) if trial != 1 else None
        table0 = table.clone()
        if trial == 2:
            table0[:, -1] = -1
        want_k, want_v = k.clone(), v.clone()
        want = [], [], []
        for i in range(groups):
            s = slice(i * W, i * W + W)
            plan = take_over(parents[i].tolist(), lens[s].tolist(), None if held is None else held[s].tolist(), shared + own, page, L)
            for w, (takes, length, rows) in enumerate(plan):
                want[0].append(table0[i * W + takes].tolist())
                want[1].append(length)
                want[2].append(None if held is None else int(held[i * W + takes]))
                for j in range(rows):
                    to, of = (int(table0[i * W + x, j // page]) for x in (takes, int(parents[i, w])))
                    if to != of and 0 <= to < n and 0 <= of < n:
                        want_k[to, :, j % page], want_v[to, :, j % page] = k[of, :, j % page], v[of, :, j % page]
        prob = nacl.Problem(B, H, L, D, dtype, [0])
        out = torch.full((B, shared + own + 2), -5, dtype=torch.int32, device=DEV)
        got = nacl.beam_reorder(prob, nacl.Pages(prob, k, v, table0.to(DEV)), parents.to(DEV), lens.to(DEV),
                                None if held is None else held.to(DEV), table_out=out[:, :shared + own])
        torch.cuda.synchronize()
        assert got[0].tolist() == want[0] and got[1].tolist() == want[1]
        assert got[2] is None if held is None else got[2].tolist() == want[2]
        assert (out[:, shared + own:] == -5).all()
        assert torch.equal(k, want_k) and torch.equal(v, want_v)
