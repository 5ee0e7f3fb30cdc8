"""nacl_prefix_attention against the float64 attention of each row: single
tokens and chunks, ragged and empty lengths, groups that share a prefix,
strides, hidden rows that hold anything, captured graphs."""

import math

import numpy as np
import pytest
import torch

nacl = pytest.importorskip("paper_2408_03675_amd.nacl")
from oracle.step import attend_row

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _f64(t):
    return t.detach().cpu().double().numpy()


def _lens(g, n, hi):
    t = torch.randint(0, hi + 1, (n,), generator=g, dtype=torch.int32)
    t[0] = hi
    if n > 1:
        t[1] = 0
    return t


def _make(B, H, G, T, L, D, dtype, groups, Lp, seed=0, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    dt = DT[dtype]
    r = lambda *s: torch.randn(s, generator=g).to(dt).to(DEV)
    q = (scale * torch.randn((B, H * G, T, D), generator=g)).to(dt).to(DEV)
    k, v = r(B, H, L, D), r(B, H, L, D)
    kp, vp = (r(groups, H, Lp, D), r(groups, H, Lp, D)) if Lp else (None, None)
    return q, k, v, kp, vp, _lens(g, B, L - T), _lens(g, groups, Lp)


def check_rows(q, k, v, kp, vp, lens, plens, out, lse, sm_scale, rows, row0=0, n_new=None):
    """Rows (b, hq, t) against the definition.  Tolerances, with u half a step
    of bf16 (0 for fp32): fp32 products of D terms and sums of n keys in any
    order put each logit off by at most gamma = (D + 8) 2^-24 S (S the largest
    scaled sum of |q||k|), each weight by the same relatively, doubled through
    the normalisation; the exponentials and n sums add (n + 64) 2^-24; the
    probabilities are rounded to bf16 (u), the output once (half a step of it)."""
    B, Hq, T, D = q.shape
    H, L = k.shape[1], k.shape[2]
    bf16 = q.dtype == torch.bfloat16
    u = torch.finfo(torch.bfloat16).eps / 2 if bf16 else 0.0
    half = torch.finfo(q.dtype).eps / 2
    per = B // kp.shape[0] if kp is not None else B
    got_o, got_l = _f64(out), _f64(lse)
    for b, hq, t in rows:
        h = hq // (Hq // H)
        real = n_new is None or t < n_new[b]
        n = min(L, max(0, row0 + int(lens[b]) + t + 1)) if real else 0
        kk, vv = _f64(k[b, h, :n]), _f64(v[b, h, :n])
        if kp is not None and real:
            m = int(plens[b // per])
            kk = np.concatenate((_f64(kp[b // per, h, :m]), kk))
            vv = np.concatenate((_f64(vp[b // per, h, :m]), vv))
        ref, ref_l, size, S = attend_row(_f64(q[b, hq, t]), kk, vv, sm_scale)
        o, l = got_o[b, hq, t], got_l[b, hq, t]
        if ref_l == -math.inf:
            assert l == -math.inf and (o == 0).all(), (b, hq, t)
            continue
        gamma = (D + 8) * 2.0 ** -24 * S + (len(kk) + 64) * 2.0 ** -24
        tol = half * np.abs(ref) + (u + 2 * gamma) * 1.01 * size
        assert (np.abs(o - ref) <= tol).all(), ((b, hq, t), np.abs(o - ref).max(), tol.min())
        assert abs(l - ref_l) <= gamma + 2.0 ** -23 * abs(ref_l) + 2.0 ** -22, ((b, hq, t), l, ref_l)


def _rows(B, Hq, T, most=200, seed=5):
    every = [(b, h, t) for b in range(B) for h in range(Hq) for t in range(T)]
    if len(every) <= most:
        return every
    pick = np.random.default_rng(seed).choice(len(every), most - 2, replace=False)
    return [every[0], every[-1]] + [every[i] for i in pick]


#        B  H  G  T   L     D   dtype  groups Lp
CASES = [
    (1, 1, 1, 1, 1, 128, "bf16", 1, 0),
    (1, 1, 1, 1, 1, 64, "f32", 1, 1),
    (1, 8, 4, 1, 2112, 128, "bf16", 1, 0),
    (3, 2, 1, 1, 129, 64, "bf16", 1, 31),
    (4, 2, 2, 1, 40, 128, "bf16", 2, 700),
    (5, 2, 7, 1, 333, 128, "bf16", 1, 1025),
    (6, 4, 2, 5, 333, 64, "f32", 3, 1999),
    (2, 1, 8, 3, 100, 128, "f32", 2, 65),
    (33, 1, 8, 1, 70, 128, "bf16", 1, 513),
    (12, 2, 4, 2, 50, 64, "bf16", 4, 257),
    (2, 2, 4, 65, 200, 128, "bf16", 1, 300),
    (1, 3, 1, 130, 130, 64, "bf16", 1, 0),
    (70, 1, 2, 1, 33, 128, "f32", 1, 150),
    (1, 2, 64, 1, 300, 128, "bf16", 1, 90),
    (1, 1, 2, 2, 20000, 128, "bf16", 1, 70000),
    (130, 2, 4, 1, 20, 128, "bf16", 1, 2000),
    (64, 1, 2, 2, 20, 64, "bf16", 2, 1111),
]


@pytest.mark.parametrize("case", CASES, ids=str)
def test_rows(case):
    B, H, G, T, L, D, dtype, groups, Lp = case
    q, k, v, kp, vp, lens, plens = _make(*case)
    prob = nacl.Problem(B, H, L, D, dtype, [L - 1], q_group=G)
    step = nacl.Step(prob, T, lens=lens.to(DEV))
    prefix = nacl.Prefix(prob, kp, vp, lens=plens.to(DEV)) if Lp else None
    out, lse = nacl.prefix_attention(prob, step, q, k, v, prefix=prefix)
    torch.cuda.synchronize()
    check_rows(q, k, v, kp, vp, lens, plens, out, lse, prob.c.sm_scale, _rows(B, H * G, T))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("groups,Lp", [(1, 0), (2, 300)])
def test_hidden_rows_may_hold_anything(dtype, groups, Lp):
    """Rows past the lengths, later tokens of the step, padding and a row's
    neighbours with NaN and infinities; lengths below 0 and past the end; a
    strided cache, queries and prefix; row0."""
    B, H, G, T, L, D = 4, 2, 3, 4, 90, 128
    q, _, _, _, _, _, _ = _make(B, H, G, T, L, D, dtype, groups, 0, seed=1)
    dt = DT[dtype]
    g = torch.Generator().manual_seed(2)
    q = q.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)  # [B, T, Hq, D] in memory
    k, v = (torch.randn((B, L, H, D), generator=g).to(dt).to(DEV).permute(0, 2, 1, 3) for _ in range(2))
    lens = torch.tensor([40, -200, 1000, 7], dtype=torch.int32)
    n_new = torch.tensor([4, 4, 4, 2], dtype=torch.int32)
    k[0, :, 40 + 5 + T:] = float("nan")
    v[0, :, 40 + 5 + T:] = float("inf")
    k[0, :, 40 + 5 + 2] = float("nan")  # tokens 2 and 3 see it, 0 and 1 do not
    v[0, :, 40 + 5 + 3] = float("inf")
    k[1], v[1] = float("nan"), float("nan")  # nothing of it is seen
    v[3, :, 7 + 5 + 2:] = float("nan")
    kp = vp = plens = None
    if Lp:
        kp, vp = (torch.randn((groups, Lp, H, D), generator=g).to(dt).to(DEV).permute(0, 2, 1, 3) for _ in range(2))
        plens = torch.tensor([Lp - 33, 0], dtype=torch.int32)
        kp[0, :, Lp - 33:], vp[1] = float("nan"), float("nan")
    prob = nacl.Problem(B, H, L, D, dtype, [L - 1], q_group=G, sm_scale=0.2, k_stride=k.stride()[:3], v_stride=v.stride()[:3])
    step = nacl.Step(prob, T, lens=lens.to(DEV), row0=5, n_new=n_new.to(DEV))
    prefix = nacl.Prefix(prob, kp, vp, lens=plens.to(DEV)) if Lp else None
    out, lse = nacl.prefix_attention(prob, step, q, k, v, prefix=prefix)
    torch.cuda.synchronize()
    odd = {(0, hq, t) for hq in range(H * G) for t in (2, 3)}
    rows = [x for x in _rows(B, H * G, T) if x not in odd]
    check_rows(q, k, v, kp, vp, lens, plens, out, lse, 0.2, rows, row0=5, n_new=n_new.tolist())
    for x in odd:
        assert torch.isnan(lse[x]) and torch.isnan(out[x]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_logits(dtype):
    """Keys whose logits are -infinity weigh nothing; a row that sees only such
    keys is an empty one; +infinity gives NaN, as the softmax does."""
    B, H, G, T, L, D = 2, 1, 1, 1, 50, 64
    q, k, v, _, _, _, _ = _make(B, H, G, T, L, D, dtype, 1, 0)
    q[...] = q.abs() + 0.5
    q[1] *= -1
    k[0, 0, :25] = float("-inf")
    k[1] = float("inf")
    lens = torch.tensor([40, 40], dtype=torch.int32)
    prob = nacl.Problem(B, H, L, D, dtype, [L - 1])
    step = nacl.Step(prob, T, lens=lens.to(DEV))
    out, lse = nacl.prefix_attention(prob, step, q, k, v)
    sub_k, sub_v = k.clone(), v.clone()
    sub_k[0, 0, :16], sub_v[0, 0, :16] = k[0, 0, 25:41], v[0, 0, 25:41]
    part = torch.tensor([15, 40], dtype=torch.int32)
    check_rows(q, sub_k, sub_v, None, None, part, None, out, lse, prob.c.sm_scale, [(0, 0, 0)])
    assert lse[1, 0, 0] == -math.inf and (out[1, 0, 0] == 0).all()
    q[1] *= -1
    out, lse = nacl.prefix_attention(prob, step, q, k, v)
    assert torch.isnan(out[1, 0, 0]).all()


def test_large_logits():
    """Logits of thousands: one key takes all the weight."""
    B, H, G, T, L, D = 3, 2, 4, 1, 500, 128
    q, k, v, kp, vp, lens, plens = _make(B, H, G, T, L, D, "bf16", 1, 900, scale=300.0)
    prob = nacl.Problem(B, H, L, D, "bf16", [L - 1], q_group=G)
    prefix = nacl.Prefix(prob, kp, vp, lens=plens.to(DEV))
    out, lse = nacl.prefix_attention(prob, nacl.Step(prob, T, lens=lens.to(DEV)), q, k, v, prefix=prefix)
    check_rows(q, k, v, kp, vp, lens, plens, out, lse, prob.c.sm_scale, _rows(B, H * G, T))


def test_same_results_and_nothing_else_written():
    """Two calls agree bit for bit, on another stream too; memory behind the
    outputs and the workspace stays as it was."""
    B, H, G, T, L, D = 5, 2, 4, 2, 600, 128
    q, k, v, kp, vp, lens, plens = _make(B, H, G, T, L, D, "bf16", 1, 1500)
    prob = nacl.Problem(B, H, L, D, "bf16", [L - 1], q_group=G)
    step = nacl.Step(prob, T, lens=lens.to(DEV))
    prefix = nacl.Prefix(prob, kp, vp, lens=plens.to(DEV))
    need = nacl.prefix_workspace(prob, step, prefix, DEV).numel()
    ws = torch.full((need + 4096,), 77, dtype=torch.uint8, device=DEV)
    n = B * H * G * T
    obuf = torch.full((n * D + 512,), 7.0, dtype=torch.bfloat16, device=DEV)
    lbuf = torch.full((n + 512,), 7.0, dtype=torch.float32, device=DEV)
    out, lse = obuf[:n * D].view(B, H * G, T, D), lbuf[:n].view(B, H * G, T)
    nacl.prefix_attention(prob, step, q, k, v, prefix=prefix, out=out, lse=lse, ws=ws[:need])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        again, lse2 = nacl.prefix_attention(prob, step, q, k, v, prefix=prefix)
    torch.cuda.synchronize()
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    assert (obuf[n * D:] == 7).all() and (lbuf[n:] == 7).all() and (ws[need:] == 77).all()
    only, none = nacl.prefix_attention(prob, step, q, k, v, prefix=prefix, lse=False)
    assert none is None and torch.equal(only, out)


def test_two_graphs_replay_in_turn():
    """Two captured calls, each with its own workspace, replay in any order and
    follow the lengths."""
    D, G, H = 128, 4, 2
    made = []
    for B, L, Lp in ((3, 300, 700), (2, 50, 0)):
        q, k, v, kp, vp, lens, plens = _make(B, H, G, 1, L, D, "bf16", 1, Lp, seed=B)
        prob = nacl.Problem(B, H, L, D, "bf16", [L - 1], q_group=G)
        lens = (lens // 2).to(DEV)
        step = nacl.Step(prob, 1, lens=lens)
        prefix = nacl.Prefix(prob, kp, vp) if Lp else None
        ws = nacl.prefix_workspace(prob, step, prefix, DEV)
        out, lse = nacl.prefix_attention(prob, step, q, k, v, prefix=prefix, ws=ws)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            nacl.prefix_attention(prob, step, q, k, v, prefix=prefix, out=out, lse=lse, ws=ws)
        made.append((graph, prob, step, prefix, q, k, v, lens, out, lse))
    for i in (0, 1, 1, 0, 1, 0):
        graph, prob, step, prefix, q, k, v, lens, out, lse = made[i]
        lens += 1
        graph.replay()
        want, want_l = nacl.prefix_attention(prob, step, q, k, v, prefix=prefix)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_l)


def test_log_sum_exp_feeds_the_score():
    """The current token's log-sum-exp over prefix and cache is nacl_score's lse
    for a generation-phase round."""
    B, H, G, L, D, Lp = 2, 2, 4, 700, 128, 333
    q, k, v, kp, vp, _, plens = _make(B, H, G, 1, L, D, "bf16", 1, Lp)
    qs = q.stride()
    prob = nacl.Problem(B, H, L, D, "bf16", [L - 1], q_group=G, q_stride=(qs[0], qs[1], 0))
    step = nacl.Step(prob, 1, row0=L - 1)
    prefix = nacl.Prefix(prob, kp, vp)
    _, lse = nacl.prefix_attention(prob, step, q, k, v, prefix=prefix)
    F = nacl.score(prob, q.expand(B, H * G, L, D), k, nacl.workspace(prob, DEV), lse=lse)
    a = (q.double().view(B, H, G, D) @ k.double().transpose(2, 3).contiguous()) * prob.c.sm_scale
    b = (q.double().view(B, H, G, D) @ kp[0].double().transpose(1, 2).contiguous()) * prob.c.sm_scale
    z = torch.logsumexp(torch.cat((a, b), dim=3), dim=3, keepdim=True)
    ref = (a - z).exp().sum(dim=2)
    assert ((F.double() - ref).abs() <= 1e-3 * ref + 1e-30).all()


@pytest.mark.parametrize("G,T,B,Lp", [(2, 12, 2, 0), (8, 9, 2, 300), (1, 150, 1, 40)])
def test_hidden_values_in_larger_blocks(G, T, B, Lp):
    """Blocks of 32 and 128 rows: a token with an infinite value and one with a
    NaN value reach the queries from it on, earlier ones keep their results."""
    H, L, D = 2, T + 90, 128
    q, k, v, kp, vp, _, _ = _make(B, H, G, T, L, D, "bf16", 1, Lp, seed=3)
    lens = torch.full((B,), 70, dtype=torch.int32)
    plens = torch.tensor([Lp], dtype=torch.int32) if Lp else None
    prob = nacl.Problem(B, H, L, D, "bf16", [L - 1], q_group=G)
    step = nacl.Step(prob, T, lens=lens.to(DEV))
    prefix = nacl.Prefix(prob, kp, vp) if Lp else None
    v[0, 0, 70 + T // 2] = float("inf")
    v[0, 1, 70 + T // 3, 5] = float("nan")
    k[B - 1, 1, 70 + T - 1] = float("nan")
    out, lse = nacl.prefix_attention(prob, step, q, k, v, prefix=prefix)
    torch.cuda.synchronize()
    late = lambda b, hq, t: (b == 0 and t >= (T // 2, T // 3)[hq // G]) or (b == B - 1 and hq // G == 1 and t == T - 1)
    rows = [x for x in _rows(B, H * G, T, 400) if not late(*x)]
    check_rows(q, k, v, kp, vp, lens, plens, out, lse, prob.c.sm_scale, rows)
    assert torch.isinf(out[0, 0, T // 2:]).all()
    odd = torch.isnan(out[0, G, T // 3:T - 1])
    assert odd[:, 5].all() and not odd[:, :5].any() and not odd[:, 6:].any()
    assert torch.isnan(lse[B - 1, G:, T - 1]).all()


@pytest.mark.parametrize("B,G,T,D,Lp,groups", [(65, 2, 1, 128, 901, 1), (43, 3, 2, 64, 640, 1), (80, 7, 1, 128, 77, 2)])
def test_blocks_of_256_rows(B, G, T, D, Lp, groups):
    """One block and a bit, full blocks, groups, chunks that end inside a tile."""
    H, L = 2, T + 20
    q, k, v, kp, vp, lens, plens = _make(B, H, G, T, L, D, "bf16", groups, Lp, seed=B)
    prob = nacl.Problem(B, H, L, D, "bf16", [L - 1], q_group=G)
    prefix = nacl.Prefix(prob, kp, vp, lens=plens.to(DEV))
    out, lse = nacl.prefix_attention(prob, nacl.Step(prob, T, lens=lens.to(DEV)), q, k, v, prefix=prefix)
    torch.cuda.synchronize()
    check_rows(q, k, v, kp, vp, lens, plens, out, lse, prob.c.sm_scale, _rows(B, H * G, T, 300))
