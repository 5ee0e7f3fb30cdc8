"""The operators of decoding over a paged cache, several beams to a prompt among
them, with the sizes that programs call them at: pages for the new tokens, the new
tokens into the pages, attention over the pages, the beams' selection from the
logits, and the reordering of what the beams hold.

The kinds of case and what they stand for:

  assign   nacl.pages_assign: the step's lengths to page tables and to the slots of
           the new tokens; sequences that ended or were evicted give pages back,
           growing ones take them.
  append   nacl.paged_append: the new tokens' queries and keys normalised and
           rotated, keys and values written into their slots.
  attend   nacl.paged_attention: the new tokens over the rows that their sequences'
           pages hold, with every row's log-sum-exp.
  select   nacl.beam_select: of every group's beams and the vocabulary the best
           continuations.
  reorder  nacl.beam_reorder: every beam takes what its parent holds; a parent's
           first child takes its pages over, the others get copies in the pages of
           beams that ended.

`own` chooses between the plain form in elementary torch operations and the
library's calls.
"""

import math

import torch

DEVICE = "cuda"
own = False


# --------------------------------------------------------------------------
# Cases

def listed():
    return [
        # One new token each of 64 sequences, pages of 16 rows: the step's first call.
        dict(name="assign_step", kind="assign", B=64, T=1, page=16, rows=8256, ended=2),
        # Prompts of up to 2048 tokens join where others ended.
        dict(name="assign_prompts", kind="assign", B=256, T=2048, page=64, rows=12409, ended=64),
        # One new token each of 64 sequences.
        dict(name="append_token", kind="append", B=64, H=8, G=4, T=1, D=128, rot=128, page=16, rows=1088, dtype="bf16",
             norm=True, interleaved=False, fused=True, by_row=False),
        # Ragged prompts of grouped-query heads, pages laid out [page, row, head].
        dict(name="append_prompt", kind="append", B=3, H=8, G=4, T=9999, D=128, rot=128, page=64, rows=10240,
             dtype="bf16", norm=True, interleaved=False, fused=True, by_row=True),
        # One sequence over a short cache: where latency counts.
        dict(name="attend_token", kind="attend", B=1, H=8, G=4, T=1, D=128, page=16, rows=2112, dtype="bf16",
             by_row=False),
        # 32 sequences of different lengths.
        dict(name="attend_ragged", kind="attend", B=32, H=8, G=4, T=1, D=128, page=16, rows=8256, dtype="bf16",
             by_row=False),
        # Three sequences of up to 128k tokens, 64 query heads.
        dict(name="attend_long", kind="attend", B=3, H=8, G=8, T=1, D=128, page=64, rows=131072, dtype="bf16",
             by_row=True),
        # fp32 heads of 64, five tokens at once, pages of an odd number of rows.
        dict(name="attend_f32_odd", kind="attend", B=6, H=4, G=2, T=5, D=64, page=27, rows=1999, dtype="f32",
             by_row=False),
        # Four beams of one prompt over a 32000-token vocabulary.
        dict(name="select_row", kind="select", B=1, W=4, K=4, V=32000, dtype="f32"),
        # 32 prompts of eight beams over 128k tokens, twice as many candidates as beams.
        dict(name="select_batch", kind="select", B=32, W=8, K=16, V=131072, dtype="bf16"),
        # Four beams of one prompt, 64 tokens behind a shared prompt.
        dict(name="reorder_four", kind="reorder", B=1, W=4, H=8, D=128, page=16, shared=2048, rows=64, dead=1,
             dtype="bf16", by_row=False),
        # 16 prompts of eight beams, up to 576 rows of their own.
        dict(name="reorder_batch", kind="reorder", B=16, W=8, H=8, D=128, page=16, shared=1024, rows=576, dead=3,
             dtype="bf16", by_row=False),
    ]


def _log(rng, lo, hi):
    """A whole number whose logarithm is uniform over [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("assign", "append", "attend", "attend", "attend", "select", "select", "reorder"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    elt = 4 if dtype == "f32" else 2
    page = rng.choice((16, 16, 32, 64, 128, rng.randint(5, 100)))
    if kind == "select":
        V = rng.choice((_log(rng, 256, 262144), _log(rng, 16384, 262144)))
        W = rng.choice((1, 2, 4, 5, 8, _log(rng, 2, 32)))
        K = rng.choice((W, 2 * W, _log(rng, 1, 64)))
        return dict(kind=kind, B=_log(rng, 1, max(1, min(64, (1 << 24) // (V * W)))), W=W, K=min(K, 64, W * V), V=V,
                    dtype=dtype)
    if kind == "assign":
        B = _log(rng, 1, 512)
        T = rng.choice((1, 1, rng.randint(2, 8), _log(rng, 9, max(9, (1 << 18) // B))))
        return dict(kind=kind, B=B, T=T, page=page, rows=T + _log(rng, 16, 12288), ended=rng.randint(0, (B - 1) // 3))
    H, G, D = rng.choice((1, 2, 4, 8, 32)), rng.choice((1, 1, 2, 4, 7, 8)), rng.choice((64, 128, 128))
    if H == 32:
        G = rng.choice((1, 2))
    by_row = rng.random() < 0.4
    if kind == "append":
        T = rng.choice((1, rng.randint(2, 8), _log(rng, 16, 16384)))
        # At most 250 MB of new rows.
        T = min(T, 250000000 // (H * (G + 2) * D * elt))
        B = _log(rng, 1, max(1, min(64, (1 << 18) // (T * H * (G + 2)))))
        return dict(kind=kind, B=B, H=H, G=G, T=T, D=D, rot=rng.choice((D, D, D // 2)), page=page,
                    rows=T + _log(rng, 16, 1024), dtype=dtype, norm=rng.random() < 0.5,
                    interleaved=rng.random() < 0.3, fused=rng.random() < 0.5, by_row=by_row)
    if kind == "reorder":
        W = rng.choice((2, 4, 5, 8, _log(rng, 2, 16)))
        B = _log(rng, 1, 16)
        # At most 2^18 rows of all heads.
        rows = max(1, min(_log(rng, 1, 2048), (1 << 18) // (B * W * H)))
        return dict(kind=kind, B=B, W=W, H=H, D=D, page=page, shared=page * _log(rng, 1, max(1, 2048 // page)),
                    rows=rows, dead=rng.randint(0, W - 1), dtype=dtype, by_row=by_row)
    T = rng.choice((1, 1, 1, rng.randint(2, 8)))
    B = rng.choice((1, _log(rng, 1, 64), _log(rng, 8, 64)))
    # At most 2^26 (query row, key) pairs and 2^21 cache rows over all heads.
    rows = rng.choice((_log(rng, 16, 16384), _log(rng, 1024, 131072)))
    rows = T + max(8, min(rows, (1 << 26) // (B * H * G * T), (1 << 21) // (B * H * (elt // 2))))
    return dict(kind=kind, B=B, H=H, G=G, T=T, D=D, page=page, rows=rows, dtype=dtype, by_row=by_row)


# --------------------------------------------------------------------------
# Inputs

def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    return g


def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _randn(g, shape, dtype):
    return torch.randn(shape, generator=g, device=DEVICE, dtype=dtype)


def _lens(g, n, lo, hi):
    """n lengths in [lo, hi], the first of them hi."""
    t = torch.randint(lo, hi + 1, (n,), generator=g, device=DEVICE, dtype=torch.int32)
    t[0] = hi
    return t


def _up(n, d):
    return (n + d - 1) // d


def _pool(g, c, n):
    """Pages [n, H, page, D], their rows either head by head or row by row."""
    H, P, D = c["H"], c["page"], c["D"]
    if c["by_row"]:
        return _randn(g, (n, P, H, D), _dtype(c["dtype"])).transpose(1, 2)
    return _randn(g, (n, H, P, D), _dtype(c["dtype"]))


def _table(g, B, entries, spare=3):
    """A table of B sequences whose pages lie anywhere in the pool; the pool's pages."""
    n = B * entries + spare
    return torch.randperm(n, generator=g, device=DEVICE)[:B * entries].view(B, entries).int(), n


def _inputs(c, seed):
    """What both forms and the 64-bit reference are computed from."""
    g = _generator(seed)
    if c["kind"] == "select":
        # Logits as a language model's: a broad bulk and, in each row, some
        # tokens far above it.  The beams' scores are sums of log-probabilities;
        # some beams have ended.
        N, V = c["B"] * c["W"], c["V"]
        x = torch.randn((N, V), generator=g, device=DEVICE).mul_(2.0)
        at = torch.randint(0, V, (N, max(1, V // 500)), generator=g, device=DEVICE)
        x.scatter_add_(1, at, torch.rand(at.shape, generator=g, device=DEVICE) * 9.0)
        shape = (c["B"], c["W"])
        scores = -20.0 - 3.0 * torch.rand(shape, generator=g, device=DEVICE)
        ended = (torch.rand(shape, generator=g, device=DEVICE) < 0.1).int()
        return dict(logits=x.to(_dtype(c["dtype"])), scores=scores, ended=ended, end_token=2 % V)
    B, P = c["B"], c["page"]
    if c["kind"] == "assign":
        T = c["T"]
        entries = _up(c["rows"], P)
        table, n = _table(g, B, entries)
        lens = _lens(g, B, 0, c["rows"] - T)
        n_new = torch.full((B,), T, device=DEVICE, dtype=torch.int32)
        if T > 1:
            n_new = _lens(g, B, 0, T)
        # What a sequence holds covers its rows; some were evicted since and hold
        # more than they need; the last ones have ended.
        held = (lens + P - 1) // P
        held = torch.where(torch.rand((B,), generator=g, device=DEVICE) < 0.1, torch.clamp(held + 5, max=entries), held)
        if c["ended"]:
            lens[-c["ended"]:] = 0
            n_new[-c["ended"]:] = 0
        held = held.int()
        used = torch.arange(entries, device=DEVICE) < held[:, None]
        owned = torch.zeros((n,), dtype=torch.bool, device=DEVICE)
        owned[table[used].long()] = True
        rest = torch.nonzero(~owned)[:, 0]
        rest = rest[torch.randperm(rest.numel(), generator=g, device=DEVICE)].int()
        free = torch.zeros((n,), dtype=torch.int32, device=DEVICE)
        free[:rest.numel()] = rest
        n_free = torch.tensor([rest.numel()], dtype=torch.int32, device=DEVICE)
        table = torch.where(used, table, -1).int()
        return dict(table=table, lens=lens, n_new=n_new, held=held, free=free, n_free=n_free)
    if c["kind"] == "reorder":
        # The beams of a prompt share its pages; behind them each has its own.
        W, rows = c["W"], c["rows"]
        first, entries = c["shared"] // P, _up(rows, P) + 1
        own_pages, n_own = _table(g, B * W, entries, spare=0)
        shared = torch.arange(B * first, device=DEVICE, dtype=torch.int32).view(B, 1, first) + n_own
        table = torch.cat((shared.expand(B, W, first).reshape(B * W, first), own_pages), dim=1).contiguous()
        n = n_own + B * first
        lens = (c["shared"] + _lens(g, B, (rows + 1) // 2, rows)).int().repeat_interleave(W)
        # dead beams of each group have no child; every other has one at least.
        order = torch.rand((B, W), generator=g, device=DEVICE).argsort(dim=1)
        alive = order[:, c["dead"]:]
        pick = torch.randint(0, W - c["dead"], (B, c["dead"]), generator=g, device=DEVICE)
        parents = torch.cat((alive, alive.gather(1, pick)), dim=1)
        parents = parents.gather(1, torch.rand((B, W), generator=g, device=DEVICE).argsort(dim=1)).int().contiguous()
        held = torch.full((B * W,), first + entries, dtype=torch.int32, device=DEVICE)
        return dict(k=_pool(g, c, n), v=_pool(g, c, n), table=table, parents=parents, lens=lens, held=held)
    H, G, T, D, rows = (c[x] for x in ("H", "G", "T", "D", "rows"))
    table, n = _table(g, B, _up(rows, P))
    s = dict(k=_pool(g, c, n), v=_pool(g, c, n), table=table)
    if c["kind"] == "attend":
        s["lens"] = _lens(g, B, (rows - T) // 4, rows - T)
        s["q"] = _randn(g, (B, H * G, T, D), _dtype(c["dtype"]))
        return s
    s["lens"] = _lens(g, B, 0, rows - T)
    s["n_new"] = _lens(g, B, _up(T, 2), T)
    if c["fused"]:
        # The projections' one output, [B, T, (Hq + 2 H) D].
        x = _randn(g, (B, T, H * G + 2 * H, D), _dtype(c["dtype"])).permute(0, 2, 1, 3)
        s["q"], s["kn"], s["vn"] = x[:, :H * G], x[:, H * G:H * G + H], x[:, H * G + H:]
    else:
        s["q"], s["kn"], s["vn"] = (_randn(g, (B, h, T, D), _dtype(c["dtype"])) for h in (H * G, H, H))
    t = torch.arange(T, device=DEVICE)
    j = s["lens"].long()[:, None] + t
    slot = table.long().gather(1, j // P) * P + j % P
    s["slots"] = torch.where(t < s["n_new"][:, None], slot, -1).int()
    # An evicted cache holds fewer rows than the sequence has tokens.
    s["positions"] = ((5 * s["lens"])[:, None] + t.int()).contiguous()
    i = torch.arange(c["rot"] // 2, device=DEVICE, dtype=torch.float64)
    s["inv_freq"] = (10000.0 ** (-2.0 * i / c["rot"])).float()
    # Padding tokens leave what is there.
    s["q_out"] = torch.zeros((B, H * G, T, D), dtype=_dtype(c["dtype"]), device=DEVICE)
    s["wq"] = s["wk"] = None
    if c["norm"]:
        s["wq"], s["wk"] = ((1.0 + 0.2 * _randn(g, (D,), torch.float32)).to(_dtype(c["dtype"])) for _ in range(2))
    return s


def prepare(case, seed):
    c, s = case, _inputs(case, seed)
    s["case"] = c
    if not own:
        return s
    from paper_2408_03675_amd import nacl
    if c["kind"] == "select":
        shape = (c["B"], c["K"])
        s["parents"], s["tokens"] = (torch.empty(shape, dtype=torch.int32, device=DEVICE) for _ in range(2))
        s["out"] = torch.empty(shape, dtype=torch.float32, device=DEVICE)
        s["ws"] = nacl.beam_workspace(c["B"], c["W"], c["V"], c["K"], DEVICE)
        return s
    B = c["B"] * c.get("W", 1)
    H, G, D = c.get("H", 1), c.get("G", 1), c.get("D", 64)
    rows = c["rows"] + c.get("shared", 0)
    s["prob"] = nacl.Problem(B, H, rows, D, c.get("dtype", "bf16"), [rows - 1], q_group=G)
    if c["kind"] == "assign":
        s["step"] = nacl.Step(s["prob"], c["T"], lens=s["lens"], n_new=s["n_new"])
        s["slots"] = torch.empty((B, c["T"]), dtype=torch.int32, device=DEVICE)
        s["held_out"], s["n_free_out"] = torch.empty_like(s["held"]), torch.empty_like(s["n_free"])
        s["missing"] = torch.empty_like(s["n_free"])
        return s
    s["pages"] = nacl.Pages(s["prob"], s["k"], s["v"], s["table"])
    if c["kind"] == "reorder":
        s["table_out"], s["lens_out"], s["held_out"] = (torch.empty_like(s[x]) for x in ("table", "lens", "held"))
        return s
    s["step"] = nacl.Step(s["prob"], c["T"], lens=s["lens"], n_new=s.get("n_new"))
    if c["kind"] == "append":
        s["rotation"] = nacl.Rotation(s["prob"], s["inv_freq"], q_weight=s["wq"], k_weight=s["wk"], eps=1e-6,
                                      interleaved=c["interleaved"])
        return s
    s["out"] = torch.empty((B, H * G, c["T"], D), dtype=_dtype(c["dtype"]), device=DEVICE)
    s["lse"] = torch.empty((B, H * G, c["T"]), dtype=torch.float32, device=DEVICE)
    s["ws"] = nacl.paged_workspace(s["prob"], s["step"], s["pages"], device=DEVICE)
    return s


# --------------------------------------------------------------------------
# The plain form

def _plain_assign(c, s):
    B, T, P = c["B"], c["T"], c["page"]
    table, held, free = s["table"], s["held"].long(), s["free"]
    entries = table.shape[1]
    at = torch.arange(entries, device=DEVICE)
    want = (s["lens"].long() + s["n_new"] + P - 1).div(P, rounding_mode="floor").clamp(max=entries)
    # The stack of free pages: what it held, then what comes back.
    back = table[(at >= want[:, None]) & (at < held[:, None])]
    stack = torch.cat((free[:int(s["n_free"])], back))
    free[:stack.numel()] = stack
    take = (want - held).clamp(min=0)
    total = take.cumsum(0)
    granted = total <= stack.numel()
    new = (at >= held[:, None]) & (at < want[:, None]) & granted[:, None]
    n = int(new.sum())
    table[new] = stack.flip(0)[:n]
    held_out = torch.where(granted | (take == 0), want, held)
    t = torch.arange(T, device=DEVICE)
    j = s["lens"].long()[:, None] + t
    page = j.div(P, rounding_mode="floor")
    ok = (t < s["n_new"][:, None]) & (page < held_out[:, None])
    slots = table.long().gather(1, page.clamp(max=entries - 1)) * P + j % P
    slots = torch.where(ok, slots, -1).int()
    missing = (total[-1:] - stack.numel()).clamp(min=0).int()
    n_free = torch.full((1,), stack.numel() - n, dtype=torch.int32, device=DEVICE)
    return table, held_out.int(), free, n_free, slots, missing


def _rotate_rows(x, w, cos, sin, interleaved):
    """x [B, h, T, D] normalised with weights w (None: not) and rotated, in
    32 bits; cos, sin [B, 1, T, rot / 2]."""
    y = x.float()
    if w is not None:
        y = y * torch.rsqrt((y * y).mean(dim=-1, keepdim=True) + 1e-6) * w.float()
    n = cos.shape[-1]
    out = y.clone()
    if interleaved:
        a, b = y[..., 0:2 * n:2], y[..., 1:2 * n:2]
        out[..., 0:2 * n:2], out[..., 1:2 * n:2] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = y[..., :n], y[..., n:2 * n]
        out[..., :n], out[..., n:2 * n] = a * cos - b * sin, b * cos + a * sin
    return out.to(x.dtype)


def _plain_append(c, s):
    P = c["page"]
    angle = s["positions"].double()[:, None, :, None] * s["inv_freq"].double()
    cos, sin = angle.cos().float(), angle.sin().float()
    q = _rotate_rows(s["q"], s["wq"], cos, sin, c["interleaved"])
    kn = _rotate_rows(s["kn"], s["wk"], cos, sin, c["interleaved"])
    real = torch.arange(c["T"], device=DEVICE) < s["n_new"][:, None]
    s["q_out"].copy_(torch.where(real[:, None, :, None], q, s["q_out"]))
    b, t = torch.nonzero(s["slots"] >= 0, as_tuple=True)
    slot = s["slots"][b, t].long()
    page, off = slot.div(P, rounding_mode="floor"), slot % P
    s["k"][page, :, off] = kn[b, :, t]
    s["v"][page, :, off] = s["vn"][b, :, t]
    return s["q_out"], s["k"], s["v"]


def _rows_of(c, s, x):
    """The rows that the sequences' pages hold, [B, H, rows, D] in 32 bits."""
    y = s[x][s["table"].long()]  # [B, entries, H, page, D]
    return y.permute(0, 2, 1, 3, 4).reshape(c["B"], c["H"], -1, c["D"])[:, :, :c["rows"]].float()


def _plain_attend(c, s):
    B, H, G, T, D = (c[x] for x in ("B", "H", "G", "T", "D"))
    q = s["q"].float().view(B, H, G * T, D)
    a = q @ _rows_of(c, s, "k").transpose(2, 3).contiguous() * (1.0 / math.sqrt(D))
    L = a.shape[-1]
    seen = s["lens"][:, None, None] + torch.arange(1, T + 1, device=DEVICE)[None, :, None]
    hidden = torch.arange(L, device=DEVICE) >= seen  # [B, T, L]
    a = a.view(B, H, G, T, L).masked_fill_(hidden[:, None, None], -math.inf).view(B, H, G * T, L)
    m = a.amax(dim=-1, keepdim=True)
    w = (a - m).exp_()
    total = w.sum(dim=-1, keepdim=True)
    out = (w @ _rows_of(c, s, "v")) / total
    return out.to(s["q"].dtype).view(B, H * G, T, D), (m + total.log()).view(B, H * G, T)


def _plain_select(c, s):
    B, W, V, K = (c[x] for x in ("B", "W", "V", "K"))
    # Candidates of different beams come close, so their scores are in 64 bits.
    x = s["logits"].double().view(B, W, V)
    m = x.amax(dim=-1, keepdim=True)
    x = x - (m + (x - m).exp_().sum(dim=-1, keepdim=True).log_())
    ended = s["ended"][:, :, None] != 0
    x = torch.where(ended, -math.inf, x)
    x[:, :, s["end_token"]] = torch.where(ended[:, :, 0], 0.0, x[:, :, s["end_token"]])
    x += s["scores"].double()[:, :, None]
    # The best K, ties to the lowest beam and token.
    order = torch.sort(x.view(B, W * V), dim=1, descending=True, stable=True)
    best, at = order.values[:, :K], order.indices[:, :K]
    none = best == -math.inf
    parents = torch.where(none, -1, at.div(V, rounding_mode="floor")).int()
    return parents, torch.where(none, -1, at % V).int(), best.float()


def _assignment(parents):
    """Whose pages each beam takes over: a parent's first child the parent's, every
    other beam those of the beams without a child, in order."""
    W = parents.shape[1]
    same = parents[:, :, None] == parents[:, None, :]
    first = ~(same & torch.ones((W, W), dtype=torch.bool, device=DEVICE).tril(-1)).any(dim=2)
    has_child = torch.zeros(parents.shape, dtype=torch.bool, device=DEVICE)
    has_child.scatter_(1, parents.long(), True)
    dead = torch.sort(has_child.int(), dim=1, stable=True).indices  # those without a child first
    rank = (~first).long().cumsum(1) - 1
    return torch.where(first, parents.long(), dead.gather(1, rank.clamp(min=0))), first


def _plain_reorder(c, s):
    W, P = c["W"], c["page"]
    base = W * torch.arange(c["B"], device=DEVICE)[:, None]
    takes, first = _assignment(s["parents"])
    takes = (base + takes).view(-1)
    source = (base + s["parents"]).view(-1)
    table = s["table"][takes]
    lens = s["lens"][source]
    j = torch.arange(int(s["lens"].max()), device=DEVICE)
    page = j.div(P, rounding_mode="floor")
    to, of = table.long()[:, page], s["table"].long()[source][:, page]
    i, j = torch.nonzero((j < lens[:, None]) & (to != of), as_tuple=True)
    to, of, off = to[i, j], of[i, j], j % P
    s["k"][to, :, off] = s["k"][of, :, off]
    s["v"][to, :, off] = s["v"][of, :, off]
    return table, lens, s["held"][takes], s["k"], s["v"]


# --------------------------------------------------------------------------
# One pass

def run(s):
    c = s["case"]
    if not own:
        return {"assign": _plain_assign, "append": _plain_append, "attend": _plain_attend, "select": _plain_select,
                "reorder": _plain_reorder}[c["kind"]](c, s)
    from paper_2408_03675_amd import nacl
    if c["kind"] == "assign":
        nacl.pages_assign(s["step"], c["page"], s["table"], s["held"], s["free"], s["n_free"], held_out=s["held_out"],
                          n_free_out=s["n_free_out"], slots=s["slots"], missing=s["missing"])
        return s["table"], s["held_out"], s["free"], s["n_free_out"], s["slots"], s["missing"]
    if c["kind"] == "append":
        nacl.paged_append(s["prob"], s["step"], s["rotation"], s["positions"], s["q"], s["kn"], s["vn"], s["pages"],
                          s["slots"], q_out=s["q_out"])
        return s["q_out"], s["k"], s["v"]
    if c["kind"] == "attend":
        return nacl.paged_attention(s["prob"], s["step"], s["q"], s["pages"], out=s["out"], lse=s["lse"], ws=s["ws"])
    if c["kind"] == "select":
        return nacl.beam_select(s["logits"], s["scores"], c["K"], ended=s["ended"], end_token=s["end_token"],
                                parents=s["parents"], tokens=s["tokens"], out=s["out"], ws=s["ws"])
    nacl.beam_reorder(s["prob"], s["pages"], s["parents"], s["lens"], held=s["held"], table_out=s["table_out"],
                      lens_out=s["lens_out"], held_out=s["held_out"])
    return s["table_out"], s["lens_out"], s["held_out"], s["k"], s["v"]


# --------------------------------------------------------------------------
# What a pass cannot do without

def _mean(n, lo, hi):
    """The expected sum of n lengths as _lens makes them."""
    return hi + (n - 1) * (lo + hi) / 2


def work(case):
    c = case
    elt = 4 if c.get("dtype") == "f32" else 2
    B = c["B"]
    if c["kind"] == "assign":
        # Lengths, new tokens and held pages of every sequence, its pages held
        # afterwards, the slots, and each page that changes hands: from the stack
        # into a table, or from the table of one that ended to the stack.
        live = B - c["ended"]
        new = _mean(live, 0, c["T"]) if c["T"] > 1 else live
        moved = new / c["page"] + c["ended"] * c["rows"] / 2 / c["page"]
        return dict(bytes=16 * B + 4 * B * c["T"] + 8 * moved, flops=B * c["T"])
    if c["kind"] == "select":
        n = B * c["W"]
        return dict(bytes=n * c["V"] * elt + 8 * n + 12 * B * c["K"], flops=4 * n * c["V"])
    H, D = c["H"], c["D"]
    if c["kind"] == "reorder":
        entries = c["shared"] // c["page"] + _up(c["rows"], c["page"]) + 1
        rows = c["dead"] * _mean(B, (c["rows"] + 1) // 2, c["rows"])
        return dict(bytes=4 * rows * H * D * elt + B * c["W"] * (8 * entries + 20), flops=0)
    Hq, T = H * c["G"], c["T"]
    if c["kind"] == "append":
        tokens = _mean(B, _up(T, 2), T)
        norm = 4 * (Hq + H) * D if c["norm"] else 0
        return dict(bytes=tokens * (2 * (Hq + 2 * H) * D * elt + 8) + 8 * B,
                    flops=tokens * (3 * (Hq + H) * c["rot"] + norm))
    keys = _mean(B, (c["rows"] - T) // 4, c["rows"] - T) + B * T
    return dict(bytes=2 * keys * H * D * elt + B * Hq * T * (2 * D * elt + 4) + 4 * keys / c["page"] + 4 * B,
                flops=4 * keys * Hq * T * D)


# --------------------------------------------------------------------------
# The definition in 64 bits

def _exact_append(c, s):
    H, D, P, n = c["H"], c["D"], c["page"], c["rot"] // 2
    outs = []
    turns = s["positions"].double().unsqueeze(-1) * s["inv_freq"].double()  # [B, T, n]
    z = torch.polar(torch.ones_like(turns), turns).unsqueeze(1)
    for x, w in ((s["q"], s["wq"]), (s["kn"], s["wk"])):
        y = x.double()
        if w is not None:
            y = y / (y.square().sum(-1, keepdim=True) / D + 1e-6).sqrt() * w.double()
        # A pair is a complex number, which the rotation multiplies by e^(i angle).
        pair = y[..., :2 * n].unflatten(-1, (n, 2) if c["interleaved"] else (2, n))
        if not c["interleaved"]:
            pair = pair.transpose(-1, -2)
        turned = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * z)
        if not c["interleaved"]:
            turned = turned.transpose(-1, -2)
        outs.append(torch.cat((turned.flatten(-2), y[..., 2 * n:]), dim=-1))
    q_out, k, v = s["q_out"].double(), s["k"].double(), s["v"].double()
    for b, m in enumerate(s["n_new"].tolist()):
        q_out[b, :, :m] = outs[0][b, :, :m]
        at = s["slots"][b, :m].long()
        for h in range(H):
            k[at // P, h, at % P] = outs[1][b, h, :m]
            v[at // P, h, at % P] = s["vn"][b, h, :m].double()
    return q_out, k, v


def _exact_attend(c, s):
    B, H, G, T, D, P = (c[x] for x in ("B", "H", "G", "T", "D", "page"))
    out = torch.zeros((B, H * G, T, D), dtype=torch.float64, device=DEVICE)
    lse = torch.zeros((B, H * G, T), dtype=torch.float64, device=DEVICE)
    for b, n in enumerate(s["lens"].tolist()):
        at = torch.arange(n + T, device=DEVICE)
        page = s["table"][b].long()[at // P]
        for h in range(H):
            k, v = (s[x][page, h, at % P].double() for x in ("k", "v"))
            for t in range(T):
                q = s["q"][b, h * G:h * G + G, t].double()
                a = (k[:n + t + 1] @ q.T.contiguous()) / math.sqrt(D)  # [keys, G]
                norm = torch.logsumexp(a, dim=0)
                lse[b, h * G:h * G + G, t] = norm
                out[b, h * G:h * G + G, t] = (v[:n + t + 1].T.contiguous() @ torch.exp(a - norm)).T
    return out, lse


def _exact_select(c, s):
    B, W, V, K = (c[x] for x in ("B", "W", "V", "K"))
    best = []
    for b in range(B):
        found = []
        for w in range(W):
            score = s["scores"][b, w].double().view(1)
            if bool(s["ended"][b, w]):
                found.append(score)
                continue
            x = s["logits"][b * W + w].double()
            found.append(score + torch.topk(x, min(K, V)).values - torch.logsumexp(x, dim=0))
        found = torch.cat(found + [torch.full((K,), -math.inf, dtype=torch.float64, device=DEVICE)])
        best.append(torch.topk(found, K).values)
    return None, None, torch.stack(best)


def _exact_assign(c, s):
    # One sequence after the other, on the host.
    P, T = c["page"], c["T"]
    table, held = s["table"].tolist(), s["held"].tolist()
    lens, n_new = s["lens"].tolist(), s["n_new"].tolist()
    free, n = s["free"].tolist(), int(s["n_free"])
    want = [min(len(row), -(-(have + new) // P)) for row, have, new in zip(table, lens, n_new)]
    for row, old, w in zip(table, held, want):
        for page in row[w:old]:
            free[n] = page
            n += 1
    asked = short = 0
    had, slots = n, []
    for b, w in enumerate(want):
        asked += max(0, w - held[b])
        if w > held[b] and asked > had:
            short = asked - had
        else:
            for e in range(held[b], w):
                n -= 1
                table[b][e] = free[n]
            held[b] = w
        rows = range(lens[b], min(lens[b] + n_new[b], held[b] * P))
        slots.append([table[b][j // P] * P + j % P for j in rows] + [-1] * (T - len(rows)))
    return tuple(torch.tensor(x, dtype=torch.int32, device=DEVICE) for x in (table, held, free, [n], slots, [short]))


def _exact_reorder(c, s):
    # One group after the other, on the host; the rows of a beam at a time.
    W, P = c["W"], c["page"]
    table, lens, held = s["table"].tolist(), s["lens"].tolist(), s["held"].tolist()
    k, v = s["k"].clone(), s["v"].clone()
    out = [], [], []
    for g, parents in enumerate(s["parents"].tolist()):
        spare = [w for w in range(W) if w not in parents]
        for i, parent in enumerate(parents):
            takes = spare.pop(0) if parent in parents[:i] else parent
            source, takes = g * W + parent, g * W + takes
            for x, values in zip(out, (table[takes], lens[source], held[takes])):
                x.append(values)
            for e in range(-(-lens[source] // P)):
                to, of, n = table[takes][e], table[source][e], min(P, lens[source] - e * P)
                if to != of:
                    k[to, :, :n], v[to, :, :n] = s["k"][of, :, :n], s["v"][of, :, :n]
    return tuple(torch.tensor(x, dtype=torch.int32, device=DEVICE) for x in out) + (k.double(), v.double())


def exact(case, seed):
    """run's outputs for these inputs in 64 bits."""
    form = {"assign": _exact_assign, "append": _exact_append, "attend": _exact_attend, "select": _exact_select,
            "reorder": _exact_reorder}[case["kind"]]
    return form(case, _inputs(case, seed))
