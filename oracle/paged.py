"""Plain references of decoding over a paged cache and of beam search: the pages of
a step, the beams' continuations in float64, and what beams take over from their
parents.  Test infrastructure only; shares no code with the GPU path."""

import math

import numpy as np


def assign_pages(page, n_pages, table, held, free, n_free, lens, n_new, T, L, row0=0, shared=None):
    """(table, held, free, n_free, slots, missing) after a step of T tokens, lists
    of whole numbers."""
    table, held, free = [list(r) for r in table], list(held), list(free)
    B, entries = len(table), len(table[0])
    new = [max(0, min(T, n)) for n in n_new]
    want = [min(entries, -(-max(0, min(L, row0 + lens[b] + new[b])) // page)) for b in range(B)]
    held = [max(0, min(entries, n)) for n in held]
    stack = free[:max(0, min(n_pages, n_free))]
    for b in range(B):
        for e in range(max(want[b], shared[b] if shared else 0), held[b]):
            if len(stack) < n_pages:
                stack.append(table[b][e])
    free[:len(stack)] = stack
    asked, stood = 0, len(stack)
    for b in range(B):
        need = max(0, want[b] - held[b])
        asked += need
        if need and asked > stood:
            continue
        for e in range(held[b], want[b]):
            table[b][e] = stack.pop()
        held[b] = want[b]
    slots = []
    for b in range(B):
        row = []
        for t in range(T):
            j = row0 + lens[b] + t
            ok = t < new[b] and 0 <= j < L and j // page < held[b] and 0 <= table[b][j // page] < n_pages
            row.append(table[b][j // page] * page + j % page if ok else -1)
        slots.append(row)
    return table, held, free, len(stack), slots, max(0, asked - stood)


def beam_values(x, score, ended=False, end_token=0):
    """(values [V], largest error of a value that fp32 exponentials explain) of one
    beam; -inf: no continuation.  An exponential is off by 3 |d| 2^-24 of itself (d,
    its argument, rounded as a difference and as a product) and 4 steps of its own;
    32 are summed in fp32."""
    x = np.array(x, dtype=np.float64)
    x[np.isnan(x)] = -math.inf
    values = np.full(x.shape, -math.inf)
    if not math.isfinite(score):
        return values, 0.0
    if ended:
        values[end_token] = score
        return values, 0.0
    m = x.max()
    if m == -math.inf:
        return values, 0.0
    if m == math.inf:
        values[x == m] = score - math.log((x == m).sum())
        return values, 0.0
    w = np.exp(x - m)
    d = np.where(w > 0, m - x, 0.0)
    seen = np.isfinite(x)
    values[seen] = score + ((x[seen] - m) - math.log(w.sum()))
    return values, float((w * (3 * d + 36)).sum() / w.sum()) * 2.0 ** -24


def best(values, K):
    """The K best of values [W, V], ties by beam, then token: (beams, tokens,
    values), -1, -1, -inf where there are none."""
    flat = np.asarray(values).reshape(-1)
    order = np.argsort(-flat, kind="stable")[:K]
    order = order[flat[order] > -math.inf]
    V = np.asarray(values).shape[1]
    pad = [-1] * (K - len(order))
    return ([int(i // V) for i in order] + pad, [int(i % V) for i in order] + pad,
            [float(flat[i]) for i in order] + [-math.inf] * len(pad))


def take_over(parents, lens, held, entries, page, L):
    """One group: for every beam, (the beam whose table row it takes, its length, the
    rows to copy from its parent's pages)."""
    W = len(parents)
    ok = [0 <= p < W for p in parents]
    first = [ok[i] and parents[i] not in parents[:i] for i in range(W)]
    spare = [w for w in range(W) if w not in parents]
    out = []
    for i, p in enumerate(parents):
        takes = p if first[i] else spare.pop(0)
        room = entries if held is None or not ok[i] else max(0, min(entries, held[takes], held[p]))
        n = max(0, min(lens[p], L, room * page)) if ok[i] else 0
        out.append((takes, n, 0 if first[i] else n))
    return out
