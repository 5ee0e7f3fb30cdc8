"""Plain float64 references of the decoding step's operators: rotation of the
new tokens, attention to a cache and a shared prefix, and the draw of the next
token.  Test infrastructure only; shares no code with the GPU path."""

import math

import numpy as np


def rotate(x, positions, inv_freq, weight=None, eps=0.0, interleaved=False):
    """x [T, D], one head of one sequence, normalised (with weights) and rotated
    by positions [T]; the first 2 len(inv_freq) entries turn."""
    x = np.array(x, dtype=np.float64)
    T, D = x.shape
    if weight is not None:
        for t in range(T):
            x[t] = x[t] / math.sqrt(np.mean(x[t] ** 2) + eps) * np.asarray(weight, dtype=np.float64)
    n = len(inv_freq)
    y = x.copy()
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        angle = np.asarray(positions, dtype=np.float64) * float(inv_freq[i])
        y[:, a] = x[:, a] * np.cos(angle) - x[:, b] * np.sin(angle)
        y[:, b] = x[:, b] * np.cos(angle) + x[:, a] * np.sin(angle)
    return y


def attend_row(q, k, v, scale):
    """One query row q [D] over the keys it sees, k, v [n, D]: (output,
    log-sum-exp, sum of probability times |value|, largest scale * sum |q||k|).
    Nothing seen, or no weight: zeros and -inf."""
    q, k, v = (np.asarray(t, dtype=np.float64) for t in (q, k, v))
    if len(k) == 0:
        return np.zeros(q.shape[0]), -math.inf, np.zeros(q.shape[0]), 0.0
    a = scale * (k @ q)
    m = a.max()
    if m == -math.inf:
        return np.zeros(q.shape[0]), -math.inf, np.zeros(q.shape[0]), 0.0
    w = np.exp(a - m)
    z = w.sum()
    return (w @ v) / z, m + math.log(z), (w @ np.abs(v)) / z, float((scale * (np.abs(k) @ np.abs(q))).max())


def draw_token(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, weight=None):
    """(token, ln of its probability) of one row of logits; weight(d, t): the
    weight of a logit d below the largest (default exp(d / t))."""
    x = np.array(x, dtype=np.float64)
    x[np.isnan(x)] = -math.inf
    m = x.max()
    if m == -math.inf:
        return -1, -math.inf
    if not temperature > 0:
        temperature, top_k = 1.0, 1
    order = np.argsort(-x, kind="stable")
    if top_k > 0:
        order = order[:top_k]
    with np.errstate(all="ignore"):
        w = np.exp((x - m) / temperature) if weight is None else weight(x - m, temperature)
    w = np.where(x == m, 1.0, np.where((x == -math.inf) | (m == math.inf), 0.0, w))
    if top_p < 1:
        reach = np.cumsum(w[order])
        order = order[:1 + int((reach < top_p * reach[-1]).sum())]
    if min_p > 0:
        order = order[w[order] >= min(min_p, 1.0)]
    order = np.sort(order)
    cum = np.cumsum(w[order])
    at = int((cum <= u * cum[-1]).sum())
    if at == len(order) or w[order[at]] == 0:
        at = int(np.flatnonzero(w[order] > 0)[-1])
    return int(order[at]), math.log(w[order[at]] / cum[-1])
