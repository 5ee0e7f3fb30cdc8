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
    order = sorted(range(len(x)), key=lambda i: (-x[i], i))
    if top_k > 0:
        order = order[:top_k]
    if weight is None:
        def weight(d, t):
            return math.exp(d / t)
    w = {i: 1.0 if x[i] == m else 0.0 if x[i] == -math.inf or m == math.inf else weight(x[i] - m, temperature) for i in order}
    if top_p < 1:
        total, reach, kept = sum(w.values()), 0.0, []
        for i in order:
            kept.append(i)
            reach += w[i]
            if reach >= top_p * total:
                break
        order = kept
    if min_p > 0:
        order = [i for i in order if w[i] >= min(min_p, 1.0)]
    total, cum, token = sum(w[i] for i in order), 0.0, None
    for i in sorted(order):
        if w[i] > 0:
            token = i
        cum += w[i]
        if cum > u * total:
            break
    return token, math.log(w[token] / total)
