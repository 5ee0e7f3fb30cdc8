"""The bound that the few-row attention's outputs are held to, on the CPU: it
passes probabilities of two bf16 and refuses those of one."""

import numpy as np
import pytest
import torch

from oracle.step import attend_row


def excess(out, q, k, v, sm_scale, u):
    """By how much a bf16 output row passes its tolerance (at most 0: right):
    fp32 products of D terms and sums of n keys put each logit off by
    (D + 8) 2^-24 S (S the largest scaled sum of |q||k|) and each weight by the
    same, doubled through the normalisation; the exponentials and sums add
    (n + 64) 2^-24; the probabilities are rounded by u, the output once."""
    ref, _, size, S = attend_row(q, k, v, sm_scale)
    gamma = (len(q) + 8) * 2.0 ** -24 * S + (len(k) + 64) * 2.0 ** -24
    return (np.abs(out - ref) - torch.finfo(torch.bfloat16).eps / 2 * np.abs(ref) - (u + 2 * gamma) * 1.01 * size).max()


def _bf16(x):
    return torch.from_numpy(x).to(torch.bfloat16).double().numpy()


@pytest.mark.parametrize("n", [9, 24, 39])
def test_one_bf16_is_refused(n):
    rng = np.random.default_rng(n)
    D, refused = 64, 0
    for _ in range(32):
        q, k, v = (_bf16(s * rng.standard_normal(d)) for s, d in ((0.25, D), (1, (n, D)), (1, (n, D))))
        a = k @ q / 8
        w = np.exp(a - a.max())
        one = _bf16(w)
        two = one + _bf16(w - one)
        assert excess(_bf16(two @ v / w.sum()), q, k, v, 1 / 8, 2.0 ** -17) <= 0
        refused += excess(_bf16(one @ v / w.sum()), q, k, v, 1 / 8, 2.0 ** -17) > 0
    assert refused >= 30
