"""nacl_sample's tokens as members of the kept set at their place in the draw,
with their own probability: finite masks, far slices, infinite temperatures."""

import math

import numpy as np
import pytest
import torch

nacl = pytest.importorskip("paper_2408_03675_amd.nacl")
from test_gpu_sample import DEV, _sample

pytestmark = pytest.mark.gpu
F32_MIN, BF16_MIN = float(torch.finfo(torch.float32).min), float(torch.finfo(torch.bfloat16).min)


def _kept(x, t, k, p, m):
    """Indices, in order, and float64 weights of the tokens that the settings keep."""
    order = np.argsort(-x, kind="stable")
    if k > 0:
        order = order[:k]
    w = np.exp((x - x.max()) / t)
    if p < 1:
        reach = np.cumsum(w[order])
        order = order[:1 + int((reach < p * reach[-1]).sum())]
    order = np.sort(order[w[order] >= m])
    return order, w[order]


def check_draw(x, token, lp, u, t, k, p, m):
    """The token is kept, its share of [0, 1) holds u and lp is the logarithm of
    that share, for a top-p and a min-p within their rounding.  A weight's
    exponent is off by |ln w| 2^-22 and its value by two steps of fp32, so for
    |ln w| <= 30 by 2^-17 at most; tokens within 2^-18 of a top-p border are kept or
    not, which moves the sum by 2^-17 at most: together 2^-16.  The running sums'
    error is the weighted mean of the same, below 2^-17."""
    d = 2.0 ** -18
    if not t > 0:
        assert token == int(np.argmax(x)) and lp == 0
        return
    for dp in (-d, 0, d):
        for dm in (1 - d, 1, 1 + d):
            order, w = _kept(x, t, k, p if p >= 1 else max(p + dp, 0.0), min(m * dm, 1.0))
            at = np.flatnonzero(order == token)
            if len(at) == 0 or w[at[0]] == 0:
                continue
            cum = np.cumsum(w)
            after, share = cum[at[0]] / cum[-1], w[at[0]] / cum[-1]
            if after - share <= u + 2 * d and after >= u - 2 * d and abs(lp - math.log(share)) <= 2.0 ** -16:
                return
    raise AssertionError((token, lp, u, t, k, p, m))


def _settings(rng, N):
    f = lambda x: [float(np.float32(i)) for i in x]
    return (f(rng.random(N)), f(rng.choice([0.5, 0.8, 1.0, 1.5], N)), [int(i) for i in rng.choice([0, 3, 40, 500, 5000], N)],
            f(rng.choice([1.0, 0.95, 0.6, 0.999], N)), f(rng.choice([0.0, 0.0, 0.02, 0.3], N)))


@pytest.mark.parametrize("N,V,dtype", [(24, 32000, torch.float32), (24, 9001, torch.bfloat16), (12, 131072, torch.bfloat16),
                                       (40, 300, torch.float32)])
def test_kept_tokens(N, V, dtype):
    g = torch.Generator().manual_seed(V)
    x = torch.randn((N, V), generator=g) * 2
    x.scatter_add_(1, torch.randint(0, V, (N, max(1, V // 500)), generator=g), 8 * torch.rand((N, max(1, V // 500)), generator=g))
    x = x.to(dtype)
    s = _settings(np.random.default_rng(V), N)
    got, lps = _sample(x.to(DEV), *s)
    ref = x.double().numpy()
    for n in range(N):
        check_draw(ref[n], got[n], lps[n], *(i[n] for i in s))


@pytest.mark.parametrize("V", [20000, 100000])
@pytest.mark.parametrize("dtype,mask", [(torch.float32, -1e9), (torch.float32, F32_MIN), (torch.bfloat16, -1e9),
                                        (torch.bfloat16, BF16_MIN), (torch.float32, -1e5)])
def test_masks_of_finite_values(V, dtype, mask):
    """A vocabulary of which whole stretches are masked by a large negative
    number or the type's lowest, and rows in which one token or a few are left."""
    N = 16
    g = torch.Generator().manual_seed(V)
    x = torch.randn((N, V), generator=g) * 2
    x[:, 3000:V - 40] = mask
    x[4:8, :] = mask
    x[4:8, V - 7:V - 3] = torch.tensor([1.0, 3.0, 2.0, 3.0])
    x[8] = mask
    x[8, 12345] = -4.0
    x = x.to(dtype)
    rng = np.random.default_rng(V)
    s = _settings(rng, N)
    got, lps = _sample(x.to(DEV), *s)
    ref = x.double().numpy()
    for n in range(N):
        check_draw(ref[n], got[n], lps[n], *(i[n] for i in s))
    # All of one value, the lowest among them: as any other flat row.
    flat = torch.full((2, V), mask).to(dtype)
    got, lps = _sample(flat.to(DEV), [0.25, 0.75], [1.0, 1.0], [0, 4], [1.0, 1.0], [0.0, 0.0])
    assert got[0] == V // 4 and abs(lps[0] + math.log(V)) < 1e-5 * math.log(V)
    assert got[1] == 3 and abs(lps[1] + math.log(4)) < 1e-6


def test_infinite_temperature_and_infinite_logits():
    """Infinite logits share the row at any temperature, an infinite one too."""
    inf = math.inf
    x = torch.full((5, 600), 2.0)
    x[:, 100], x[:, 400] = inf, inf
    x[:, 7], x[:, 8] = -inf, math.nan
    x[4, 100] = x[4, 400] = 2.0
    got, lps = _sample(x.to(DEV), [0.25, 0.75, 0.75, 0.75, 0.5], [inf] * 5, [0, 0, 2, 0, 0], [1.0, 1.0, 1.0, 0.75, 1.0],
                       [0.0, 0.0, 0.0, 0.5, 0.0])
    assert got[:4] == [100, 400, 400, 400]
    assert all(abs(lp - math.log(0.5)) < 1e-6 for lp in lps[:4])
    assert got[4] == 301 and abs(lps[4] + math.log(598)) < 1e-6  # 598 equal tokens, 7 and 8 hidden


@pytest.mark.parametrize("sign", [-1, 1])
@pytest.mark.parametrize("t", [1.0, 3e3, 1e6, 1e12])
def test_denormal_logits(t, sign):
    """Logits of less than 2^-126, whose products with the temperature's
    reciprocal vanish: still in order, with equal weights."""
    V = 3000
    x = sign * 1e-42 * torch.rand((6, V), generator=torch.Generator().manual_seed(V))
    s = ([0.1, 0.5, 0.9, 0.3, 0.7, 0.5], [t] * 6, [0, 0, 0, 900, 2000, 0], [0.5, 0.25, 0.875, 1.0, 0.5, 1.0], [0.0] * 5 + [0.5])
    got, lps = _sample(x.to(DEV), *s)
    ref = x.double().numpy()
    for n in range(6):
        check_draw(ref[n], got[n], lps[n], *(i[n] for i in s))
