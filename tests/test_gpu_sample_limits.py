"""nacl_sample at the ends of its settings' ranges."""

import math

import pytest
import torch

nacl = pytest.importorskip("paper_2408_03675_amd.nacl")
from test_gpu_sample import DEV, _sample

pytestmark = pytest.mark.gpu


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
