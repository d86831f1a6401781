"""Classes drawn where a row's values, its number of classes left or its masses fall on a border of the kernels' own: the definition in 64
bits of test_gpu_draws, and its tolerances.  Needs a GPU."""
import math

import pytest

from tests.test_gpu_draws import TYPES, _call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [64, 65, 200, 512, 513, 700, 1024, 1025, 5000])
def test_a_nan_in_any_class_of_a_row_below_zero(n, dtype):
    """Whichever lane holds the NaN, the row is no empty one: class -1 and a log probability that is NaN."""
    import torch
    places = sorted({p for p in (0, 7, 8, 9, n // 2, 511, 512, 519, 520, n - 2, n - 1) if p < n})
    for rest in (-math.inf, -3.0, torch.finfo(getattr(torch, dtype)).min):
        x = torch.full((len(places) + 1, n), rest, device="cuda:0").to(getattr(torch, dtype))
        for row, p in enumerate(places):
            x[row, p] = math.nan
        out, lp = _call(x, torch.full((len(places) + 1,), 0.5, device="cuda:0"))
        assert (out[:-1] == -1).all() and torch.isnan(lp[:-1]).all(), (n, rest, places, lp.tolist())
        assert (lp[-1].item() == -math.inf) == (rest == -math.inf) and not math.isnan(lp[-1].item())
