"""Classes drawn where a row's values, its number of classes left or its masses fall on a border of the kernels' own: the definition in 64
bits of test_gpu_draws, and its tolerances.  Needs a GPU."""
import math

import pytest

from tests.test_gpu_draws import TYPES, _call, _check

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


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,k,block", [(1500, 180, 8), (4000, 300, 8), (16000, 900, 16), (20000, 700, 16), (20000, 1100, 16), (50001, 700, 32), (50001, 1000, 32)])
def test_as_many_classes_from_a_value_on_as_top_k_asks_for(n, k, block, dtype):
    """k classes above the others, one in a block of neighbours each, its last: the list of candidates is what is left, and the block's others are
    not.  With one class more or less asked for, and with a min-p that leaves all of them."""
    import torch
    rows = 24
    x = torch.full((rows, n), 9.5, device="cuda:0")
    high = torch.arange(k, device="cuda:0") * block + block - 1
    x[:, high] = 10.0
    x[rows // 2:, high] += torch.arange(k, device="cuda:0") % 7 * 0.0625   # (the same in all three types)
    x = x.to(getattr(torch, dtype))
    u = (torch.arange(rows, device="cuda:0").float() + 0.37) / rows
    for s in ({"k": [k] * rows}, {"k": [k + 1 - r % 3 for r in range(rows)]}, {"k": [k] * rows, "q": [0.1] * rows}, {"k": [k] * rows, "p": [0.5 + 0.02 * r for r in range(rows)]}):
        _check(x, u, **s)
