"""Classes drawn where a row's values, its number of classes left or its masses fall on a border of the kernels' own: the definition in 64
bits of test_gpu_draws, and its tolerances.  Needs a GPU."""
import math

import numpy as np
import pytest

from paper_1102_0183_amd import binding
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


def _weights(x):
    """exp(x) for x <= 0 as the kernels sum it up: a power of two out of 256 and three terms of the series, each rounded to 64 bits."""
    L, t = math.log(2.0) / 256, np.maximum(np.asarray(x, np.float64), -900.0)
    z = t.astype(np.longdouble) * np.longdouble(256.0 * 1.4426950408889634074)
    k = np.rint(z)
    f, series = z - k, np.full(t.shape, L ** 3 / 6)
    for term in (L * L / 2, L, 1.0):
        series = (series.astype(np.longdouble) * f + np.longdouble(term)).astype(np.float64)
    k = k.astype(np.int64)
    return (t >= -700) * np.ldexp(np.exp2((k & 255) / 256.0), k >> 8) * series


def _next_to_a_border(x, left, spare, rows, step):
    """(rows of x with two classes, `spare`, changed, p): p times the mass of a row is the mass of its `left` largest, but for so many `step`s."""
    w = _weights(x)
    w[list(spare)] = 0.0
    prefix, rest = math.fsum(np.sort(w)[::-1][:left]), math.fsum(w)
    p = np.float32(prefix / (rest + 3e-5))
    while prefix / float(p) <= rest:
        p = np.nextafter(p, np.float32(0))
    out = np.repeat(x[None], rows, 0)
    for i in range(rows):
        want = (prefix + (i - rows // 2) * step) / float(p) - rest
        a = np.float32(math.log(want))
        while _weights([a])[0] >= want:
            a = np.nextafter(a, np.float32(-np.inf))
        out[i, spare[0]], out[i, spare[1]] = a, np.float32(math.log(want - _weights([a])[0]))
    return out, float(p)


@pytest.mark.parametrize("many,seed", [(410, 2), (410, 10), (500, 5), (500, 7), (900, 0), (900, 1), (900, 3), (900, 10)])
def test_a_border_within_rounding_between_two_lists_of_a_flat_row(many, seed):
    """Top-p of p times the mass of exactly the 9500 largest of 20000 classes, to a rounding: hundreds of classes close above the border and hundreds
    close below, with a gap between them, so that the kernel looks at the two sides one after the other and its sums may contradict each other.
    Drawn is one of the 9500, or of one class more (a border within rounding may fall on either side)."""
    import torch
    rows, draws, n, left = 16, 32, 20000, 9500
    g = np.random.default_rng(seed)
    above, below = -(19 + 63.5 * 3 / 128) / 16 + np.linspace(-4e-4, 4e-4, many), -(19 + 66.5 * 3 / 128) / 16 + np.linspace(-4e-4, 4e-4, 390)
    rest = np.concatenate([[0.0], g.uniform(-1.2, 0, left - many - 1), above, below, g.uniform(-2, -1.4, n - 16 - left - 390)]).astype(np.float32)
    x = np.concatenate([np.full(16, -2.0, np.float32), g.permutation(rest)])
    spare = [i for i in np.argsort(x) if i >= 16][:2]
    x, p = _next_to_a_border(x, left, spare, rows, np.spacing(5000.0))
    x = torch.from_numpy(x).to("cuda:0").repeat_interleave(draws, 0)
    u = torch.from_numpy(g.random(rows * draws).astype(np.float32)).to("cuda:0")
    out, lp = _call(x, u, p=[p] * (rows * draws))
    border = torch.sort(x[0], descending=True)[0][left]
    drawn = x.gather(1, out.long()[:, None])[:, 0]
    # the log probability of it among the 9500, or the 9501: 5e-5 apart
    w = torch.sort(x.double().exp(), 1, descending=True)[0]
    mass = w[:, :left].sum(1)
    off = torch.stack([lp.double() - (drawn.double() - m.log()) for m in (mass, mass + w[:, left])]).abs().min(0)[0]
    assert (off <= 2.0 ** -24 * lp.double().abs() + 1e-12).all()
    assert (drawn >= border).all(), (torch.nonzero(drawn < border)[:, 0] // draws, drawn[drawn < border], border)


@pytest.mark.parametrize("n,block,live,left,k", [(9000, 8, 900, 450, 0), (9000, 8, 600, 400, 600), (20000, 16, 1200, 700, 0), (20000, 16, 700, 350, 700),
                                                 (20000, 16, 1200, 650, 900), (50001, 32, 1500, 800, 0), (50001, 32, 900, 500, 900)])
def test_equal_rows_draw_the_same_next_to_a_border_of_rounding(n, block, live, left, k):
    """Lists of hundreds of classes come together in any order; their masses do not depend on it.  Rows of which top-p is to leave exactly `left`
    classes, to a rounding, many times over in one call and in calls after each other: the same bits in all of them."""
    import torch
    rows, copies = 12, 20 if n > 40000 else 300
    g = np.random.default_rng(n + live)
    x, at = np.full(n, -np.inf, np.float32), g.permutation(n // block)[:live] * block + g.integers(0, block, live)   # (one in a block of neighbours)
    x[at] = g.uniform(-3, 0, live)
    x[at[0]] = 0.0
    x, p = _next_to_a_border(x, left, at[np.argsort(x[at])[:2]], rows, np.spacing(_weights(x).sum()) / 2)
    x = torch.from_numpy(x).to("cuda:0").repeat_interleave(copies, 0)
    u = torch.full((rows * copies,), 0.43, device="cuda:0")
    first = None
    for _ in range(20):
        out, lp = _call(x, u, p=[p] * (rows * copies), k=[k] * (rows * copies))
        got = torch.stack([out, lp.view(torch.int32)]).view(2, rows, copies)
        first = got[:, :, :1].clone() if first is None else first
        assert (got == first).all(), [(got[:, r] != first[:, r]).sum().item() for r in range(rows)]


def test_arrays_that_classes_of_images_are_not_drawn_with():
    """Misaligned arrays, and results over what the call reads, are refused as cnn_draw_classes refuses them; nothing is written."""
    import torch
    net = binding.Cnn("1x12x12-4C3-MP2-30N-200N")
    rng = np.random.default_rng(1)
    net.set_weights(rng.uniform(-0.08, 0.08, net.num_weights).astype(np.float32))
    n = 6
    images = torch.from_numpy(rng.uniform(-1, 1, (n, net.image_size)).astype(np.float32)).to("cuda:0")
    scratch = torch.zeros(net.forward_batch_scratch_bytes(n), dtype=torch.uint8, device="cuda:0")
    words = torch.zeros(7 * 64, dtype=torch.int32, device="cuda:0")
    keep = images.clone()
    T, k, p, q, u, out, lp = (words.data_ptr() + 256 * i for i in range(7))
    words.view(torch.float32)[:64] = 1.0   # (T)

    def call(x=images.data_ptr(), T=T, k=k, p=None, q=q, u=u, out=out, lp=lp, scratch=scratch):
        torch.cuda.synchronize()
        return binding.lib().cnn_draw_batch(net._h, x, n, T, k, p, q, u, out, lp, scratch.data_ptr(), scratch.numel(), n)
    before = words.clone()
    for kw in (dict(u=None), dict(out=None), dict(T=T + 2), dict(k=k + 1), dict(p=p + 3), dict(q=q + 2), dict(u=u + 1), dict(out=out + 2), dict(lp=lp + 2),
               dict(out=u), dict(out=u + 4 * (n - 1)), dict(out=k - 4), dict(lp=out), dict(lp=out - 4), dict(lp=T), dict(out=images.data_ptr()),
               dict(lp=images.data_ptr() + 4 * (images.numel() - 1)), dict(out=scratch.data_ptr()), dict(lp=scratch.data_ptr() + scratch.numel() - 4)):
        assert call(**kw) == binding.E_ARG, kw
        assert "cnn_draw_batch" in binding._err(net._h), kw
    net.synchronize()
    assert torch.equal(words, before) and torch.equal(images, keep)
    assert call() == 0 and call(lp=None) == 0 and call(lp=out + 4 * n) == 0
    net.synchronize()
    assert (words.view(7, 64)[5, :n] >= 0).all()
    net.close()
