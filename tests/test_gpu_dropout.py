"""Dropout and its gradient against the definition (numpy: whole numbers for the mask, 64 bits for the values), through the C ABI.
Needs a GPU.

Tolerances.  u = 2^-24, h half a step of the type relative to the value (2^-24, 2^-8, 2^-11).
  out      v = f (x + bias): the sum, f and the product are rounded, 3 u |v|; the residual's sum another u |out|, the result h |out|
  g_x      f and the product: 2 u |v|, and h |v|
  g_bias   a sum of n terms in any order: (n + 3) u of the sum of their magnitudes
and half of the type's smallest step where it has run out of exponents.
"""
import numpy as np
import pytest

from paper_1102_0183_amd import binding

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"float32": (2.0 ** -24, 2.0 ** -149), "bfloat16": (2.0 ** -8, 2.0 ** -133), "float16": (2.0 ** -11, 2.0 ** -24)}
G = 0x9E3779B97F4A7C15
WORD = (1 << 64) - 1


def _mix64(z):
    with np.errstate(over="ignore"):
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        return z ^ (z >> np.uint64(31))


def _kept(rows, cols, p, seed, step):
    key = _mix64(np.array([(seed + G * (step + 1)) & WORD], dtype=np.uint64))
    pairs = (cols + 1) // 2
    with np.errstate(over="ignore"):
        z = _mix64(key + np.uint64(G) * np.arange(1, rows * pairs + 1, dtype=np.uint64))
    b = np.stack([z >> np.uint64(32), z & np.uint64(0xFFFFFFFF)], 1).reshape(rows, 2 * pairs)[:, :cols]
    return b >= np.uint64(round(float(np.float32(p)) * 2.0 ** 32))


def _factor(p):
    p = float(np.float32(p))
    return 1.0 / (1.0 - p) if p < 1 else 0.0


def _matrix(rows, cols, dtype, gen, pad=0, offset=0, scale=1.0):
    import torch
    wide = torch.randn(rows * (cols + pad) + offset, generator=gen, device="cuda:0").mul_(scale).to(getattr(torch, dtype))
    return wide[offset:].view(rows, cols + pad)[:, :cols]


def _np(t):
    return None if t is None else t.double().cpu().numpy()


def _near(got, want, tol, what):
    got, want = np.asarray(got), np.asarray(want)
    off = np.abs(got - want)
    assert (off <= tol).all(), (what, float((off - tol).max()))


def _check(out, x, bias, residual, p, seed, step, dtype):
    h, tiny = TYPES[dtype]
    rows, cols = x.shape
    keep = _kept(rows, cols, p, seed, step)
    v = np.where(keep, (_np(x) + (0.0 if bias is None else _np(bias))) * _factor(p), 0.0)
    want = v + (0.0 if residual is None else _np(residual))
    _near(_np(out), want, 3 * U * np.abs(v) + (h + U) * (np.abs(want) + 4 * U * np.abs(v)) + tiny, (x.shape, dtype, p))
    if residual is None:
        assert (_np(out)[~keep] == 0).all()
    else:
        assert (_np(out)[~keep] == _np(residual)[~keep]).all()
    return keep


def _check_grad(g_x, g_bias, g, p, seed, step, dtype):
    h, tiny = TYPES[dtype]
    rows, cols = g.shape
    v = np.where(_kept(rows, cols, p, seed, step), _np(g) * _factor(p), 0.0)
    if g_x is not None:
        _near(_np(g_x), v, (2 * U + h) * np.abs(v) + tiny, "g_x")
    if g_bias is not None:
        _near(_np(g_bias), v.sum(0), (rows + 3) * U * np.abs(v).sum(0) + 2.0 ** -149, "g_bias")


def _scratch(rows, cols):
    import torch
    return torch.empty(binding.dropout_grad_scratch_bytes(rows, cols), dtype=torch.uint8, device="cuda:0")


SHAPES = [(1, 1), (1, 2), (3, 1), (2, 7), (1, 8), (5, 9), (64, 150), (7, 255), (33, 256), (100, 257), (3, 2049), (1, 100003), (1001, 719), (5000, 3), (300, 4096)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_units_and_gradients_match_the_definition(rows, cols, dtype):
    import torch
    gen = torch.Generator(device="cuda:0").manual_seed(rows * 1000 + cols)
    x, bias, residual = _matrix(rows, cols, dtype, gen), _matrix(1, cols, dtype, gen)[0].contiguous(), _matrix(rows, cols, dtype, gen)
    for p, b, r in ((0.5, bias, None), (0.1, None, residual), (0.37, bias, residual), (0.9, None, None)):
        out = torch.full((rows, cols), 77.0, dtype=x.dtype, device=x.device)
        binding.dropout(x, out, p, 123456789, cols, b, r)
        _check(out, x, b, r, p, 123456789, cols, dtype)
        g_bias = torch.full((cols,), 77.0, device=x.device)
        binding.dropout_grad(x, out, p, 123456789, cols, g_bias, _scratch(rows, cols))
        _check_grad(out, g_bias, x, p, 123456789, cols, dtype)
        g_bias.fill_(77.0)
        binding.dropout_grad(x, None, p, 123456789, cols, g_bias, _scratch(rows, cols))
        _check_grad(None, g_bias, x, p, 123456789, cols, dtype)
        out.fill_(77.0)
        binding.dropout_grad(x, out, p, 123456789, cols)
        _check_grad(out, None, x, p, 123456789, cols, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,offset", [(1, 0), (3, 1), (0, 1), (5, 3), (8, 0), (7, 2)])
@pytest.mark.parametrize("rows,cols", [(5, 37), (40, 300), (9, 1031)])
def test_rows_start_anywhere_and_what_lies_between_stays(rows, cols, pad, offset, dtype):
    import torch
    gen = torch.Generator(device="cuda:0").manual_seed(cols)
    x, residual = _matrix(rows, cols, dtype, gen, pad, offset), _matrix(rows, cols, dtype, gen, 2 * pad, offset)
    wide = torch.full((offset + rows * (cols + pad + 1),), 77.0, dtype=x.dtype, device=x.device)
    out = wide[offset:].view(rows, cols + pad + 1)[:, :cols]
    binding.dropout(x, out, 0.3, 5, 6, None, residual)
    _check(out, x, None, residual, 0.3, 5, 6, dtype)
    assert (wide[offset:].view(rows, -1)[:, cols:] == 77).all() and (wide[:offset] == 77).all()
    wide.fill_(77.0)
    g_bias = torch.empty(cols, device=x.device)
    binding.dropout_grad(x, out, 0.3, 5, 6, g_bias, _scratch(rows, cols))
    _check_grad(out, g_bias, x, 0.3, 5, 6, dtype)
    assert (wide[offset:].view(rows, -1)[:, cols:] == 77).all() and (wide[:offset] == 77).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(3, 50), (200, 515)])
def test_nothing_everything_and_hardly_anything_dropped(rows, cols, dtype):
    import torch
    gen = torch.Generator(device="cuda:0").manual_seed(2)
    x, residual = _matrix(rows, cols, dtype, gen), _matrix(rows, cols, dtype, gen)
    for p in (0.0, 1.0, 1e-12, 2.0 ** -33, 2.0 ** -20, 1.0 - 2.0 ** -24, 0.999):
        out = torch.empty_like(x)
        binding.dropout(x, out, p, 1, 1, None, residual) if p < 0.9999 or dtype != "float16" else binding.dropout(x.mul(0), out, p, 1, 1, None, residual)
        if p == 0.0:
            assert torch.equal(out, (x.float() + residual.float()).to(x.dtype))
        elif p == 1.0:
            assert torch.equal(out, residual)
        elif p < 0.9999:
            _check(out, x, None, residual, p, 1, 1, dtype)
    g_bias = torch.empty(cols, device=x.device)
    binding.dropout_grad(x, out, 1.0, 1, 1, g_bias, _scratch(rows, cols))
    assert (out == 0).all() and (g_bias == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_dropped_infinities_and_nan_are_gone(dtype):
    import math
    import torch
    rows, cols, p = 40, 64, 0.5
    keep = torch.from_numpy(_kept(rows, cols, p, 3, 4)).to("cuda:0")
    x = torch.ones(rows, cols, device="cuda:0").to(getattr(torch, dtype))
    x[~keep] = math.nan
    x[:, ::3] = torch.where(keep[:, ::3], x[:, ::3], -math.inf)
    residual = torch.full_like(x, 2.0)
    out = torch.empty_like(x)
    binding.dropout(x, out, p, 3, 4, None, residual)
    assert torch.equal(out, torch.where(keep, 4.0, 2.0).to(x.dtype))
    g_bias = torch.empty(cols, device="cuda:0")
    binding.dropout_grad(x, out, p, 3, 4, g_bias, _scratch(rows, cols))
    assert torch.equal(out, torch.where(keep, 2.0, 0.0).to(x.dtype)) and torch.equal(g_bias, 2.0 * keep.float().sum(0))
    x[keep] = math.nan   # and kept ones stay
    binding.dropout(x, out, p, 3, 4)
    assert torch.equal(torch.isnan(out), keep)


@pytest.mark.parametrize("dtype", TYPES)
def test_in_place(dtype):
    import torch
    gen = torch.Generator(device="cuda:0").manual_seed(2)
    x, residual = _matrix(70, 301, dtype, gen), _matrix(70, 301, dtype, gen)
    want = torch.empty_like(x)
    binding.dropout(x, want, 0.4, 8, 9, None, residual)
    a, b = x.clone(), residual.clone()
    binding.dropout(a, a, 0.4, 8, 9, None, residual)
    binding.dropout(x, b, 0.4, 8, 9, None, b)
    assert torch.equal(a, want) and torch.equal(b, want)
    binding.dropout_grad(x, want, 0.4, 8, 9)
    a = x.clone()
    binding.dropout_grad(a, a, 0.4, 8, 9)
    assert torch.equal(a, want)


def test_the_mask_depends_on_the_numbers_alone():
    """Another type, another stride, other rows behind the same ones: the same mask; another seed, step or width: another one."""
    import torch
    ones = torch.ones(100, 333, device="cuda:0")

    def mask(x, seed=1 << 63, step=(1 << 64) - 2, p=0.5, d_step=None):
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        binding.dropout(x, out, p, seed, step, d_step=d_step)
        return out != 0
    a = mask(ones)
    assert np.array_equal(a.cpu().numpy(), _kept(100, 333, 0.5, 1 << 63, (1 << 64) - 2))
    assert torch.equal(a, mask(ones.bfloat16())) and torch.equal(a, mask(torch.ones(100, 400, device="cuda:0").half()[:, :333]))
    assert torch.equal(a[:31], mask(ones[:31]))
    two = torch.tensor([2], device="cuda:0")
    assert torch.equal(a, mask(ones, step=(1 << 64) - 4, d_step=two))
    # (333 and 334 columns have 167 pairs a row, and so the same draws; 335 have 168)
    assert torch.equal(a, mask(torch.ones(100, 334, device="cuda:0"))[:, :333])
    for other in (mask(ones, seed=2), mask(ones, step=0), mask(ones, step=1), mask(torch.ones(100, 335, device="cuda:0"))[1:, :333]):
        assert abs((a[-len(other):] != other).float().mean().item() - 0.5) < 0.02      # 33300 tosses: 7 standard deviations are 0.019
    kept = mask(torch.ones(1000, 1000, device="cuda:0"), p=0.3).float()
    assert abs(kept.mean().item() - 0.7) < 0.0033      # 7 standard deviations of a million tosses
    assert (kept.mean(0) - 0.7).abs().max() < 0.11 and (kept.mean(1) - 0.7).abs().max() < 0.11


def test_gradients_agree_with_differences():
    """The pass is linear in its units, bias and residual: a difference of two passes is the gradient, but for roundings."""
    import torch
    gen = torch.Generator(device="cuda:0").manual_seed(6)
    x, bias, g = _matrix(20, 31, "float32", gen), _matrix(1, 31, "float32", gen)[0].contiguous(), _matrix(20, 31, "float32", gen)
    g_x, g_bias = torch.empty_like(x), torch.empty(31, device="cuda:0")
    binding.dropout_grad(g, g_x, 0.25, 77, 3, g_bias, _scratch(20, 31))

    def error(x, bias):
        out = torch.empty_like(x)
        binding.dropout(x, out, 0.25, 77, 3, bias)
        return (out.double() * g.double()).sum().item()
    base = error(x, bias)
    for at in range(0, 20 * 31, 37):
        y = x.clone()
        y.view(-1)[at] += 0.5
        # two sums of 620 products of some 4 each in 64 bits, of outputs rounded to 2^-24 of values up to 6
        assert abs((error(y, bias) - base) / 0.5 - g_x.view(-1)[at].item()) < 620 * 6 * 6 * 2 * 2.0 ** -23
    for c in range(0, 31, 5):
        y = bias.clone()
        y[c] += 0.5
        assert abs((error(x, y) - base) / 0.5 - g_bias[c].item()) < 620 * 6 * 6 * 2 * 2.0 ** -23


def test_no_rows_have_a_bias_gradient_of_zero():
    import torch
    g_bias = torch.full((100,), 7.0, device="cuda:0")
    g = torch.empty(0, 100, device="cuda:0")
    binding.dropout_grad(g, None, 0.5, 1, 1, g_bias, _scratch(0, 100))
    assert (g_bias == 0).all()


def test_captured_and_replayed_with_other_steps():
    import torch
    gen = torch.Generator(device="cuda:0").manual_seed(4)
    rows, cols = 700, 130
    x, out, g_x, g_bias = _matrix(rows, cols, "bfloat16", gen), *(torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda:0") for _ in range(2)), torch.empty(cols, device="cuda:0")
    at, scratch = torch.zeros(1, dtype=torch.int64, device="cuda:0"), _scratch(rows, cols)

    def both():
        binding.dropout(x, out, 0.2, 9, 1000, d_step=at)
        binding.dropout_grad(x, g_x, 0.2, 9, 1000, g_bias, scratch, d_step=at)
    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for step in (0, 1, 5, 1 << 40):
        at.fill_(step)
        graph.replay()
        torch.cuda.synchronize()
        _check(out, x, None, None, 0.2, 9, 1000 + step, "bfloat16")
        _check_grad(g_x, g_bias, x, 0.2, 9, 1000 + step, "bfloat16")


def test_the_same_call_gives_the_same_bits_on_any_stream():
    import torch
    gen = torch.Generator(device="cuda:0").manual_seed(4)
    g = _matrix(3000, 517, "float16", gen)
    g_x, want = torch.empty_like(g), torch.empty(517, device="cuda:0")
    binding.dropout_grad(g, g_x, 0.2, 9, 1, want, _scratch(3000, 517))
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    keep = []
    for st in streams * 2:
        keep.append((torch.empty_like(g), torch.empty(517, device="cuda:0"), _scratch(3000, 517)))
        torch.cuda.synchronize()
        binding.dropout_grad(g, keep[-1][0], 0.2, 9, 1, keep[-1][1], keep[-1][2], stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(a, g_x) and torch.equal(b, want) for a, b, _ in keep)


def test_rows_beyond_32_bits():
    """Elements further than 2^32 into a matrix: the last rows of a wide one."""
    import torch
    rows, cols, stride = 5, 40, (1 << 30) + 8
    x = torch.empty((rows - 1) * stride + cols, dtype=torch.bfloat16, device="cuda:0")
    x = x.as_strided((rows, cols), (stride, 1))
    gen = torch.Generator(device="cuda:0").manual_seed(4)
    x.copy_(torch.randn(rows, cols, generator=gen, device="cuda:0"))
    out = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda:0")
    binding.dropout(x, out, 0.5, 1, 2)
    _check(out, x, None, None, 0.5, 1, 2, "bfloat16")
    binding.dropout(out, x, 0.0, 1, 2)
    assert torch.equal(x, out)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(200, 515), (31, 4000)])
def test_the_largest_share_below_all_of_them(rows, cols, dtype):
    """p = 1 - 2^-24: 256 numbers of 2^32 keep a unit, times 2^24.  Steps whose masks keep one, some or none, found by the definition."""
    import torch
    p, seed = 1.0 - 2.0 ** -24, 77
    gen = torch.Generator(device="cuda:0").manual_seed(rows)
    x, residual, bias = (_matrix(n, cols, dtype, gen, scale=2.0 ** -14) for n in (rows, rows, 1))
    bias = bias[0].contiguous()
    kept = [int(_kept(rows, cols, p, seed, step).sum()) for step in range(400)]
    some = [s for s in range(400) if kept[s]]
    assert some and _factor(p) == 2.0 ** 24
    out, g_bias = torch.empty_like(x), torch.empty(cols, device=x.device)
    for step in some[:3] + [kept.index(0)]:
        binding.dropout(x, out, p, seed, step)
        _check(out, x, None, None, p, seed, step, dtype)
        binding.dropout(x, out, p, seed, step, bias, residual)
        _check(out, x, bias, residual, p, seed, step, dtype)
        binding.dropout_grad(x, out, p, seed, step, g_bias, _scratch(rows, cols))
        _check_grad(out, g_bias, x, p, seed, step, dtype)
        assert int((out != 0).sum()) == kept[step]
