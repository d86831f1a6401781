"""Scores of classes and their gradient against the definition in 64 bits (on the CPU), through the C ABI.  Needs a GPU.

Tolerances.  u = 2^-24, half a step of fp32.  A lane adds at most `n` terms one after the other (the row's classes over the
lanes that share it), all of one sign, each exponential off by a few u and by |d| u for its exponent, and lanes, wavefronts
and parts are joined in at most 20 more roundings: s and t are off by (n + 100) u relative to themselves.  From that
  log s    (n + 100) u, and its own rounding
  log p    that, a rounding of x - m and one of the difference: 2 u (|x - m| + |log s|)
  entropy  log s - t / s: (n + 100) u (1 + log s + 2 H)
  p        exp of log p: u (3 |log p| + |log s| + 10) of p, the normaliser taken as given
"""
import math

import numpy as np
import pytest

from paper_1102_0183_amd import binding

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = ["float32", "bfloat16", "float16"]


def _reference(x, labels, top):
    """(log p of the labels, entropy, m, S, indices, their log p) of rows of float64, numpy."""
    rows, n = x.shape
    with np.errstate(all="ignore"):
        none = np.isnan(x).any(1) | (x == np.inf).any(1)
        m = x.max(1)
        empty = m == -np.inf
        d = x - np.where(empty, 0.0, m)[:, None]
        e = np.exp(d)
        S = np.log(e.sum(1))
        log_p = np.where(empty[:, None], -np.inf, d - S[:, None])
        H = np.where(empty, 0.0, -np.where(e > 0, np.exp(log_p) * log_p, 0.0).sum(1))
        order = np.argsort(-x, axis=1, kind="stable")[:, :top]
    top_lp = np.take_along_axis(log_p, order, 1)
    lp = np.array([log_p[r, l] if 0 <= l < n else 0.0 for r, l in enumerate(labels)])
    nan = np.full(rows, np.nan)
    has = np.array([0 <= l < n for l in labels])
    return (np.where(none & has, nan, lp), np.where(none, nan, H), np.where(none, nan, m), np.where(none, nan, S),
            np.where(none[:, None], -1, order), np.where(none[:, None], np.nan, top_lp))


def _call(x, labels, top, want=("lp", "h", "norm", "top", "top_lp"), stream=None, scratch=None):
    import torch
    rows, n = x.shape
    f = lambda *s: torch.full(s, 77.0, dtype=torch.float32, device=x.device)  # noqa: E731
    out = {"lp": f(rows), "h": f(rows), "norm": f(rows, 2), "top": torch.full((rows, top), 77, dtype=torch.int32, device=x.device), "top_lp": f(rows, top)}
    if scratch is None:
        scratch = torch.empty(binding.class_scores_scratch_bytes(rows, n, top), dtype=torch.uint8, device=x.device)
    got = {k: (v if k in want else None) for k, v in out.items()}
    binding.class_scores(x, labels, got["lp"], got["h"], got["norm"], got["top"], got["top_lp"], scratch, stream)
    return out


def _terms(rows, n):
    """Terms that one lane adds at most: one wavefront a row up to 8192 classes, or 32768 of many rows, else four or more, and one more
    tile where a row starts oddly."""
    if n <= 64:
        return 1
    return 16 * (math.ceil(math.ceil(n / 1024) / (1 if n <= 8192 or (rows >= 4096 and n <= 32768) else 4)) + 1)


def _check(x, labels, top, out):
    """Every output against the definition, for a device matrix x."""
    rows, n = x.shape
    lp, H, m, S, order, top_lp = _reference(x.double().cpu().numpy(), labels.cpu().numpy(), top)
    g = {k: v.cpu().numpy().astype(np.float64) if v.dtype.is_floating_point else v.cpu().numpy() for k, v in out.items()}
    a = (_terms(rows, n) + 100) * U
    S0 = np.where(np.isfinite(S), np.abs(S), 0.0)

    def near(got, want, tol, what):
        with np.errstate(over="ignore"):
            want = np.where(np.isinf(want.astype(np.float32)), want.astype(np.float32), want)   # (lowest - largest: no float holds it)
        fine = np.isfinite(want)
        np.testing.assert_array_equal(np.isnan(got), np.isnan(want), err_msg=what)
        np.testing.assert_array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)], err_msg=what)
        off = np.abs(got[fine] - want[fine])
        assert (off <= np.broadcast_to(tol, want.shape)[fine]).all(), (what, off.max() if off.size else 0, x.shape, x.dtype)

    near(g["norm"][:, 0], m, 0.0, "m")
    near(g["norm"][:, 1], S, a + U * S0, "S")
    near(g["lp"], lp, a + 2 * U * (np.abs(lp) + 2 * S0), "log p")
    near(g["h"], H, a * (1 + S0 + 2 * np.abs(H)), "entropy")
    np.testing.assert_array_equal(g["top"], order)
    near(g["top_lp"], top_lp, a + 2 * U * (np.abs(top_lp) + 2 * S0[:, None]), "log p of the best")


def _rows(rows, n, dtype, seed, pad=0, offset=0):
    import torch
    gen = torch.Generator(device="cuda:0").manual_seed(seed)
    wide = torch.randn(rows * (n + pad) + offset, generator=gen, device="cuda:0").mul_(3).to(getattr(torch, dtype))
    x = wide[offset:].view(rows, n + pad)[:, :n]
    labels = torch.randint(0, n, (rows,), generator=gen, device="cuda:0", dtype=torch.int32)
    return x, labels


SHAPES = [(1, 1, 1), (1, 2, 2), (3, 5, 5), (33, 10, 3), (2, 16, 16), (5, 33, 7), (1, 64, 64), (67, 64, 1), (2, 65, 64), (7, 100, 20),
          (9, 1000, 5), (3, 1023, 64), (3, 1024, 1), (2, 1025, 30), (5, 2049, 8), (2, 4096, 64), (3, 4097, 64), (1, 5000, 64), (2, 8193, 3),
          (1, 20001, 20), (600, 5001, 2), (3, 131073, 64), (1, 300007, 33)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n,top", SHAPES)
def test_scores_match_the_definition(rows, n, top, dtype):
    x, labels = _rows(rows, n, dtype, 17 * n + rows)
    _check(x, labels, top, _call(x, labels, top))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,offset", [(1, 0), (3, 1), (0, 1), (5, 3), (7, 2)])
@pytest.mark.parametrize("rows,n,top", [(5, 37, 4), (4, 1500, 9), (3, 9001, 20)])
def test_rows_start_anywhere(rows, n, top, pad, offset, dtype):
    x, labels = _rows(rows, n, dtype, 5, pad, offset)
    _check(x, labels, top, _call(x, labels, top))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [10, 64, 200, 3000, 20000, 90000])
def test_masked_classes_empty_rows_lowest_values_infinities_and_nan(n, dtype):
    import torch
    x, labels = _rows(12, n, dtype, 3)
    low = torch.finfo(x.dtype).min
    x[0] = -math.inf                          # nothing left
    x[1] = low                                # all equal, the lowest there is
    x[2, 1:] = -math.inf                      # one class left
    x[3, : n // 2] = -math.inf
    labels[3] = 0                             # the label's class is off
    x[4, ::3] = low
    x[5, n // 2] = math.inf
    x[6, n - 1] = math.nan
    x[7] = -math.inf
    x[7, n - 1] = math.nan                    # nothing else
    x[8] = torch.finfo(x.dtype).max
    x[8, 0] = low
    labels[9] = -1
    labels[10] = n
    labels[11] = -2 ** 31
    for top in {1, min(n, 20), min(n, 64)}:
        _check(x, labels, top, _call(x, labels, top))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [50, 700, 5000, 70001])
def test_ties_go_to_the_lower_index_and_order_does_not_matter(n, dtype):
    """Constant rows, rows that rise and fall, few values, zeros of both signs, the best at both ends."""
    import torch
    t = getattr(torch, dtype)
    i = torch.arange(n, device="cuda:0")
    rows = [torch.zeros(n, device="cuda:0"), i / n, -i / n, (i % 7).float(), ((i * 7919) % n).float() / n * 4,
            torch.where(i % 2 == 0, -0.0, 0.0), (i == n - 1).float(), (i == 0).float(), (i // (n // 3)).float(), torch.full((n,), -3.0, device="cuda:0")]
    x = torch.stack(rows).to(t)
    labels = torch.full((len(rows),), n - 1, dtype=torch.int32, device="cuda:0")
    for top in (1, 13, 50 if n == 50 else 64):
        _check(x, labels, top, _call(x, labels, top))


def _sampled(x, labels, top, out, at):
    """_check of a few rows."""
    import torch
    i = torch.tensor(sorted(set(at)), device="cuda:0")
    _check(x[i], labels[i], top, {k: v[i] for k, v in out.items()})


@pytest.mark.parametrize("rows,n,top,dtype", [
    (4100, 100, 20, "bfloat16"), (5000, 40, 16, "float32"), (4097, 300, 12, "float16"), (4099, 128, 64, "float32"), (4096, 64, 64, "bfloat16"),
    (4096, 8300, 3, "bfloat16"), (4097, 32768, 20, "float16"), (4097, 33000, 64, "bfloat16"), (5000, 5000, 1, "float32"), (9000, 16, 16, "float16"),
])
def test_many_rows(rows, n, top, dtype):
    x, labels = _rows(rows, n, dtype, n, pad=n % 2)
    x[rows // 3, 1:] = -math.inf
    x[rows // 2, 3] = math.nan
    _sampled(x, labels, top, _call(x, labels, top), [0, 1, rows // 3, rows // 2, rows - 2, rows - 1] + list(range(5, rows, rows // 9)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n,top", [(1, 2, 0), (2, 16, 0), (70, 10, 3), (5, 16, 16), (9, 33, 20), (3, 64, 64), (7, 100, 20), (300, 300, 0), (4, 1000, 5),
                                        (3, 1016, 64), (2, 65, 1), (5000, 700, 30)])
def test_rows_that_are_nearly_sure_keep_the_digits_of_small_logarithms(rows, n, top, dtype):
    """log p of the best class, -log(1 + R), R the sum of the others' e^-g.  A term is off by 2.5 U g (its difference, its product) and 2 U,
    their sum by 22 U, the logarithm by 4 U and the share of R by 5 U: (2.5 g + 36) U in all."""
    import torch
    gen = torch.Generator(device="cuda:0").manual_seed(n)
    gap = torch.rand(rows, n, generator=gen, device="cuda:0") * 10 + 8
    x = (-gap).to(getattr(torch, dtype))
    best = torch.randint(0, n, (rows,), generator=gen, device="cuda:0", dtype=torch.int32)
    x[torch.arange(rows), best.long()] = 0.25
    out = _call(x, best, top)
    d = x.double().cpu().numpy()
    g = 0.25 - d
    for r, b in enumerate(best.tolist()):
        d[r, b] = -np.inf
    want = -np.log1p(np.exp(d - 0.25).sum(1))
    tol = np.abs(want) * (2.5 * g.max() + 36) * U
    assert (np.abs(out["lp"].cpu().numpy() - want) <= tol).all()
    assert (np.abs(out["norm"][:, 1].cpu().numpy() + want) <= tol).all()
    if top:
        assert torch.equal(out["top"][:, 0], best) and torch.equal(out["top_lp"][:, 0], out["lp"])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n,top", [(1, 9217, 64), (2, 8192, 64), (5, 65536, 20), (3, 65537, 20), (37, 50003, 25), (128, 66001, 20), (127, 66001, 20),
                                        (200, 100003, 64), (256, 30011, 8), (257, 30011, 8), (40, 102401, 0), (1, 102399, 0), (512, 8000, 5), (513, 8000, 5)])
def test_few_long_rows(rows, n, top, dtype):
    """Rows that one, four or eight wavefronts share, and parts of them, on both sides of the rules' edges."""
    x, labels = _rows(rows, n, dtype, n + rows, pad=n % 3)
    at = sorted({0, rows - 1, rows // 3, rows // 2})
    if rows > 4:
        x[rows // 3, 1:] = -math.inf
        x[rows // 2, n - 1] = math.nan
        x[1, ::2] = -math.inf
        x[2] = x[2, 0].item()
        at = sorted(set(at) | {1, 2, rows - 2})
    _sampled(x, labels, top, _call(x, labels, top), at)


@pytest.mark.parametrize("rows,n,top,dtype", [
    ((1 << 28) + 77, 2, 1, "float16"),          # more rows than a launch has places for, in every kernel
    ((1 << 24) + 9, 10, 9, "bfloat16"),
    ((1 << 22) + 5, 1030, 9, "bfloat16"),
    ((1 << 20) + 3, 4100, 0, "bfloat16"),
])
def test_more_rows_than_a_launch_holds(rows, n, top, dtype):
    """Rows go on behind the last workgroup; their places pass 32 bits.  (Rows repeat 65536 different ones.)"""
    import torch
    some, l = _rows(65536 + 1, n, dtype, 3)
    x = torch.empty(rows, n, dtype=some.dtype, device="cuda:0")
    for a in range(0, rows, some.shape[0]):
        x[a:a + some.shape[0]] = some[:rows - a]
    labels = l.repeat(-(-rows // some.shape[0]))[:rows].contiguous()
    out = _call(x, labels, top)
    at = [0, 1, rows - 1, rows - 2, rows // 2, (rows // 4) | 1, rows - 70000 if rows > 70000 else 3]
    _sampled(x, labels, top, out, at)
    first = _call(some[:1000].contiguous(), l[:1000].contiguous(), top)
    k = (rows // some.shape[0] - 1) * some.shape[0]
    there, here = out["lp"][k:k + 1000], first["lp"]      # (the sums in another order, it may be)
    assert ((there - here).abs() <= 2 * (_terms(rows, n) + 100) * U * (2 + 2 * math.log(n) + here.abs())).all()


@pytest.mark.parametrize("n,top", [(700, 5), (5000, 20)])
def test_rows_that_lie_far_apart(n, top):
    """Offsets beyond 32 bits, of elements and of bytes."""
    import torch
    stride = (1 << 31) + 3
    wide = torch.empty(stride + n, dtype=torch.bfloat16, device="cuda:0")
    x = wide.as_strided((2, n), (stride, 1))
    x.copy_(_rows(2, n, "bfloat16", 6)[0])
    labels = torch.tensor([n - 1, 3], dtype=torch.int32, device="cuda:0")
    _check(x, labels, top, _call(x, labels, top))
    g = torch.randn(2, 2, device="cuda:0")
    _check_grad(x, labels, g[0].contiguous(), g[1].contiguous(), x)      # in place


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shift", [-30000.0, 500.0, 65000.0])
@pytest.mark.parametrize("n", [12, 3000, 9000, 40000])
def test_a_shift_of_all_classes_is_not_seen(n, shift, dtype):
    """Large values of one sign: what is rounded is their difference."""
    import torch
    x, labels = _rows(4, n, "float32", n)
    x = (x + shift).clamp(-65504, 65504).to(getattr(torch, dtype))
    x[1, : n // 2] = shift
    _check(x, labels, 5, _call(x, labels, 5))
    _check_grad(x, labels, torch.ones(4, device="cuda:0"), torch.ones(4, device="cuda:0"))


@pytest.mark.parametrize("n", [20, 3000, 50000])
def test_each_output_alone_and_nothing_behind_the_last_row(n):
    """(Sums may be added in another order where fewer outputs are asked for: each call has the tolerance of all.)"""
    import torch
    x, labels = _rows(3, n, "bfloat16", 9)
    every = _call(x, labels, 4)
    for k in every:
        out = _call(x, labels, 4, want=(k,))
        assert all((v == 77).all() for j, v in out.items() if j != k)
        _check(x, labels, 4, {**every, k: out[k]})
        again = _call(x, labels, 4, want=(k,))
        assert torch.equal(out[k], again[k])
    # rows of a larger buffer: what lies behind stays
    big = {k: torch.full((8,) + tuple(v.shape[1:]), 55, dtype=v.dtype, device=v.device) for k, v in every.items()}
    cut = {k: v[:3] for k, v in big.items()}
    scratch = torch.empty(binding.class_scores_scratch_bytes(3, n, 4), dtype=torch.uint8, device="cuda:0")
    binding.class_scores(x, labels, cut["lp"], cut["h"], cut["norm"], cut["top"], cut["top_lp"], scratch)
    for k, v in big.items():
        assert torch.equal(v[:3], every[k]) and (v[3:] == 55).all()


def test_two_streams_a_captured_call_and_the_same_bits_again():
    import torch
    x, labels = _rows(3, 60000, "float16", 4)
    y, labels_y = _rows(9, 70, "float32", 5)
    want_x, want_y = _call(x, labels, 11), _call(y, labels_y, 11)
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(s1):
            a = _call(x, labels, 11, stream=s1)
        with torch.cuda.stream(s2):
            b = _call(x, labels, 11, stream=s2)
            c = _call(y, labels_y, 11, stream=s2)
        torch.cuda.synchronize()
        for k in want_x:
            assert torch.equal(a[k], want_x[k]) and torch.equal(b[k], want_x[k]) and torch.equal(c[k], want_y[k])
    # captured: replayed on other values in the same places
    g = torch.cuda.CUDAGraph()
    scratch = torch.empty(binding.class_scores_scratch_bytes(3, 60000, 11), dtype=torch.uint8, device="cuda:0")
    held = {k: torch.empty_like(v) for k, v in want_x.items()}
    with torch.cuda.graph(g):
        binding.class_scores(x, labels, held["lp"], held["h"], held["norm"], held["top"], held["top_lp"], scratch)
    for seed in (4, 21, 22, 23):
        x.copy_(_rows(3, 60000, "float16", seed)[0])
        g.replay()
        torch.cuda.synchronize()
        _check(x, labels, 11, held)
        eager = _call(x, labels, 11)
        assert all(torch.equal(eager[k], held[k]) for k in held)


def _grad_reference(x, labels, m, S, H, g_lp, g_h):
    rows, n = x.shape
    with np.errstate(all="ignore"):
        log_p = (x - m[:, None]) - S[:, None]
        p = np.exp(log_p)
        g = -g_lp[:, None] * p - np.where(p > 0, g_h[:, None] * p * (log_p + H[:, None]), np.where(np.isnan(p), np.nan, 0.0))
        size = np.abs(g_lp)[:, None] * p + np.where(p > 0, np.abs(g_h[:, None]) * p * (np.abs(log_p) + H[:, None]), 0.0)
    for r, l in enumerate(labels):
        if 0 <= l < n:
            g[r, l] += g_lp[r]
        else:
            g[r] += g_lp[r] * p[r]
    g[m == -np.inf] = 0.0
    tol = size * U * (3 * np.where(p > 0, np.abs(log_p), 0.0) + np.where(np.isfinite(S), np.abs(S), 0.0)[:, None] + 16)
    tol[m == -np.inf] = size[m == -np.inf] = 0.0
    for r, l in enumerate(labels):
        if 0 <= l < n:
            tol[r, l] += 2 * U * (np.abs(g_lp[r]) + size[r, l])
    return g, tol


def _check_grad(x, labels, g_lp, g_h, grad=None):
    import torch
    rows, n = x.shape
    out = _call(x, labels, 0)
    before = x.double().cpu().numpy()
    grad = torch.empty(rows, n, dtype=x.dtype, device=x.device) if grad is None else grad
    binding.class_scores_grad(x, grad, out["norm"], labels if g_lp is not None else None, g_lp, out["h"] if g_h is not None else None, g_h)
    z = np.zeros(rows)
    f = lambda t: z if t is None else t.double().cpu().numpy()  # noqa: E731
    want, tol = _grad_reference(before, labels.cpu().numpy(), f(out["norm"][:, 0]), f(out["norm"][:, 1]), f(out["h"]), f(g_lp), f(g_h))
    got = grad.double().cpu().numpy()
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
    fine = ~np.isnan(want)
    fi = torch.finfo(x.dtype)
    tol = tol + (np.abs(want) + tol) * fi.eps / 2 + fi.smallest_normal * fi.eps / 2 + 2.0 ** -126   # the type's rounding; tiny p are zero
    assert (np.abs(got - want)[fine] <= tol[fine]).all(), (x.shape, x.dtype, np.nanmax(np.abs(got - want) / tol))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n", [(1, 1), (5, 2), (40, 10), (3, 64), (2, 65), (7, 1000), (3, 1025), (2, 5003), (70, 513), (1, 131071)])
@pytest.mark.parametrize("which", ["both", "log p", "entropy"])
def test_gradients_match_the_formula(rows, n, dtype, which):
    import torch
    x, labels = _rows(rows, n, dtype, n + rows, pad=n % 3, offset=rows % 2)
    labels[::4] = -1
    labels[1::5] = n
    if n > 2:
        x[rows // 2, :: 2] = -math.inf
        x[rows - 1] = -math.inf
    gen = torch.Generator(device="cuda:0").manual_seed(1)
    g = torch.randn(2, rows, generator=gen, device="cuda:0")
    _check_grad(x, labels, g[0].contiguous() if which != "entropy" else None, g[1].contiguous() if which != "log p" else None)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [10, 700, 5001])
def test_gradients_in_place_and_between_other_columns(n, dtype):
    import torch
    x, labels = _rows(6, n, dtype, 2, pad=3)
    x[2] = math.nan
    x[3, 0] = math.inf
    g = torch.randn(2, 6, device="cuda:0")
    wide = torch.full((6, n + 9), 7.0, dtype=x.dtype, device="cuda:0")
    _check_grad(x, labels, g[0].contiguous(), g[1].contiguous(), wide[:, 4:4 + n])
    assert (wide[:, :4] == 7).all() and (wide[:, 4 + n:] == 7).all()
    apart = wide[:, 4:4 + n].clone()
    _check_grad(x, labels, g[0].contiguous(), g[1].contiguous(), x)      # over the rows themselves
    assert torch.equal(x.isnan(), apart.isnan()) and torch.equal(x.nan_to_num(), apart.nan_to_num())


def test_gradients_of_more_rows_than_a_launch_holds():
    """In place, on a buffer whose places pass 32 bits; a row's gradient is its own, whatever the number of rows."""
    import torch
    rows, n = (1 << 21) + 3, 1025
    some, l = _rows(4097, n, "bfloat16", 8)
    x = some.repeat(-(-rows // 4097), 1)[:rows]
    labels = l.repeat(-(-rows // 4097))[:rows].contiguous()
    out = _call(some, l, 0)
    norm, h = (out[k].repeat(*([-(-rows // 4097)] + [1] * (out[k].dim() - 1)))[:rows].contiguous() for k in ("norm", "h"))
    gen = torch.Generator(device="cuda:0").manual_seed(3)
    g, e = (torch.randn(rows, generator=gen, device="cuda:0") for _ in range(2))
    binding.class_scores_grad(x, x, norm, labels, g, h, e)
    for a in (0, 4097, 1 << 20, rows - 4097 - rows % 4097, rows - rows % 4097):
        a -= a % 4097
        b = min(rows, a + 4097)
        want = torch.empty_like(some[:b - a])
        binding.class_scores_grad(some[:b - a], want, norm[a:b], l[:b - a], g[a:b], h[a:b], e[a:b])
        assert torch.equal(x[a:b], want), a


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n", [(1, 2), (70, 10), (9, 64), (300, 300), (4, 1000)])
def test_gradients_of_rows_that_are_nearly_sure(rows, n, dtype):
    """The label's, g (1 - p), is off by what its log p is, (2.5 gap + 36) U of it, the series' 8 U, the product's and the type's rounding."""
    import torch
    gen = torch.Generator(device="cuda:0").manual_seed(n + 1)
    x = (-(torch.rand(rows, n, generator=gen, device="cuda:0") * 10 + 8)).to(getattr(torch, dtype))
    label = torch.randint(0, n, (rows,), generator=gen, device="cuda:0", dtype=torch.int32)
    i = torch.arange(rows, device="cuda:0"), label.long()
    x[i] = 0.25
    g = torch.randn(rows, generator=gen, device="cuda:0")
    out, grad = _call(x, label, 0), torch.empty_like(x)
    binding.class_scores_grad(x, grad, out["norm"], label, g)
    d = x.double().cpu().numpy()
    gap = 0.25 - d.min()
    d[np.arange(rows), label.cpu().numpy()] = -np.inf
    want = g.double().cpu().numpy() * -np.expm1(-np.log1p(np.exp(d - 0.25).sum(1)))
    fi = torch.finfo(x.dtype)
    tol = np.abs(want) * ((2.5 * gap + 48) * U + fi.eps / 2 * (1 + 1e-3)) + fi.smallest_normal * fi.eps / 2
    assert (np.abs(grad[i].double().cpu().numpy() - want) <= tol).all()


@pytest.mark.parametrize("n", [7, 90, 1500])
def test_gradients_are_those_of_differences(n):
    """Central differences of the definition in 64 bits, h = 1e-4: off by h^2 / 6 of a third derivative (below 8 times the two
    weights and |log p|) and 1e-16 / h, beside the kernel's own tolerance."""
    import torch
    x, labels = _rows(3, n, "float32", n)
    g = torch.randn(2, 3, device="cuda:0")
    out = _call(x, labels, 0)
    grad = torch.empty_like(x)
    binding.class_scores_grad(x, grad, out["norm"], labels, g[0].contiguous(), out["h"], g[1].contiguous())
    x0, l, w = x.double().cpu().numpy(), labels.cpu().numpy(), g.double().cpu().numpy()

    def value(y):
        r = _reference(y, l, 1)
        return w[0] * r[0] + w[1] * r[1]

    h = 1e-4
    for c in {0, 1, n // 2, n - 1, int(l[0]), int(l[1]), int(l[2])}:
        step = np.zeros_like(x0)
        step[:, c] = h
        d = (value(x0 + step) - value(x0 - step)) / (2 * h)
        size = np.abs(w).sum(0)
        tol = 8 * size * 40 * h * h / 6 + 1e-11 + 100 * U * size * 20
        assert (np.abs(grad[:, c].double().cpu().numpy() - d) <= tol).all()


def test_bad_tensors_are_refused():
    import torch
    x, labels = _rows(3, 100, "float32", 1)
    f = torch.empty(3, device="cuda:0")
    for bad in (x.double(), x.t(), x[:, ::2], x[0]):
        with pytest.raises(AssertionError):
            binding.class_scores(bad, d_entropy=f)
    for kw in (dict(d_labels=labels.long(), d_log_probs=f), dict(d_labels=labels[:2], d_log_probs=f), dict(d_entropy=f[:2]),
               dict(d_entropy=f.half()), dict(d_normaliser=f), dict(d_top=torch.empty(2, 3, dtype=torch.int32, device="cuda:0")),
               dict(d_entropy=torch.empty(3))):
        with pytest.raises(AssertionError):
            binding.class_scores(x, **kw)
    with pytest.raises(binding.CnnError):
        binding.class_scores(x, d_log_probs=f)


FAR = [1.1e7, 1.2e7, 2e7, 1e8, 1e9, 5e9, 1e10, 1e12, 1e15, 1e20, 1e30, 1e36, 1.5e38, 2.3e38, 3.3e38]


def _far_rows(n, dtype, values):
    """Rows of values v, for v of both signs far from 0: constant, as far as v from each other, rising to v and falling from it, half of
    them masked, and one class at v among ordinary ones, the first, in the middle, the last."""
    import torch
    gen = torch.Generator(device="cuda:0").manual_seed(n)
    rand = lambda: torch.randn(n, generator=gen, device="cuda:0")  # noqa: E731
    rise = torch.arange(1, n + 1, device="cuda:0") / n
    rows = []
    for v in values:
        for s in (v, -v):
            masked = torch.full((n,), s, device="cuda:0")
            masked[::2] = -math.inf
            rows += [torch.full((n,), s, device="cuda:0"), rand().clamp(-3, 3) / 3 * s, rise * s, rise.flip(0) * s, masked]
        for at in (0, n // 2, n - 1):
            rows.append(rand())
            rows[-1][at] = v
    return torch.stack(rows).to(getattr(torch, dtype))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("n,top", [(40, 20), (200, 20), (900, 5), (1024, 20), (3000, 20), (9001, 3), (30000, 64), (70001, 20), (110000, 2)])
def test_finite_values_far_from_zero(n, top, dtype):
    """Every finite row has a distribution, whatever its size: with all outputs, without the entropy, without the best, and the
    gradient from those normalisers.  (The longest in parts of rows.)"""
    import torch
    x = _far_rows(n, dtype, FAR if n <= 5000 else FAR[n % 4::4])
    rows = x.shape[0]
    labels = (torch.arange(rows, device="cuda:0", dtype=torch.int32) * 7919) % n
    every = _call(x, labels, top)
    assert torch.isfinite(every["norm"]).all() and (every["top"] >= 0).all()
    _check(x, labels, top, every)
    for want in (("lp", "norm"), ("lp", "top", "top_lp")):
        out = _call(x, labels, top, want=want)
        _check(x, labels, top, {**every, **{k: out[k] for k in want}})
    g = torch.randn(2, rows, generator=torch.Generator(device="cuda:0").manual_seed(2), device="cuda:0")
    _check_grad(x, labels, g[0].contiguous(), g[1].contiguous())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,offset", [(0, 1), (1, 0), (3, 5), (5, 7)])
@pytest.mark.parametrize("n,top", [(1017, 9), (1018, 64), (1019, 20), (1022, 9), (1023, 33), (1024, 64), (1024, 9)])
def test_nearly_sure_rows_are_the_same_wherever_they_start(n, top, pad, offset, dtype):
    """Rows of equal values, at every distance from a 16-byte boundary: the same logarithms to the last bit, and those of the definition
    to the (2.5 g + 36) U of the test of aligned ones above."""
    import torch
    rows = 16
    gen = torch.Generator(device="cuda:0").manual_seed(n)
    one = (-(torch.rand(n, generator=gen, device="cuda:0") * 10 + 13)).to(getattr(torch, dtype))
    one[n // 3] = 0.25
    wide = torch.zeros(rows * (n + pad) + offset, dtype=one.dtype, device="cuda:0")
    x = wide[offset:].view(rows, n + pad)[:, :n]
    x.copy_(one.expand(rows, n))
    labels = torch.full((rows,), n // 3, dtype=torch.int32, device="cuda:0")
    out = _call(x, labels, top)
    d = one.double().cpu().numpy()
    gap = 0.25 - d.min()
    d[n // 3] = -np.inf
    want = -np.log1p(np.exp(d - 0.25).sum())
    tol = abs(want) * (2.5 * gap + 36) * U
    assert (np.abs(out["lp"].cpu().numpy().astype(np.float64) - want) <= tol).all()
    assert (np.abs(out["norm"][:, 1].cpu().numpy().astype(np.float64) + want) <= tol).all()
    for k in ("lp", "norm", "top", "top_lp"):
        assert torch.equal(out[k], out[k][:1].expand_as(out[k])), k


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n,top", [(300, 8, 3), (300, 700, 20), (300, 1500, 9), (300, 1500, 0), (300, 9000, 5), (64, 30000, 5), (40, 90000, 20), (40, 110000, 0)])
def test_no_probability_is_above_one(rows, n, top, dtype):
    """Rows with a class beside which the others are nothing: its log p, above -n e^-39, is 0 to the tolerance of the definition (rows of up
    to 1024 classes: to that number), and not above it."""
    import torch
    gen = torch.Generator(device="cuda:0").manual_seed(n)
    best = torch.randint(0, n, (rows,), generator=gen, device="cuda:0", dtype=torch.int32)
    m = torch.rand(rows, generator=gen, device="cuda:0") * 40 - 20
    m[1::4] *= 1500
    m = m.to(getattr(torch, dtype)).double()
    x = (m - 40 - m.abs() / 8)[:, None].expand(rows, n).contiguous()
    i = torch.arange(rows, device="cuda:0"), best.long()
    x[i] = m
    x = x.to(getattr(torch, dtype))
    out = _call(x, best, top)
    off = n * 2e-17 + (0 if n <= 1024 else (_terms(rows, n) + 100) * U)
    assert (out["lp"] <= 0).all() and (out["lp"] >= -off).all()
    assert (out["norm"][:, 1] >= 0).all() and (out["norm"][:, 1] <= off).all() and (out["h"] >= 0).all()
    if top:
        assert torch.equal(out["top"][:, 0], best) and (out["top_lp"] <= 0).all()
    grad = torch.empty_like(x)
    binding.class_scores_grad(x, grad, out["norm"], best, torch.ones(rows, device="cuda:0"))
    assert (grad[i] >= 0).all()
