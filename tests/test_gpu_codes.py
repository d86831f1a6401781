"""Layers of 4-bit weights against the definition in 64 bits, through the C ABI.  Needs a GPU.

Tolerances.  u = 2^-24, h half a step of the result's type (2^-24, 2^-8, 2^-11).  x times a code's value is exact; a result is a sum of
n_in such products and n_in / 32 products with scales in some order, every addition off by at most one step of fp32 (the matrix cores'
may cut off) of a partial sum, which is below the sum of the magnitudes: 2 u (n_in + n_in / 32 + 20) of that, and h of the result.
Where all terms and sums are whole numbers below 2^24 (times a power of two), the result is exact.
"""
import numpy as np
import pytest

from paper_1102_0183_amd import binding
from paper_1102_0183_amd.binding import CODES_E2M1, CODES_INT4

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = {"float32": (2.0 ** -24, 2.0 ** -149), "bfloat16": (2.0 ** -8, 2.0 ** -133), "float16": (2.0 ** -11, 2.0 ** -24)}
VALUES = {CODES_INT4: [float(c - 8) for c in range(16)], CODES_E2M1: [0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6]}


def _layer(n_out, n_in, group, dtype, kind, seed, pad=0):
    """(codes, scales, weights in 64 bits); rows of codes `pad` bytes apart, which hold anything."""
    import torch
    gen = torch.Generator(device="cuda:0").manual_seed(seed)
    nbytes = (n_in + 1) // 2
    codes = torch.randint(0, 256, (n_out, nbytes + pad), generator=gen, device="cuda:0", dtype=torch.uint8)[:, :nbytes]
    scales = torch.empty(n_out, -(-n_in // group), device="cuda:0").uniform_(0.01, 0.05, generator=gen).to(getattr(torch, dtype))
    return codes, scales, _weights(codes, scales, n_in, group, kind)


def _weights(codes, scales, n_in, group, kind):
    import torch
    c = torch.stack([codes & 15, codes >> 4], 2).view(codes.shape[0], -1)[:, :n_in].long()
    return torch.tensor(VALUES[kind], dtype=torch.float64, device="cuda:0")[c] * scales.double().repeat_interleave(group, 1)[:, :n_in]


def _rows(rows, n_in, dtype, seed, pad=0, offset=0):
    import torch
    gen = torch.Generator(device="cuda:0").manual_seed(seed)
    wide = torch.randn(rows * (n_in + pad) + offset, generator=gen, device="cuda:0").to(getattr(torch, dtype))
    return wide[offset:].view(rows, n_in + pad)[:, :n_in]


def _check(y, x, w, bias, what):
    import torch
    h, tiny = TYPES[str(y.dtype).split(".")[1]]
    n_in = x.shape[1]
    x = x.double()
    want, most = x @ w.t(), x.abs() @ w.abs().t()
    if bias is not None:
        want, most = want + bias.double(), most + bias.double().abs()
    tol = 2 * U * (n_in + n_in / 32 + 20) * most + h * want.abs() * 1.01 + tiny
    off = (y.double() - want).abs()
    assert (off <= tol).all(), (what, (off - tol).max().item())
    assert torch.isfinite(y).all()


def _run(x, codes, scales, group, kind, bias=None, y_dtype=None, n_out=None):
    import torch
    y = torch.full((x.shape[0], codes.shape[0]), 77.0, dtype=y_dtype or x.dtype, device="cuda:0")
    binding.quantised_product(x, codes, scales, y, group, kind, bias)
    return y


SHAPES = [(1, 1, 1), (1, 2, 3), (2, 31, 5), (1, 32, 16), (3, 33, 17), (5, 127, 31), (6, 128, 64), (16, 129, 33), (17, 150, 10), (1, 4096, 100), (4, 2501, 77),
          (33, 300, 50), (64, 1000, 130), (100, 257, 20), (1, 20000, 5), (150, 512, 48)]


@pytest.mark.parametrize("kind", [CODES_INT4, CODES_E2M1])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_in,n_out", SHAPES)
def test_products_match_the_definition(rows, n_in, n_out, dtype, kind):
    import torch
    x = _rows(rows, n_in, dtype, rows + n_in)
    for group, with_bias, y_dtype in ((32, False, None), (64, True, torch.float32), (128, True, None), (256, False, torch.float32), (1 << 24, True, None)):
        codes, scales, w = _layer(n_out, n_in, group, dtype, kind, n_in + n_out)
        bias = torch.randn(n_out, device="cuda:0", generator=torch.Generator(device="cuda:0").manual_seed(1)) if with_bias else None
        _check(_run(x, codes, scales, group, kind, bias, y_dtype), x, w, bias, (rows, n_in, n_out, dtype, kind, group))


# few rows of many outputs (two and four tiles of outputs a workgroup), two tiles of rows, and tiles of 64 rows (21 of fp32): columns that fill
# slabs of 128, do not, and are fewer than one
LARGE = [(1, 2176, 16390), (3, 2100, 16400), (9, 2100, 16500), (2, 200, 65540), (12, 130, 65537), (30, 260, 10000), (23, 700, 5001), (70, 512, 12290),
         (64, 300, 24577), (130, 100, 9000), (65, 1666, 12300), (200, 129, 6200)]


@pytest.mark.parametrize("kind", [CODES_INT4, CODES_E2M1])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_in,n_out", LARGE)
def test_products_of_many_outputs(rows, n_in, n_out, dtype, kind):
    import torch
    x = _rows(rows, n_in, dtype, rows + n_in)
    bias = torch.randn(n_out, device="cuda:0", generator=torch.Generator(device="cuda:0").manual_seed(1))
    for group, y_dtype in ((32, torch.float32), (64, None), (128, torch.float32)):
        codes, scales, w = _layer(n_out, n_in, group, dtype, kind, n_in + n_out)
        _check(_run(x, codes, scales, group, kind, bias, y_dtype), x, w, bias, (rows, n_in, n_out, dtype, kind, group))


@pytest.mark.parametrize("kind", [CODES_INT4, CODES_E2M1])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("group", [32, 64, 128, 512])
@pytest.mark.parametrize("rows,n_in,n_out", [(64, 1024, 24600), (1, 640, 40), (7, 515, 33), (40, 1024, 70), (130, 384, 100)])
def test_whole_numbers_are_exact(rows, n_in, n_out, group, dtype, kind):
    """Sums of at most 1024 products of 8 and 8 and a scale of a quarter to 2: every bit."""
    import torch
    gen = torch.Generator(device="cuda:0").manual_seed(rows)
    x = torch.randint(-8, 9, (rows, n_in), generator=gen, device="cuda:0").to(getattr(torch, dtype))
    codes, scales, _ = _layer(n_out, n_in, group, dtype, kind, 3)
    scales = torch.exp2(torch.randint(-2, 2, scales.shape, generator=gen, device="cuda:0").float()).to(x.dtype)
    want = x.double() @ _weights(codes, scales, n_in, group, kind).t()
    y = _run(x, codes, scales, group, kind, None, torch.float32)
    assert torch.equal(y.double(), want)


@pytest.mark.parametrize("kind,one", [(CODES_INT4, 9), (CODES_E2M1, 2)])
def test_every_code_and_all_bits_of_32(kind, one):
    """A row with one number in it comes out times each code's value, with all of its 24 bits."""
    import torch
    n_in = 200
    gen = torch.Generator(device="cuda:0").manual_seed(5)
    x = torch.zeros(n_in, n_in, device="cuda:0")
    v = torch.randn(n_in, generator=gen, device="cuda:0") * torch.exp2(torch.randint(-30, 30, (n_in,), generator=gen, device="cuda:0").float())
    x[torch.arange(n_in), torch.arange(n_in)] = v
    codes = torch.arange(16, device="cuda:0", dtype=torch.uint8)[:, None].mul(17).expand(16, n_in // 2).contiguous()
    scales = torch.ones(16, -(-n_in // 32), device="cuda:0")
    y = _run(x, codes, scales, 32, kind)
    want = v.double()[:, None] * torch.tensor(VALUES[kind], dtype=torch.float64, device="cuda:0")
    assert torch.equal(y, want.float())
    assert torch.equal(y[:, one], v)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad,offset,code_pad", [(1, 0, 0), (3, 1, 1), (0, 1, 3), (8, 0, 16), (7, 2, 5)])
@pytest.mark.parametrize("rows,n_in,n_out", [(3, 100, 20), (20, 1031, 37), (66, 523, 12345)])
def test_rows_start_anywhere_and_what_lies_between_stays(rows, n_in, n_out, pad, offset, code_pad, dtype):
    import torch
    x = _rows(rows, n_in, dtype, 4, pad, offset)
    codes, scales, w = _layer(n_out, n_in, 64, dtype, CODES_INT4, 6, code_pad)
    wide = torch.full((rows, n_out + pad + 1), 77.0, dtype=x.dtype, device="cuda:0")
    binding.quantised_product(x, codes, scales, wide[:, :n_out], 64, CODES_INT4)
    _check(wide[:, :n_out], x, w, None, "strides")
    assert (wide[:, n_out:] == 77).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", [CODES_INT4, CODES_E2M1])
def test_infinities_and_nan_stay_in_their_rows(kind, dtype):
    import math
    import torch
    x = _rows(20, 300, dtype, 1)
    codes, scales, w = _layer(50, 300, 32, dtype, kind, 2)
    clean = _run(x, codes, scales, 32, kind)
    x[3, 299] = math.nan
    x[7, 0] = math.inf
    x[8, 40] = -math.inf
    y = _run(x, codes, scales, 32, kind)
    others = [r for r in range(20) if r not in (3, 7, 8)]
    assert torch.equal(y[others], clean[others]) and torch.isnan(y[3]).all()
    for row, at, sign in ((7, 0, 1.0), (8, 40, -1.0)):
        v = w[:, at] * sign
        assert torch.equal(torch.isnan(y[row]), v == 0)
        assert torch.equal(y[row][v != 0].double(), torch.where(v[v != 0] > 0, math.inf, -math.inf))
    # a scale that is no number spoils its output alone
    scales = scales.clone()
    scales[4, 2] = math.nan
    y = _run(x, codes, scales, 32, kind)
    assert torch.isnan(y[:, 4]).all() and torch.equal(torch.isnan(y[others][:, 5:]), torch.isnan(clean[others][:, 5:]))


def test_large_and_small_numbers_of_32_bits():
    """Rows near both ends of the exponents: the pieces of a float neither overflow nor lose what matters."""
    import torch
    codes, scales, w = _layer(30, 256, 128, "float32", CODES_E2M1, 2)
    for scale in (1e37, 1e30, 1e-20, 1e-30):
        x = _rows(6, 256, "float32", 1) * (scale / 8)
        _check(_run(x, codes, scales, 128, CODES_E2M1), x, w, None, scale)


def test_the_same_call_gives_the_same_bits_and_rows_do_not_depend_on_others():
    import torch
    x = _rows(48, 3000, "bfloat16", 1)
    codes, scales, _ = _layer(500, 3000, 64, "bfloat16", CODES_INT4, 2)
    a = _run(x, codes, scales, 64, CODES_INT4, None, torch.float32)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    y = torch.empty_like(a)
    torch.cuda.synchronize()
    binding.quantised_product(x, codes, scales, y, 64, CODES_INT4, stream=st)
    torch.cuda.synchronize()
    assert torch.equal(a, y)


def test_captured_and_replayed():
    import torch
    x = _rows(3, 1000, "float16", 1)
    codes, scales, w = _layer(300, 1000, 128, "float16", CODES_INT4, 2)
    y = torch.empty(3, 300, dtype=torch.float16, device="cuda:0")
    binding.quantised_product(x, codes, scales, y, 128)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.quantised_product(x, codes, scales, y, 128)
    for k in range(4):
        x.copy_(_rows(3, 1000, "float16", 10 + k))
        graph.replay()
        torch.cuda.synchronize()
        _check(y, x, w, None, k)
        _check(_run(x, codes, scales, 128, CODES_INT4), x, w, None, k)


def test_codes_beyond_32_bits():
    """Rows of codes further than 2^32 bytes from the first one."""
    import torch
    n_out, n_in, stride = 6, 300, (1 << 30) + 3
    codes, scales, w = _layer(n_out, n_in, 32, "bfloat16", CODES_INT4, 2)
    far = torch.empty((n_out - 1) * stride + 150, dtype=torch.uint8, device="cuda:0").as_strided((n_out, 150), (stride, 1))
    far.copy_(codes)
    x = _rows(2, n_in, "bfloat16", 1)
    _check(_run(x, far, scales, 32, CODES_INT4), x, w, None, "far")


@pytest.mark.parametrize("kind", [CODES_INT4, CODES_E2M1])
@pytest.mark.parametrize("scale_type,dtype", [(binding.TYPE_F32, "float32"), (binding.TYPE_BF16, "bfloat16"), (binding.TYPE_F16, "float16")])
def test_a_layer_of_the_library_in_4_bits(scale_type, dtype, kind):
    """Weights of a network, rounded on the host, uploaded and multiplied: the layer's sums but for the rounding of its weights."""
    import torch
    net = binding.Cnn("1x29x29-20C4-MP2-40C5-MP3-150N-10N")
    rng = np.random.default_rng(1)
    net.set_weights(rng.uniform(-0.05, 0.05, net.num_weights).astype(np.float32))
    flat = net.get_weights()
    net.close()
    w = flat[-(10 + 1500) - 150 * 360:-(10 + 1500)].reshape(150, 360)
    codes, scales = binding.quantise_weights(w, 64, kind, scale_type)
    s = torch.from_numpy(scales.view(np.int16)).view(torch.bfloat16) if scale_type == binding.TYPE_BF16 else torch.from_numpy(scales)
    codes, s = torch.from_numpy(codes).to("cuda:0"), s.to("cuda:0")
    x = _rows(9, 360, dtype, 3)
    held = _weights(codes, s, 360, 64, kind)
    _check(_run(x, codes, s, 64, kind), x, held, None, "layer")
    # a weight is off by half a step (1 of 7, or a part of 6 between 4 and 6) and the rounding of its scale
    step = (0.5 if kind == CODES_INT4 else 1.0) / (7 if kind == CODES_INT4 else 6) + 2.0 ** -7
    assert (held.cpu().numpy() - w).__abs__().max() <= 0.05 * step


@pytest.mark.parametrize("kind,codes_of", [(CODES_INT4, (9, 7)), (CODES_E2M1, (2, 10))])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,n_in,n_out", [(1, 20, 5), (3, 32, 5), (2, 64, 40), (20, 200, 40), (40, 224, 3000), (66, 160, 12345), (66, 33, 24600)])
def test_an_infinite_scale_makes_its_output_infinite(rows, n_in, n_out, group, dtype, kind, codes_of):
    """The last group's, whose columns end inside a slab: y is infinite with the sign of the group's sum, not NaN, and other outputs are as they were."""
    import math
    import torch
    x = torch.ones(rows, n_in, device="cuda:0", dtype=getattr(torch, dtype))
    codes = torch.full((n_out, (n_in + 1) // 2), codes_of[0] * 17, dtype=torch.uint8, device="cuda:0")
    codes[3] = codes_of[1] * 17   # values of -1
    scales = torch.full((n_out, -(-n_in // group)), 0.5, device="cuda:0", dtype=x.dtype)
    clean = _run(x, codes, scales, group, kind)
    scales[1, -1] = scales[3, -1] = math.inf
    scales[n_out - 1, -1] = -math.inf
    y = _run(x, codes, scales, group, kind)
    for o, want in ((1, math.inf), (3, -math.inf), (n_out - 1, -math.inf)):
        assert (y[:, o] == want).all(), (o, y[:, o])
    y[:, 1], y[:, 3], y[:, n_out - 1] = clean[:, 1], clean[:, 3], clean[:, n_out - 1]
    assert torch.equal(y, clean) and torch.isfinite(clean).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n_in,n_out", [(3, 700, 90), (16, 300, 50), (40, 1000, 70), (30, 260, 10000), (66, 523, 12345)])
def test_a_row_does_not_depend_on_the_others(rows, n_in, n_out, dtype):
    """As many rows, but others beside it (numbers, infinities, NaN): the same bits, first, last and between tiles."""
    import math
    import torch
    codes, scales, _ = _layer(n_out, n_in, 64, dtype, CODES_INT4, 2)
    a, b = _rows(rows, n_in, dtype, 1), _rows(rows, n_in, dtype, 2)
    keep = sorted({0, 2, rows // 2, rows - 1})
    b[1], b[rows - 2, ::3] = math.nan, math.inf
    b[keep] = a[keep]
    y, z = (_run(x, codes, scales, 64, CODES_INT4, None, torch.float32) for x in (a, b))
    assert torch.isfinite(y).all() and torch.equal(y[keep], z[keep])
    others = [r for r in range(rows) if r not in keep]
    assert (y[others] != z[others]).any(1).all()


def test_small_numbers_of_32_bits():
    """What bits a float has of 2^-133 and above count, all of them; those below count as 0."""
    import torch
    n_in, rows = 64, 150
    gen = torch.Generator(device="cuda:0").manual_seed(5)
    x = torch.zeros(rows, n_in, dtype=torch.float64, device="cuda:0")
    x[:, 0] = (1 + torch.rand(rows, generator=gen, device="cuda:0", dtype=torch.float64)) * torch.exp2(-torch.arange(rows, device="cuda:0").double())
    x[1::2] *= -1
    x = x.float()
    codes = torch.full((16, n_in // 2), 0x88, dtype=torch.uint8, device="cuda:0")
    scale = 2.0 ** 100
    scales = torch.full((16, 2), scale, device="cuda:0")
    for kind in (CODES_INT4, CODES_E2M1):
        codes.fill_(0x88 if kind == CODES_INT4 else 0)
        codes[:, 0] += torch.arange(16, device="cuda:0", dtype=torch.uint8) - (8 if kind == CODES_INT4 else 0)
        y = _run(x, codes, scales, 32, kind)
        values = torch.tensor(VALUES[kind], dtype=torch.float64, device="cuda:0")
        v = x[:, 0].double()
        want = v[:, None] * values * scale
        held = torch.trunc(v * 2.0 ** 133) * 2.0 ** -133
        # three pieces of 8 bits, cut off: exact where the last one ends at 2^-133 or above; products and their sum are rounded three times
        assert ((y.double() - held[:, None] * values * scale).abs() <= 3 * U * want.abs()).all()
        whole = v.abs() >= 2.0 ** -109
        assert ((y.double() - want).abs() <= 3 * U * want.abs())[whole].all()
