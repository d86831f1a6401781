"""Refusals of the operators that work on a caller's tensors (scores of classes, their gradient, the norm of gradients, clipping,
the clipped update) and what they say about memory: no GPU, a refused call looks at no tensor."""
import ctypes as C

import pytest

from paper_1102_0183_amd import binding
from paper_1102_0183_amd.binding import E_ARG, E_SHAPE, E_WORKSPACE, TYPE_BF16, TYPE_F16, TYPE_F32, Tensor

P = 1 << 20   # an address that is never looked at


def _scores(x=P, kind=TYPE_F32, rows=4, classes=10, stride=10, labels=P, lp=P, h=P, norm=P, n_top=3, top=P, top_lp=P, scratch=None, nbytes=0):
    return binding.lib().cnn_class_scores(None, x, kind, rows, classes, stride, labels, lp, h, norm, n_top, top, top_lp, scratch, nbytes)


@pytest.mark.parametrize("kw,code", [
    (dict(kind=3), E_ARG), (dict(kind=-1), E_ARG), (dict(classes=0), E_SHAPE), (dict(classes=(1 << 30) + 1, stride=1 << 31), E_SHAPE),
    (dict(rows=1 << 31), E_SHAPE), (dict(stride=9), E_ARG), (dict(stride=1 << 62), E_ARG), (dict(rows=1 << 30, stride=1 << 40), E_ARG),
    (dict(x=None), E_ARG), (dict(x=P + 2), E_ARG), (dict(x=P + 1, kind=TYPE_F16), E_ARG), (dict(labels=None), E_ARG),
    (dict(n_top=-1), E_ARG), (dict(n_top=11), E_ARG), (dict(n_top=65, classes=100, stride=100), E_ARG),
    (dict(rows=1, classes=100000, stride=100000), E_WORKSPACE),
    (dict(rows=1, classes=100000, stride=100000, scratch=P, nbytes=100), E_WORKSPACE),
    (dict(rows=1, classes=100000, stride=100000, scratch=P + 8, nbytes=1 << 30), E_WORKSPACE),
])
def test_bad_rows_are_refused(kw, code):
    assert _scores(**kw) == code
    assert "cnn_class_scores" in binding._err()


def test_no_rows_is_no_work():
    assert _scores(rows=0, x=None) == 0
    assert binding.class_scores_scratch_bytes(0, 100000, 20) == 0
    assert binding.lib().cnn_class_scores_grad(None, None, 0, 0, 10, 10, None, None, None, None, None, None, 10) == 0


def _grad(x=P, kind=TYPE_F32, rows=4, classes=10, stride=10, labels=P, norm=P, h=P, g_lp=P, g_h=P, grad=2 * P, grad_stride=10):
    return binding.lib().cnn_class_scores_grad(None, x, kind, rows, classes, stride, labels, norm, h, g_lp, g_h, grad, grad_stride)


@pytest.mark.parametrize("kw,code", [
    (dict(kind=7), E_ARG), (dict(classes=0), E_SHAPE), (dict(stride=9), E_ARG), (dict(grad_stride=9), E_ARG), (dict(x=None), E_ARG),
    (dict(norm=None), E_ARG), (dict(grad=None), E_ARG), (dict(grad=2 * P + 2), E_ARG), (dict(labels=None), E_ARG), (dict(h=None), E_ARG),
    (dict(g_lp=None, g_h=None), E_ARG), (dict(grad=P, grad_stride=11), E_ARG), (dict(grad=P + 4), E_ARG), (dict(grad=P + 39 * 4), E_ARG),
    (dict(grad=P - 39 * 4), E_ARG), (dict(grad=P + 20, stride=20, grad_stride=20), E_ARG),
])
def test_bad_gradients_of_rows_are_refused(kw, code):
    assert _grad(**kw) == code
    assert "cnn_class_scores_grad" in binding._err()


def test_scratch_of_scores():
    """Nothing where rows fill the chip or are short; elsewhere whole parts of every row."""
    assert binding.class_scores_scratch_bytes(10000, 10, 10) == 0
    assert binding.class_scores_scratch_bytes(1, 4096, 64) == 0
    assert binding.class_scores_scratch_bytes(512, 200000, 64) == 0
    assert binding.class_scores_scratch_bytes(1, 131072, 20) == 16 * (16 + 8 * 20)
    for rows in (1, 2, 37, 511):
        for classes in (4097, 50000, 65537, 100003, 1 << 30):
            n = binding.class_scores_scratch_bytes(rows, classes, 5)
            parts, odd = divmod(n, rows * (16 + 8 * 5))
            assert odd == 0 and parts <= 256, (rows, classes)
            assert binding.class_scores_scratch_bytes(rows, classes, 0) <= n     # enough with fewer best, too
    for bad in ((1, 10, 11), (1, 100, 65), (1, 0, 0), (1, 10, -1)):
        with pytest.raises(binding.CnnError):
            binding.class_scores_scratch_bytes(*bad)
    assert binding.lib().cnn_class_scores_scratch_bytes(1, 10, 1, None) == E_ARG


def _list(*tensors):
    a = (Tensor * max(1, len(tensors)))()
    for k, (p, n, kind) in enumerate(tensors):
        a[k] = Tensor(p, n, kind)
    return a


F, B, H = TYPE_F32, TYPE_BF16, TYPE_F16


@pytest.mark.parametrize("tensors", [[(P, 10, 3)], [(None, 10, F)], [(P + 2, 10, F)], [(P + 1, 10, B)], [(P, 1 << 45, F)],
                                     [(P, 1 << 44, F), (2 * P, 1, F)]])
def test_bad_tensors_are_refused(tensors):
    L, a, n = binding.lib(), _list(*tensors), len(tensors)
    w = _list(*[(1 << 50, t[1], F) for t in tensors])
    assert L.cnn_gradient_norm(None, a, n, P, P, 1 << 30) == E_ARG
    assert L.cnn_clip_gradients(None, a, None, n, 1.0, P, P, 1 << 30) == E_ARG
    assert L.cnn_clipped_update(None, w, a, n, 1.0, 1.0, P, P, 1 << 30) == E_ARG


@pytest.mark.parametrize("out", [
    [(P, 100, F), (3 * P, 100, F)],                # another order
    [(P + 4, 100, F), (3 * P, 50, B)],             # a shifted copy
    [(4 * P, 100, F), (4 * P + 396, 50, B)],       # what is written overlaps
    [(4 * P, 100, F), (P + 100, 50, B)],           # one over another's gradients
    [(4 * P, 99, F), (5 * P, 50, B)],              # another size
    [(4 * P, 100, F), (5 * P, 50, H)],             # another type
    [(4 * P, 100, F), (None, 50, B)], [(4 * P + 2, 100, F), (5 * P, 50, B)],
])
def test_bad_places_for_clipped_gradients_are_refused(out):
    a = _list((P, 100, F), (2 * P, 50, B))
    assert binding.lib().cnn_clip_gradients(None, a, _list(*out), 2, 1.0, P, P, 1 << 30) == E_ARG
    assert "cnn_clip_gradients" in binding._err()


def test_the_same_tensor_twice():
    """It counts twice in a norm, and cannot be written."""
    a = _list((P, 100, F), (P, 100, F))
    L = binding.lib()
    assert L.cnn_clip_gradients(None, a, None, 2, 1.0, P, P, 1 << 30) == E_ARG
    assert L.cnn_clipped_update(None, a, _list((2 * P, 100, F), (3 * P, 100, F)), 2, 1.0, 1.0, P, P, 1 << 30) == E_ARG


def test_weights_are_fp32_and_not_the_gradients():
    L, g = binding.lib(), _list((P, 100, B))
    for w in (_list((2 * P, 100, B)), _list((P, 100, F)), _list((P - 396, 100, F)), _list((P + 196, 100, F)), _list((2 * P, 99, F)), _list((None, 100, F))):
        assert L.cnn_clipped_update(None, w, g, 1, 0.1, 1.0, P, P, 1 << 30) == E_ARG
    assert L.cnn_clipped_update(None, None, g, 1, 0.1, 1.0, P, P, 1 << 30) == E_ARG


@pytest.mark.parametrize("lr,limit", [(0.1, -1.0), (0.1, float("nan")), (float("nan"), 1.0), (float("inf"), 1.0)])
def test_bad_limits_and_rates_are_refused(lr, limit):
    L, g, w = binding.lib(), _list((P, 100, B)), _list((2 * P, 100, F))
    assert L.cnn_clipped_update(None, w, g, 1, lr, limit, P, P, 1 << 30) == E_ARG
    if limit != 1.0:
        assert L.cnn_clip_gradients(None, g, None, 1, limit, P, P, 1 << 30) == E_ARG


def test_scratch_of_lists():
    L, g = binding.lib(), _list((P, 100, F))
    n = binding.gradient_scratch_bytes(1)
    for scratch, nbytes in ((None, n), (P + 8, n), (P, n - 1)):
        assert L.cnn_gradient_norm(None, g, 1, P, scratch, nbytes) == E_WORKSPACE
    assert L.cnn_gradient_norm(None, g, 1, None, P, n) == E_ARG
    assert L.cnn_gradient_norm(None, None, 1, P, P, n) == E_ARG
    assert binding.gradient_scratch_bytes(0) > 0 and binding.gradient_scratch_bytes(1000) >= binding.gradient_scratch_bytes(1)
    assert L.cnn_gradient_scratch_bytes(1, None) == E_ARG
    with pytest.raises(binding.CnnError):
        binding.gradient_scratch_bytes(1 << 30)
    assert L.cnn_gradient_norm(None, g, 1 << 30, P, P, 1 << 40) == E_ARG


def test_lists_of_more_chunks_than_are_counted():
    """2^43 elements are 2^31 chunks; the kernels count them, and the step beyond the last, in 32 bits."""
    L, n = binding.lib(), binding.gradient_scratch_bytes(2)
    for counts in ([1 << 44], [(1 << 43) + 1], [1 << 43, 1], [1 << 42] * 4):
        g = _list(*[(P, c, B) for c in counts])
        assert L.cnn_gradient_norm(None, g, len(counts), P, P, n) == E_ARG, counts


def test_an_empty_list_needs_a_device():
    empty = binding.TensorList([])
    for call in (lambda: binding.clip_gradients(empty, 1.0, None), lambda: binding.clipped_update(empty, empty, 0.1, 1.0, None),
                 lambda: binding.gradient_norm(empty, None, None)):
        with pytest.raises(AssertionError):
            call()
