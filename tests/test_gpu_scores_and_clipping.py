"""The library's own paths through the scores of classes and the clipped update (cnn_score_batch, cnn_train_many_clipped), and all
of these operators together, as a program trains an output layer with them.  Needs a GPU."""
import math

import numpy as np
import pytest

import oracle
from paper_1102_0183_amd import binding, synth
from tests.parity_helpers import TOL_ACT, build_pair, layer_bounds, to_dev

pytestmark = pytest.mark.gpu
U = 2.0 ** -24

NETS = [("cfg1", None), ("cfg5", None), ("cfg4a", None),
        (None, "1x12x12-8C3-MP2-30N-64N"),      # 64 classes: the last two layers in one launch
        (None, "1x12x12-8C3-MP2-30N-65N"),      # not so
        (None, "1x12x12-8C3-MP2-700N"),         # a fully connected layer alone
        (None, "2x9x9-5N"), (None, "1x10x10-4C3-40N-6000N")]


def _pair(name, arch):
    if name:
        wl = synth.WORKLOADS[name]
        g, o = build_pair(wl)
        return g, o, lambda n: synth.images(wl, n)
    g, o = build_pair(arch=arch, wscale=0.2, seed=5)
    rng = np.random.default_rng(1)
    return g, o, lambda n: (rng.random((n, g.image_size), dtype=np.float32) * 2 - 1)


@pytest.mark.parametrize("name,arch", NETS)
@pytest.mark.parametrize("n,batch", [(1, 1), (7, 7), (50, 16)])
def test_scores_of_a_labelled_set(name, arch, n, batch):
    """Against the oracle's probabilities in 64 bits: the sums are off by at most TOL_ACT of the largest, log p by that twice, and
    the entropy, whose derivative by a sum is p (log p + H), by |log p| + H times that."""
    import torch
    g, o, images = _pair(name, arch)
    imgs = images(n)
    d_imgs = to_dev(imgs)
    C = g.num_classes
    top = min(C, 5)
    labels = torch.arange(n, dtype=torch.int32, device="cuda:0") * 7 % C
    labels[n // 2] = -1
    f = lambda *s: torch.full(s, 9.0, device="cuda:0")  # noqa: E731
    lp, h, top_lp, best = f(n), f(n), f(n, top), torch.zeros(n, top, dtype=torch.int32, device="cuda:0")
    scratch = torch.empty(g.forward_batch_scratch_bytes(batch), dtype=torch.uint8, device="cuda:0")
    g.score_batch(d_imgs, n, scratch, batch, labels, lp, h, best, top_lp)
    g.synchronize()
    probs = np.stack([o.forward(im) for im in imgs]).reshape(n, C)
    want = np.log(probs)
    size = np.abs(want).max() + math.log(C)        # (no sum is further from the largest than that)
    tol = 2 * TOL_ACT * size
    l = labels.cpu().numpy()
    got = lp.cpu().numpy()
    for i in range(n):
        assert abs(got[i] - (want[i, l[i]] if l[i] >= 0 else 0.0)) <= tol, (i, got[i])
    H = -(probs * want).sum(1)
    assert (np.abs(h.cpu().numpy() - H) <= tol * (size + H)).all()
    b, t = best.cpu().numpy(), top_lp.cpu().numpy()
    assert (np.abs(t - np.take_along_axis(want, b, 1)) <= tol).all()
    assert (np.abs(t - -np.sort(-want, axis=1)[:, :top]) <= 2 * tol).all()
    # the same sums as the probabilities'
    p = f(n * C)
    g.forward_batch(d_imgs, n, p, scratch, batch)
    g.synchronize()
    p = p.cpu().numpy().reshape(n, C).astype(np.float64)
    assert (np.abs(np.exp(t.astype(np.float64)) - np.take_along_axis(p, b, 1)) <= 64 * U).all()
    # fewer outputs: the same, but for the roundings of sums in another order (up to 112 terms a lane, as in the scores' own tests)
    lp2 = f(n)
    g.score_batch(d_imgs, n, scratch, batch, d_labels=labels, d_log_probs=lp2)
    h2 = f(n)
    g.score_batch(d_imgs, n, scratch, batch, d_entropy=h2)
    g.synchronize()
    assert ((lp2 - lp).abs() <= 2 * (112 + 100) * U * (1 + lp.abs())).all()
    assert ((h2 - h).abs() <= 2 * (112 + 100) * U * (1 + math.log(C) + 2 * h.abs())).all()
    g.close()


def test_scores_of_a_set_are_refused():
    import torch
    g, o, images = _pair("cfg1", None)
    d = to_dev(images(2))
    lp = torch.empty(2, device="cuda:0")
    scratch = torch.empty(g.forward_batch_scratch_bytes(2), dtype=torch.uint8, device="cuda:0")
    cases = [(dict(d_log_probs=lp), binding.E_ARG), (dict(d_top_log_probs=torch.empty(2, 11, device="cuda:0")), binding.E_ARG)]
    for kw, code in cases:
        with pytest.raises(binding.CnnError) as e:
            g.score_batch(d, 2, scratch, 2, **kw)
        assert e.value.code == code
    with pytest.raises(binding.CnnError) as e:
        g.score_batch(d, 2, scratch[:256], 2, d_entropy=lp)
    assert e.value.code == binding.E_WORKSPACE
    g.set_output_units(binding.OUTPUT_TANH_SQERR)
    with pytest.raises(binding.CnnError) as e:
        g.score_batch(d, 2, scratch, 2, d_entropy=lp)
    assert e.value.code == binding.E_STATE
    g.close()


@pytest.mark.parametrize("name,arch", NETS[:-1])
def test_scores_captured_and_after_training(name, arch):
    """A captured call reads the weights and labels that are there when it is replayed."""
    import torch
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        r, _, images = _pair(name, arch)
    n, batch, C = 10, 4, r.num_classes
    d_imgs = to_dev(images(n))
    labels = torch.arange(n, dtype=torch.int32, device="cuda:0") % C
    scratch = torch.empty(r.forward_batch_scratch_bytes(batch), dtype=torch.uint8, device="cuda:0")
    new = lambda: (torch.zeros(n, device="cuda:0"), torch.zeros(n, device="cuda:0"), torch.zeros(n, 2, dtype=torch.int32, device="cuda:0"))  # noqa: E731
    held, eager = new(), new()
    torch.cuda.synchronize()
    r.score_batch(d_imgs, n, scratch, batch, labels, held[0], held[1], held[2])
    r.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        r.score_batch(d_imgs, n, scratch, batch, labels, held[0], held[1], held[2])
    last = None
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        r.score_batch(d_imgs, n, scratch, batch, labels, eager[0], eager[1], eager[2])
        r.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, eager))
        assert last is None or not torch.equal(last, held[0])
        last = held[0].clone()
        labels.copy_((labels + 1) % C)
        torch.cuda.synchronize()
        r.train_many_clipped(d_imgs, labels, 0.05, 0.5)
        r.synchronize()
    r.close()


MODES = [binding.MODE_STAGES, binding.MODE_PERSISTENT, binding.MODE_RESIDENT]


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("name,limit", [("cfg1", 0.3), ("cfg1", math.inf), ("cfg5", 0.5), ("cfg1", 0.0)])
def test_clipped_steps(name, limit, mode):
    """Every step against the gradients that a second network of the same weights and mode gives: the norm to a rounding, the
    weights to the rounding of each step (those of the steps before are taken over)."""
    import torch
    wl = synth.WORKLOADS[name]
    g, _ = build_pair(wl)
    r, _ = build_pair(wl)
    for net in (g, r):
        net.set_mode(mode)
    n = 5
    imgs, labs = synth.images(wl, n), synth.labels(wl, n)
    d_imgs, d_labs = to_dev(imgs), to_dev(labs)
    norms = torch.full((n,), -1.0, device="cuda:0")
    lr = 0.05
    clipped = 0
    for t in range(n):
        before = g.get_weights().astype(np.float64)
        r.set_weights(before.astype(np.float32))
        grad = r.debug_gradients(d_imgs[t].contiguous(), int(labs[t])).astype(np.float64)
        N = math.sqrt(math.fsum(grad * grad))
        g.train_many_clipped(d_imgs[t:], d_labs[t:], lr, limit, norms[t:t + 1], n=1)
        g.synchronize()
        assert abs(float(norms[t]) - N) <= N * U * (1 + 1e-6)
        lim = float(np.float32(limit))
        clipped += N > lim
        step = float(np.float32(lr)) * (lim / N if N > lim else 1.0)
        want = before - step * grad
        assert (np.abs(g.get_weights() - want) <= np.abs(want) * U + step * np.abs(grad) * U * 1e-3).all()
    assert clipped == (0 if limit == math.inf else clipped) and (limit != 0.3 or clipped)
    # all of them in a call: the same bits
    one = g.get_weights()
    g2, _ = build_pair(wl)
    g2.set_mode(mode)
    norms2 = torch.zeros(n, device="cuda:0")
    g2.train_many_clipped(d_imgs, d_labs, lr, limit, norms2)
    g2.synchronize()
    np.testing.assert_array_equal(g2.get_weights(), one)
    assert torch.equal(norms, norms2)
    if limit == math.inf:     # no clipping: train_many, to rounding
        g2.set_weights(build_pair(wl)[0].get_weights())
        g2.train_many(d_imgs, d_labs, lr)
        g2.synchronize()
        assert np.abs(g2.get_weights() - one).max() <= 1e-5 * np.abs(one).max()
    for net in (g, r, g2):
        net.close()


@pytest.mark.parametrize("mode", MODES)
def test_an_image_with_a_bad_label_is_passed_over(mode):
    import torch
    wl = synth.WORKLOADS["cfg1"]
    imgs, labs = synth.images(wl, 3), synth.labels(wl, 3)
    d_imgs = to_dev(imgs)
    nets = []
    for bad in (True, False):
        g, _ = build_pair(wl)
        g.set_mode(mode)
        d_labs = to_dev(np.array([labs[0], -3, labs[2]], dtype=np.int32)) if bad else to_dev(labs[[0, 2]].copy())
        norms = torch.full((3,), -1.0, device="cuda:0")
        g.train_many_clipped(d_imgs if bad else d_imgs[[0, 2]].contiguous(), d_labs, 0.05, 0.2, norms if bad else norms[:2])
        if bad:
            with pytest.raises(binding.CnnError) as e:
                g.synchronize()
            assert e.value.code == binding.E_ARG and float(norms[1]) == 0.0 and float(norms[2]) > 0.0
        g.synchronize()
        nets.append(g.get_weights())
        g.close()
    np.testing.assert_array_equal(*nets)


def test_clipped_training_is_refused():
    wl = synth.WORKLOADS["cfg1"]
    g, _ = build_pair(wl)
    d_imgs, d_labs = to_dev(synth.images(wl, 1)), to_dev(synth.labels(wl, 1))
    for lr, limit in ((0.1, -1.0), (0.1, math.nan), (math.inf, 1.0)):
        with pytest.raises(binding.CnnError) as e:
            g.train_many_clipped(d_imgs, d_labs, lr, limit)
        assert e.value.code == binding.E_ARG
    g.close()


@pytest.mark.parametrize("rows,width,classes", [(64, 40, 10), (33, 64, 1501), (5, 32, 9001)])
@pytest.mark.parametrize("captured", [False, True])
def test_an_output_layer_trained_with_all_of_them(rows, width, classes, captured):
    """Scores, their gradient and the clipped update, a few steps, against the same in 64 bits.

    u = 2^-24, X = max|x|, W = max|w|, `off` how far weights are from those in 64 bits.  A sum (width terms) is off by z = width X
    off + (width + 2) u width X W, log p by 2 z and its own rounding, a gradient of the sums by 2 z / rows and u (log p + 20) of
    itself, a weight's gradient (rows terms, each at most 2 X / rows) by e = 4 X z + 2 X (rows + 60) u.  The norm is then off by
    the root of the number of weights times e, the factor by that share, and a step adds lr f e and lr f |g| times that share."""
    import torch
    gen = torch.Generator(device="cuda:0").manual_seed(classes)
    x = torch.randn(rows, width, generator=gen, device="cuda:0")
    labels = torch.randint(0, classes, (rows,), generator=gen, device="cuda:0", dtype=torch.int32)
    labels[1] = -1
    w = torch.randn(classes, width, generator=gen, device="cuda:0") * 0.05
    b = torch.zeros(classes, device="cuda:0")
    w64, b64 = w.double().cpu(), b.double().cpu()
    x64, l64 = x.double().cpu(), labels.long().cpu()
    dw, db = torch.empty_like(w), torch.empty_like(b)
    f = lambda *s: torch.empty(*s, device="cuda:0")  # noqa: E731
    logits, lp, h, norm, n2 = f(rows, classes), f(rows), f(rows), f(rows, 2), f(1)
    g_lp = torch.full((rows,), -1.0 / rows, device="cuda:0")
    g_h = torch.full((rows,), -0.1 / rows, device="cuda:0")
    s1 = torch.empty(binding.class_scores_scratch_bytes(rows, classes), dtype=torch.uint8, device="cuda:0")
    s2 = torch.empty(binding.gradient_scratch_bytes(2), dtype=torch.uint8, device="cuda:0")
    weights, grads = binding.TensorList([w, b]), binding.TensorList([dw, db])
    lr, limit = 0.5, 0.25

    def step():
        torch.addmm(b, x, w.t(), out=logits)
        binding.class_scores(logits, labels, lp, h, norm, d_scratch=s1)
        binding.class_scores_grad(logits, logits, norm, labels, g_lp, h, g_h)       # in place
        torch.mm(logits.t(), x, out=dw)
        torch.mv(logits.t(), ones, out=db)
        binding.clipped_update(weights, grads, lr, limit, s2, d_norm=n2)

    ones = torch.ones(rows, device="cuda:0")
    run = step
    if captured:
        keep = [t.clone() for t in (w, b)]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()                                     # (libraries set themselves up)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        w.copy_(keep[0])
        b.copy_(keep[1])
        run = graph.replay
    big = float(x.abs().max())
    off = 0.0
    for k in range(4):
        sums = width * big * off + (width + 2) * U * width * big * float(w64.abs().max())
        run()
        torch.cuda.synchronize()
        z = torch.nn.functional.log_softmax(x64 @ w64.t() + b64, 1)
        p = z.exp()
        has = (l64 >= 0).double()
        g = -p * has[:, None]
        g[torch.arange(rows), l64.clamp(min=0)] += has
        H = -(p * z).sum(1)
        g = (g * (-1.0 / rows) + 0.1 / rows * p * (z + H[:, None]))
        gw, gb = g.t() @ x64, g.sum(0)
        N = float((gw.square().sum() + gb.square().sum()).sqrt())
        scale = lr * min(1.0, limit / N)
        e = 4 * big * sums + 2 * big * (rows + 60) * U
        share = math.sqrt(w.numel() + b.numel()) * e / N + U
        assert abs(float(n2) - N) <= N * share, (float(n2), N)
        want_lp = torch.where(l64 >= 0, z[torch.arange(rows), l64.clamp(min=0)], torch.zeros(rows, dtype=torch.float64))
        assert ((lp.double().cpu() - want_lp).abs() <= 2 * sums + (classes / 64 + 120) * U * (2 + want_lp.abs())).all()
        off += scale * (e + float(gw.abs().max()) * share) + U * float(w64.abs().max())
        w64, b64 = w64 - scale * gw, b64 - scale * gb
        assert (w.double().cpu() - w64).abs().max() <= off and (b.double().cpu() - b64).abs().max() <= off


@pytest.mark.parametrize("name,arch", NETS)
@pytest.mark.parametrize("n,batch", [(1, 1), (7, 7), (50, 16), (300, 300)])
def test_a_sum_that_is_no_number(name, arch, n, batch):
    """A weight of NaN in the output layer: its class's sum is NaN for every image, whichever kernels add it up, so that no image has
    a distribution; and as before once the weight is a number again."""
    import torch
    g, o, images = _pair(name, arch)
    C, top = g.num_classes, min(g.num_classes, 3)
    d_imgs = to_dev(images(n))
    labels = torch.arange(n, dtype=torch.int32, device="cuda:0") % C
    labels[n // 2] = C
    scratch = torch.empty(g.forward_batch_scratch_bytes(batch), dtype=torch.uint8, device="cuda:0")

    def scores():
        lp, h, best = (torch.full(s, 9.0, device="cuda:0") for s in ((n,), (n,), (n, top)))
        which = torch.full((n, top), 9, dtype=torch.int32, device="cuda:0")
        torch.cuda.synchronize()
        g.score_batch(d_imgs, n, scratch, batch, labels, lp, h, which, best)
        g.synchronize()
        return lp, h, which, best

    weights = g.get_weights()
    first = scores()
    begin, end = layer_bounds(o)[-1]
    inputs = (end - begin) // C - 1
    for k in (0, C - 1):
        bad = weights.copy()
        bad[begin + C + k * inputs + inputs // 2] = math.nan
        g.set_weights(bad)
        lp, h, which, best = scores()
        has = labels < C
        assert lp[has].isnan().all() and (lp[~has] == 0).all() and h.isnan().all() and (which == -1).all() and best.isnan().all()
    g.set_weights(weights)
    assert all(torch.equal(a, b) for a, b in zip(first, scores()))
    g.close()


WIDE = [("cfg5", mode) for mode in MODES] + [("cfg4a", binding.MODE_STAGES), ("cfg4a", binding.MODE_RESIDENT), ("cfg4b", binding.MODE_STAGES)]


@pytest.mark.parametrize("name,mode", WIDE)
def test_an_image_with_a_bad_label_is_passed_over_by_a_large_net(name, mode):
    """As above where the update is two launches: the first has added up what gradients were left, the second leaves all alone."""
    import torch
    wl = synth.WORKLOADS[name]
    imgs, labs = synth.images(wl, 4), synth.labels(wl, 4)
    d_imgs = to_dev(imgs)
    weights, norms = [], []
    for bad in (True, False):
        g, _ = build_pair(wl)
        assert g.num_weights > 30 * 4096
        g.set_mode(mode)
        d_labs = to_dev(np.array([labs[0], -3, wl.n_classes, labs[3]], dtype=np.int32)) if bad else to_dev(labs[[0, 3]].copy())
        norms.append(torch.full((4,), -1.0, device="cuda:0"))
        g.train_many_clipped(d_imgs if bad else d_imgs[[0, 3]].contiguous(), d_labs, 0.05, 0.2, norms[-1] if bad else norms[-1][:2])
        if bad:
            with pytest.raises(binding.CnnError) as e:
                g.synchronize()
            assert e.value.code == binding.E_ARG
        g.synchronize()
        weights.append(g.get_weights())
        g.close()
    np.testing.assert_array_equal(*weights)
    assert (norms[0][1:3] == 0).all() and torch.equal(norms[0][[0, 3]], norms[1][:2]) and (norms[1][:2] > 0).all()


@pytest.mark.parametrize("name,mode", WIDE)
def test_clipped_steps_of_a_large_net(name, mode):
    """As test_clipped_steps, limits on both sides of the norms, with the winners' and the matrix cores' stages: every step clips, or none."""
    import torch
    wl = synth.WORKLOADS[name]
    g, _ = build_pair(wl)
    r, _ = build_pair(wl)
    for net in (g, r):
        net.set_mode(mode)
    n, lr = 3, 0.05
    imgs, labs = synth.images(wl, n), synth.labels(wl, n)
    d_imgs, d_labs = to_dev(imgs), to_dev(labs)
    norm = torch.full((1,), -1.0, device="cuda:0")
    for t in range(n):
        for share in (0.37, 1.7):
            before = g.get_weights().astype(np.float64)
            r.set_weights(before.astype(np.float32))
            grad = r.debug_gradients(d_imgs[t].contiguous(), int(labs[t])).astype(np.float64)
            N = math.sqrt(math.fsum(grad * grad))
            limit = float(np.float32(share * N))
            g.train_many_clipped(d_imgs[t:], d_labs[t:], lr, limit, norm, n=1)
            g.synchronize()
            assert abs(float(norm) - N) <= N * U * (1 + 1e-6)
            step = float(np.float32(lr)) * (limit / N if share < 1 else 1.0)
            want = before - step * grad
            assert (np.abs(g.get_weights() - want) <= np.abs(want) * U + step * np.abs(grad) * U * 1e-3).all()
    for net in (g, r):
        net.close()


def test_captured_clipped_steps():
    """Recorded in stage mode, and replayed on labels and weights as they are then; refused in the modes whose launches are cooperative,
    before anything is launched."""
    import torch
    wl = synth.WORKLOADS["cfg1"]
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        r, _ = build_pair(wl)
    g, _ = build_pair(wl)
    for net in (g, r):
        net.set_mode(binding.MODE_STAGES)
    n = 3
    d_imgs, d_labs = to_dev(synth.images(wl, n)), to_dev(synth.labels(wl, n))
    norms, want = torch.zeros(n, device="cuda:0"), torch.zeros(n, device="cuda:0")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        r.train_many_clipped(d_imgs, d_labs, 0.05, 0.3, norms)
    for _ in range(4):
        graph.replay()
        g.train_many_clipped(d_imgs, d_labs, 0.05, 0.3, want)
        torch.cuda.synchronize()
        assert torch.equal(norms, want) and (norms > 0).all()
        np.testing.assert_array_equal(r.get_weights(), g.get_weights())
        d_labs.copy_((d_labs + 1) % wl.n_classes)
        torch.cuda.synchronize()
    before = r.get_weights()
    some = torch.zeros(1, device="cuda:0")
    for mode in (binding.MODE_PERSISTENT, binding.MODE_RESIDENT):
        r.set_mode(mode)
        r.synchronize()
        with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=s):
            with pytest.raises(binding.CnnError) as e:
                r.train_many_clipped(d_imgs, d_labs, 0.05, 0.3, norms)
            some.add_(1)       # (a graph of something)
        assert e.value.code == binding.E_STATE
        np.testing.assert_array_equal(r.get_weights(), before)
        r.train_many_clipped(d_imgs, d_labs, 0.05, 0.3, norms)      # the handle goes on
        r.synchronize()
        assert (norms > 0).all()
        before = r.get_weights()
    for net in (g, r):
        net.close()
