"""What the operators at the two ends of training are measured on: the scores of classes and their gradient, the norm of
gradients over many tensors, clipping by it and the update with clipped gradients.

Five kinds of pass:

  scores  log probability of every row's label, entropy, normaliser and the best classes (class_scores)
  grad    the gradient of log probability and entropy with respect to the sums (class_scores_grad)
  norm    the 2-norm over all tensors of a list (gradient_norm)
  clip    the gradients scaled to at most a given norm (clip_gradients)
  update  w - lr * factor * g with that factor (clipped_update)

Each is there in its plain form, elementary torch operations in 32 bits, and as calls of the library's operators.
"""
import math
import random

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}

# Weight tensors of the benchmark's nets, layer by layer: biases, then weights.
NETS = {
    # 1x29x29-20C4-MP2-40C5-MP3-150N-10N
    "digits": (20, 320, 40, 20000, 150, 54000, 10, 1500),
    # 3x32x32-300C3-MP2-300C2-MP2-300C4-MP2-300N-10N
    "colour-small-kernels": (300, 8100, 300, 360000, 300, 1440000, 300, 360000, 10, 3000),
}


def _scores(name, kind, rows, classes, dtype, top=0, pad=0, masked=False):
    return {"name": name, "kind": kind, "rows": rows, "classes": classes, "dtype": dtype, "top": top, "pad": pad, "masked": masked}


def _list(name, kind, net, dtype, max_norm, blocks=0, width=0):
    return {"name": name, "kind": kind, "net": net, "blocks": blocks, "width": width, "dtype": dtype, "max_norm": max_norm}


def listed():
    return [
        # a test set of 10000 digits: error, entropy and the three best of ten classes
        _scores("scores-digits-10000", "scores", 10000, 10, "f32", top=3),
        # one row over a large set of classes, as each answer of a serving loop needs it
        _scores("scores-one-row", "scores", 1, 131072, "bf16", top=20),
        # a few rows, an odd number of classes, some of them switched off, rows in a wider buffer
        _scores("scores-odd-rows", "scores", 37, 100003, "f32", top=5, pad=5, masked=True),
        # scoring a long batch of rows, 20 alternatives each: the largest
        _scores("scores-batch", "scores", 4096, 131072, "bf16", top=20),
        # cross-entropy and entropy term of a batch of digits
        _scores("grad-digits-10000", "grad", 10000, 10, "f32"),
        # the same over many classes, an odd number of them, in halves
        _scores("grad-odd-classes", "grad", 2000, 50001, "f16"),
        # the gradients of the benchmark net, looked at after every image
        _list("norm-digits", "norm", "digits", "f32", 1.0),
        # a thousand million 16-bit gradients in 160 tensors
        _list("norm-large", "norm", "", "bf16", 1.0, blocks=20, width=2048),
        # the gradients of the widest colour net, clipped
        _list("clip-widest", "clip", "colour-small-kernels", "f32", 1.0),
        # 250 million gradients in 320 tensors of an odd width
        _list("clip-large", "clip", "", "bf16", 1.0, blocks=40, width=719),
        # one clipped step of on-line training on the benchmark net
        _list("update-digits", "update", "digits", "f32", 0.1),
        # 200 million 32-bit weights and their 16-bit gradients
        _list("update-large", "update", "", "bf16", 1.0, blocks=4, width=2048),
    ]


def _log_int(rng, lo, hi):
    """An integer in [lo, hi], evenly spread over the logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng: random.Random):
    kind = rng.choice(["scores", "scores", "scores", "grad", "grad", "norm", "clip", "update"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    if kind in ("scores", "grad"):
        most = 4096 * 131072 if kind == "scores" else 2000 * 50001
        while True:
            rows, classes = _log_int(rng, 1, 20000), _log_int(rng, 2, 200000)
            if rows * classes * SIZE[dtype] <= most * 2:
                break
        top = rng.choice([0, 1, rng.randint(1, 64)]) if kind == "scores" else 0
        case = _scores("", kind, rows, classes, dtype, top=min(top, classes), pad=rng.choice([0, rng.randint(1, 64)]),
                       masked=rng.random() < 0.4)
    else:
        limit = rng.choice([0.01, 1.0, 1e6])   # most gradients are over the first, none over the last
        if rng.random() < 0.3:
            case = _list("", kind, rng.choice(sorted(NETS)), dtype, limit)
        else:
            most = {"norm": 1_000_000_000, "clip": 240_000_000, "update": 200_000_000}[kind] * 2 // (SIZE[dtype] if kind != "update" else 2)
            while True:
                blocks, width = _log_int(rng, 1, 60), _log_int(rng, 16, 2048)
                if 12 * blocks * width * width <= most:
                    break
            case = _list("", kind, "", dtype, limit, blocks=blocks, width=width)
    del case["name"]
    return case


# ---- what a program has in hand ------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _counts(case):
    """Elements of every tensor: a net's layers, or blocks of four square matrices, two of four times that, two vectors."""
    if case["net"]:
        return list(NETS[case["net"]])
    w = case["width"]
    return case["blocks"] * [w, w * w, w * w, w * w, w * w, w, 4 * w * w, 4 * w * w]


def _views(flat, counts):
    """The tensors of a list as they lie in one buffer, one right behind the other."""
    return list(flat.split(counts))


def prepare(case, seed):
    gen = _generator(seed)
    state = {"case": case}
    if case["kind"] in ("scores", "grad"):
        rows, classes, top = case["rows"], case["classes"], case["top"]
        wide = torch.empty(rows, classes + case["pad"], dtype=TYPES[case["dtype"]], device=DEVICE)
        wide.normal_(0.0, 2.5, generator=gen)
        x = wide[:, :classes]
        labels = torch.randint(0, classes, (rows,), generator=gen, device=DEVICE, dtype=torch.int32)
        sure = torch.rand(rows, generator=gen, device=DEVICE)   # how far the label stands out of the other classes
        x[torch.arange(rows, device=DEVICE), labels.long()] += (12.0 * sure).to(x.dtype)
        if case["masked"]:
            off = torch.rand(classes, generator=gen, device=DEVICE) < 0.3     # classes that are switched off
            x.masked_fill_(off, -math.inf)
            x[5::11] = -math.inf                                              # rows that nothing is left of
        labels[3::16] = -1                                                    # rows without a label
        state |= {"x": x, "labels": labels}
        f = lambda *n: torch.empty(*n, dtype=torch.float32, device=DEVICE)  # noqa: E731
        if case["kind"] == "scores":
            state |= {"log_probs": f(rows), "entropy": f(rows), "normaliser": f(rows, 2), "top_log_probs": f(rows, top),
                      "top": torch.empty(rows, top, dtype=torch.int32, device=DEVICE)}
            if own:
                from paper_1102_0183_amd import binding
                state["scratch"] = torch.empty(binding.class_scores_scratch_bytes(rows, classes, top), dtype=torch.uint8, device=DEVICE)
        else:   # what the scoring of the same rows left behind, and the weight of every row in the error
            m = x.amax(1).double()
            d = torch.where(torch.isneginf(x), -math.inf, x.double() - m.clamp(min=-1e300)[:, None])
            s = d.exp().sum(1)
            h = s.log() - torch.where(torch.isneginf(d), 0.0, d.exp() * d).sum(1) / s
            state["normaliser"] = torch.stack([m, s.log()], 1).float().contiguous()
            state["entropy"] = torch.where(s > 0, h, 0.0).float()
            state["g_log_probs"] = -torch.rand(rows, generator=gen, device=DEVICE)
            state["g_entropy"] = 0.01 * torch.randn(rows, generator=gen, device=DEVICE)
            state["grad"] = torch.empty(rows, classes, dtype=x.dtype, device=DEVICE)
        return state
    counts = _counts(case)
    flat = torch.empty(sum(counts), dtype=TYPES[case["dtype"]], device=DEVICE).normal_(0.0, 1e-3, generator=gen)
    state |= {"grads": _views(flat, counts), "norm": torch.empty(1, dtype=torch.float32, device=DEVICE)}
    if case["kind"] == "clip":
        state["clipped"] = torch.empty_like(flat)
    if case["kind"] == "update":
        state["weights"] = torch.empty(flat.shape, dtype=torch.float32, device=DEVICE).uniform_(-0.05, 0.05, generator=gen)
    if own:
        from paper_1102_0183_amd import binding
        state["list"] = binding.TensorList(state["grads"])
        state["scratch"] = torch.empty(binding.gradient_scratch_bytes(len(counts)), dtype=torch.uint8, device=DEVICE)
        if case["kind"] == "clip":
            state["out_list"] = binding.TensorList(_views(state["clipped"], counts))
        if case["kind"] == "update":
            state["weight_list"] = binding.TensorList(_views(state["weights"], counts))
    else:
        for name, flat in (("out", "clipped"), ("weight", "weights")):
            if flat in state:
                state[name] = _views(state[flat], counts)
    return state


LR = 1e-3


# ---- a pass --------------------------------------------------------------------------------------------------

def _plain_scores(state):
    x, labels, top = state["x"].float(), state["labels"].long(), state["case"]["top"]
    m = x.amax(1)
    empty = torch.isneginf(m)
    d = x - torch.where(empty, 0.0, m)[:, None]
    e = torch.exp(d)
    s = e.sum(1)
    log_s = torch.log(s)
    at = d.gather(1, labels.clamp(min=0)[:, None])[:, 0]
    log_probs = torch.where(empty, -math.inf, at - log_s)
    log_probs = torch.where((labels >= 0) & (labels < x.shape[1]), log_probs, 0.0)
    entropy = torch.where(empty, 0.0, log_s - torch.where(e > 0, e * d, 0.0).sum(1) / s)
    # the best first, the lowest index among equals: 64-bit keys, values in their order as whole numbers in front
    bits = (x + 0.0).view(torch.int32)
    bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    index = torch.arange(x.shape[1], device=x.device)
    best = torch.topk(bits * (1 << 32) + (0x7FFFFFFF - index), top, dim=1).indices
    top_log_probs = torch.where(empty[:, None], -math.inf, d.gather(1, best) - log_s[:, None])
    return {"log_probs": log_probs, "entropy": entropy, "normaliser": torch.stack([m, log_s], 1),
            "top": best.int(), "top_log_probs": top_log_probs}


def _plain_grad(state):
    x, labels, norm = state["x"].float(), state["labels"].long()[:, None], state["normaliser"]
    empty = torch.isneginf(norm[:, 0])[:, None]
    log_p = torch.where(empty, -math.inf, (x - norm[:, :1]) - norm[:, 1:])
    p = torch.exp(log_p)
    g_l = torch.where((labels >= 0) & ~empty, state["g_log_probs"][:, None], 0.0)
    term = state["g_entropy"][:, None] * (log_p + state["entropy"][:, None])
    hit = torch.arange(x.shape[1], device=x.device) == labels
    return (torch.where(hit, g_l, 0.0) - torch.where(p > 0, p * (g_l + term), 0.0)).to(state["x"].dtype)


def _plain_norm(grads):
    return torch.stack([g.float().square().sum(dtype=torch.float64) for g in grads]).sum().sqrt()


def run(state):
    case = state["case"]
    kind = case["kind"]
    if own:
        from paper_1102_0183_amd import binding
        if kind == "scores":
            binding.class_scores(state["x"], d_labels=state["labels"], d_log_probs=state["log_probs"], d_entropy=state["entropy"],
                                 d_normaliser=state["normaliser"], d_top=state["top"], d_top_log_probs=state["top_log_probs"],
                                 d_scratch=state["scratch"])
            return {k: state[k] for k in ("log_probs", "entropy", "normaliser", "top", "top_log_probs")}
        if kind == "grad":
            binding.class_scores_grad(state["x"], state["grad"], state["normaliser"], d_labels=state["labels"],
                                      d_g_log_probs=state["g_log_probs"], d_entropy=state["entropy"], d_g_entropy=state["g_entropy"])
            return state["grad"]
        if kind == "norm":
            binding.gradient_norm(state["list"], state["norm"], state["scratch"])
            return state["norm"]
        if kind == "clip":
            binding.clip_gradients(state["list"], case["max_norm"], state["scratch"], out=state["out_list"], d_norm=state["norm"])
            return {"clipped": state["clipped"], "norm": state["norm"]}
        binding.clipped_update(state["weight_list"], state["list"], LR, case["max_norm"], state["scratch"], d_norm=state["norm"])
        return {"weights": state["weights"], "norm": state["norm"]}
    if kind == "scores":
        return _plain_scores(state)
    if kind == "grad":
        return _plain_grad(state)
    norm = _plain_norm(state["grads"])
    if kind == "norm":
        return norm.float().view(1)
    fine = torch.isfinite(norm)
    factor = torch.where(fine & (norm > case["max_norm"]), case["max_norm"] / norm, 1.0).float()
    if kind == "clip":
        [o.copy_(g.float() * factor) for o, g in zip(state["out"], state["grads"])]
        return {"clipped": state["clipped"], "norm": norm.float().view(1)}
    step = torch.where(fine, LR * factor, 0.0)
    [w.sub_(step * g.float()) for w, g in zip(state["weight"], state["grads"])]
    return {"weights": state["weights"], "norm": norm.float().view(1)}


# ---- what a pass cannot do without ---------------------------------------------------------------------------

def work(case):
    """Every input read once, every output written once.  Sums: a difference, an exponential, a sum, a product and a sum for
    the entropy, a comparison for the best classes (scores); two flops a gradient for the norm, one or two to use it."""
    size = SIZE[case["dtype"]]
    if case["kind"] in ("scores", "grad"):
        n = case["rows"] * case["classes"]
        if case["kind"] == "scores":
            return {"bytes": n * size + case["rows"] * (4 + 4 + 4 + 8 + 8 * case["top"]), "flops": 6 * n}
        return {"bytes": 2 * n * size + case["rows"] * (4 + 8 + 4 + 4 + 4), "flops": 7 * n}
    n = sum(_counts(case))
    if case["kind"] == "norm":
        return {"bytes": n * size + 4, "flops": 2 * n}
    if case["kind"] == "clip":
        return {"bytes": 2 * n * size + 4, "flops": 3 * n}
    return {"bytes": n * (size + 8) + 4, "flops": 4 * n}


# ---- the definition in 64 bits -------------------------------------------------------------------------------

def _exact_rows(x, label, top):
    """Scores of a few rows."""
    lse = torch.logsumexp(x, 1)
    log_p = x - lse[:, None]
    p = log_p.exp()
    alive = lse > -math.inf
    entropy = torch.special.entr(torch.where(alive[:, None], p, 0.0)).sum(1)
    log_p = torch.where(alive[:, None], log_p, -math.inf)
    lp = torch.where(label >= 0, log_p[torch.arange(len(x), device=x.device), label.clamp(min=0)], 0.0)
    best = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :top]
    m = x.max(1).values
    return lp, entropy, torch.stack([m, torch.where(alive, lse - m, -math.inf)], 1), best.int(), log_p.gather(1, best)


def exact(case, seed):
    global own
    was, own = own, False
    try:
        state = prepare(case, seed)
    finally:
        own = was
    if case["kind"] in ("scores", "grad"):
        x, labels = state["x"], state["labels"].long()
        step = max(1, (1 << 25) // case["classes"])
        got = []
        for r in range(0, case["rows"], step):
            a, l = x[r:r + step].double(), labels[r:r + step]
            if case["kind"] == "scores":
                got.append(_exact_rows(a, l, case["top"]))
                continue
            # with the entropy and the normaliser that the call is given
            m, s = state["normaliser"][r:r + step].double().unbind(1)
            h, g_l, g_h = (state[k][r:r + step].double()[:, None] for k in ("entropy", "g_log_probs", "g_entropy"))
            log_p = a - (m + s)[:, None]
            p = log_p.exp()
            g = -p * g_l * (l >= 0)[:, None] - g_h * (h * p - torch.special.entr(p))
            at = torch.arange(len(a), device=a.device)[l >= 0]
            g[at, l[l >= 0]] += g_l[l >= 0, 0]
            got.append((torch.where(m[:, None] == -math.inf, 0.0, g),))
        out = [torch.cat(v) for v in zip(*got)]
        return out[0] if case["kind"] == "grad" else dict(zip(("log_probs", "entropy", "normaliser", "top", "top_log_probs"), out))
    parts = [g.double() for g in state["grads"]]
    norm = math.sqrt(math.fsum(float(g.dot(g)) for g in parts))
    share = case["max_norm"] / norm if norm > case["max_norm"] else 1.0
    as_output = torch.tensor([norm], dtype=torch.float64, device=DEVICE)
    if case["kind"] == "norm":
        return as_output
    g = torch.cat(parts)
    if case["kind"] == "clip":
        return {"clipped": g * share, "norm": as_output}
    return {"weights": state["weights"].double() - LR * share * g, "norm": as_output}
