"""Cases that time the operators around a language model's layers and its workers' gradients: layer norm, its gradient, the norm
over many tensors, and clipping.

Four operators.  `layer_norm`: rows of a batch normalised, with the residual sum where there is one.  `layer_norm_grad`: the
gradient of the rows, and of weight and bias per worker, into the workers' rows of a gradient buffer.  `grad_norm`: per worker the
norm over a list of gradients.  `clip`: the list scaled to a largest norm and laid into the workers' rows of the gradient buffer.

run() computes a case once: in elementary torch operations in 32 bits, or, where `own` is true, through the package's calls.
"""
import math

import torch

own = False

EPS, MAX_NORM, CLIP_EPS = 1e-5, 1.0, 1e-6
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "i32": torch.int32, "i64": torch.int64}


def _norm(name, workers, tokens, dim, x, y, param, masked=0.0, ids="i64", residual=False):
    return {"name": name, "op": "layer_norm", "workers": workers, "tokens": tokens, "dim": dim, "x": x, "y": y, "param": param, "masked": masked,
            "ids": ids, "residual": residual}


def _norm_grad(name, workers, tokens, dim, x, y, param, masked=0.0, ids="i64", residual=False, accumulate=False):
    return {**_norm(name, workers, tokens, dim, x, y, param, masked, ids, residual), "op": "layer_norm_grad", "accumulate": accumulate}


def _many(op, name, workers, model, src, dst="f32", layers=0, dim=0, vocab=0):
    return {"name": name, "op": op, "workers": workers, "model": model, "src": src, "dst": dst, "layers": layers, "dim": dim, "vocab": vocab}


def listed():
    return [
        # one token of a generating model: latency
        _norm("norm_1_token", 1, 1, 1024, "bf16", "bf16", "bf16"),
        # eight simulated workers' batches with padding, full-precision activations for low-precision products
        _norm("norm_8x4096x512", 8, 4096, 512, "f32", "bf16", "f32", 0.05),
        # a long batch of a large model, the residual sum taken on the way
        _norm("norm_65536x2048_residual", 1, 65536, 2048, "bf16", "bf16", "bf16", residual=True),
        # a few tokens of a fine-tuning step, added to weight gradients that are there
        _norm_grad("norm_grad_add_200", 1, 200, 768, "f32", "f32", "f32", accumulate=True),
        # eight simulated workers, weight gradients into each one's row
        _norm_grad("norm_grad_8x4096x512", 8, 4096, 512, "f32", "f32", "f32", 0.05),
        # an odd width
        _norm_grad("norm_grad_20011x1001", 1, 20011, 1001, "bf16", "bf16", "f32"),
        # a long batch of a large model, the residual stream's gradient added on the way
        _norm_grad("norm_grad_65536x2048_residual", 1, 65536, 2048, "bf16", "bf16", "bf16", residual=True),
        # the three parameters of a small text classifier, eight workers
        _many("grad_norm", "grad_norm_8_classifiers", 8, "classifier", "f32", dim=128, vocab=5000),
        # a language model's gradients in low precision, one process
        _many("grad_norm", "grad_norm_language_bf16", 1, "language", "bf16", layers=5, dim=1024, vocab=32000),
        # a small model's few tensors: latency
        _many("clip", "clip_small", 1, "language", "f32", layers=1, dim=32, vocab=500),
        # a language model's low-precision gradients clipped into a full-precision row
        _many("clip", "clip_language_bf16", 1, "language", "bf16", "f32", layers=5, dim=1024, vocab=32000),
        # ResNet-18's 62 tensors of a hundred workers, clipped into their rows of the gradient buffer
        _many("clip", "clip_100_resnet18", 100, "resnet18", "f32"),
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1))) - 0.5))))


def draw(rng):
    op = rng.choice(("layer_norm", "layer_norm_grad", "grad_norm", "clip"))
    if op in ("layer_norm", "layer_norm_grad"):
        dim = _log_int(rng, 16, 8192)
        if rng.random() < 0.5:
            dim = (dim + 7) // 8 * 8
        workers = rng.choice((1, 1, 2, 5, 16))
        tokens = min(_log_int(rng, 1, 130000 // workers), (1 << 27) // (dim * workers))
        rest = (workers, tokens, dim, rng.choice(("f32", "bf16")), rng.choice(("f32", "bf16")), rng.choice(("f32", "bf16")), rng.choice((0.0, 0.05, 0.4)),
                rng.choice(("i32", "i64")), rng.random() < 0.4)
        case = _norm("", *rest) if op == "layer_norm" else _norm_grad("", *rest, accumulate=rng.random() < 0.3)
    else:
        workers, model = rng.choice((1, 1, 3, 10, 32)), rng.choice(("classifier", "language", "resnet18", "row"))
        dim, layers = _log_int(rng, 8, 1024), rng.randint(1, 6)
        if model == "resnet18":
            workers = rng.randint(1, 40)
        vocab = min(_log_int(rng, 100, 60000), (1 << 28) // (dim * workers))
        if model == "language":
            layers = max(1, min(layers, (1 << 28) // (12 * dim * dim * workers)))
        if model == "row":      # one row of a gradient buffer
            dim = _log_int(rng, 1, min(1 << 25, (1 << 29) // workers))
        case = _many(op, "", workers, model, rng.choice(("f32", "bf16")), rng.choice(("f32", "bf16")) if op == "clip" else "f32",
                     layers if model == "language" else 0, 0 if model == "resnet18" else dim, vocab if model in ("classifier", "language") else 0)
    return {k: v for k, v in case.items() if k != "name"}


def _shapes(case):
    """The parameters of a model, in the order in which its gradient row holds them."""
    d, v = case["dim"], case["vocab"]
    if case["model"] == "row":
        return [(d,)]
    if case["model"] == "classifier":
        return [(v, d), (2 * d, d), (10, 2 * d)]
    if case["model"] == "language":
        layer = [(d,), (d,), (d, d), (d, d), (d, d), (d, d), (d,), (d,), (4 * d, d), (d, 4 * d)]
        return [(v, d)] + layer * case["layers"] + [(d,), (d,)]
    shapes, before = [(64, 3, 3, 3), (64,), (64,)], 64
    for width in (64, 128, 256, 512):
        for block in range(2):
            shapes += [(width, before, 3, 3), (width,), (width,), (width, width, 3, 3), (width,), (width,)]
            if before != width:
                shapes += [(width, before, 1, 1), (width,), (width,)]
            before = width
    return shapes + [(10, 512), (10,)]


def _ids(case, gen):
    """Token ids of which a share is empty places (-1): only their signs are looked at."""
    shape = (case["workers"], case["tokens"])
    ids = torch.randint(0, 30000, shape, generator=gen, device="cuda")
    return torch.where(torch.rand(shape, generator=gen, device="cuda") < case["masked"], torch.full_like(ids, -1), ids).to(DTYPES[case["ids"]])


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    state = {"case": case}

    def randn(shape, scale, dtype):
        return torch.randn(shape, generator=gen, device="cuda").mul_(scale).to(dtype)

    if case["op"] in ("layer_norm", "layer_norm_grad"):
        w, t, d = shape = (case["workers"], case["tokens"], case["dim"])
        x, y, param = DTYPES[case["x"]], DTYPES[case["y"]], DTYPES[case["param"]]
        # activations: tokens of different sizes, a few channels that stand out, an offset
        columns = torch.where(torch.rand((d,), generator=gen, device="cuda") < 0.01, 20.0, 1.0)
        state["x"] = (torch.randn(shape, generator=gen, device="cuda") * columns * (0.3 + torch.rand((w, t, 1), generator=gen, device="cuda")) + 0.2).to(x)
        state["weight"] = 1 + randn((d,), 0.1, torch.float32)
        state["weight"] = state["weight"].to(param)
        state["ids"] = _ids(case, gen) if case["masked"] else None
        if case["op"] == "layer_norm":
            state["bias"] = randn((d,), 0.1, param)
            state["y"] = torch.empty(shape, dtype=y, device="cuda")
            state["add"] = randn(shape, 0.5, x) if case["residual"] else None
            state["total"] = torch.empty(shape, dtype=x, device="cuda") if case["residual"] else None
        else:
            state["dy"] = randn(shape, 1e-3, y)
            state["dtotal"] = randn(shape, 1e-3, x) if case["residual"] else None
            state["dx"] = torch.empty(shape, dtype=x, device="cuda")
            state["grads"] = randn((w, 2 * d), 1e-2, torch.float32) if case["accumulate"] else torch.empty((w, 2 * d), device="cuda")
        return state
    w, shapes = case["workers"], _shapes(case)
    scales = 10 ** (torch.rand((len(shapes),), generator=gen, device="cuda") * 2 - 2)
    sizes = [math.prod(s) for s in shapes]
    state["grads"] = [randn((w,) + s, scales[i], DTYPES[case["src"]]) for i, s in enumerate(shapes)]
    state["norm"] = torch.empty((w,), device="cuda")
    if case["op"] == "clip":
        state["rows"] = torch.empty((w, sum(sizes)), dtype=DTYPES[case["dst"]], device="cuda")
        state["parts"] = [p.view((w,) + s) if w == 1 else p.unflatten(1, s) for p, s in zip(state["rows"].split(sizes, dim=1), shapes)]
    return state


def _plain(state):
    case = state["case"]
    if case["op"] in ("layer_norm", "layer_norm_grad"):
        x, weight = state["x"], state["weight"].float()
        if case["op"] == "layer_norm" and case["residual"]:
            state["total"].copy_(x.float() + state["add"].float())
            x = state["total"]
        x = x.float()
        off = x - x.mean(-1, keepdim=True)
        rstd = torch.rsqrt((off * off).mean(-1, keepdim=True) + EPS)
        there = None if state["ids"] is None else (state["ids"] >= 0).unsqueeze(-1)
        zero = torch.zeros((), device=x.device)
        if case["op"] == "layer_norm":
            y = off * rstd * weight + state["bias"].float()
            if there is not None:
                y = torch.where(there, y, zero)
                if case["residual"]:
                    state["total"].copy_(torch.where(there, state["total"].float(), zero))
            state["y"].copy_(y)
            return {"y": state["y"], "total": state["total"]} if case["residual"] else state["y"]
        dy = state["dy"].float()
        if there is not None:
            dy = torch.where(there, dy, zero)
        xhat = off * rstd
        g = dy * weight
        dx = rstd * (g - g.mean(-1, keepdim=True) - xhat * (g * xhat).mean(-1, keepdim=True))
        if case["residual"]:
            dx = dx + state["dtotal"].float()
        state["dx"].copy_(dx if there is None else torch.where(there, dx, zero))
        new = torch.cat([(dy * xhat).sum(1), dy.sum(1)], 1)
        state["grads"].copy_(state["grads"] + new if case["accumulate"] else new)
        return {"dx": state["dx"], "grads": state["grads"]}
    w = case["workers"]
    total = torch.zeros((w,), dtype=torch.float64, device="cuda")
    for g in state["grads"]:
        total += g.reshape(w, -1).float().square().sum(1, dtype=torch.float64)
    norm = torch.sqrt(total)
    state["norm"].copy_(norm)
    if case["op"] == "grad_norm":
        return state["norm"]
    c = (MAX_NORM / (norm + CLIP_EPS)).clamp(max=1.0).float()
    for g, p in zip(state["grads"], state["parts"]):
        p.copy_(g.float() * c.view((w,) + (1,) * (g.dim() - 1)))
    return {"rows": state["rows"], "norm": state["norm"]}


def run(state):
    if not own:
        return _plain(state)
    import paper_2302_07475_b200 as S
    case = state["case"]
    if case["op"] == "layer_norm":
        S.s3gd_layer_norm(state["x"], state["y"], state["weight"], state["bias"], eps=EPS, ids=state["ids"], add=state["add"], total=state["total"])
        return {"y": state["y"], "total": state["total"]} if case["residual"] else state["y"]
    if case["op"] == "layer_norm_grad":
        w, t, d = case["workers"], case["tokens"], case["dim"]
        if "ws" not in state:
            state["ws"] = S.alloc_layer_norm_workspace(w, t, d, state["x"].device)
        grads = state["grads"]
        S.s3gd_layer_norm_grad(state["dy"], state["x"], state["dx"], state["weight"], grads[:, :d], grads[:, d:], state["ws"], eps=EPS,
                               ids=state["ids"], dtotal=state["dtotal"], accumulate=case["accumulate"])
        return {"dx": state["dx"], "grads": grads}
    if "ws" not in state:
        state["ws"] = S.alloc_clip_workspace(case["workers"], state["norm"].device)
    if case["op"] == "grad_norm":
        S.s3gd_grad_norm(state["grads"], state["norm"], state["ws"])
        return state["norm"]
    S.s3gd_clip(state["grads"], MAX_NORM, state["norm"], state["ws"], out=state["parts"], eps=CLIP_EPS)
    return {"rows": state["rows"], "norm": state["norm"]}


def work(case):
    size = {k: torch.empty((), dtype=t).element_size() for k, t in DTYPES.items()}
    if case["op"] in ("layer_norm", "layer_norm_grad"):
        n, d, seen = case["workers"] * case["tokens"], case["dim"], 1 - case["masked"]
        x, y, more = size[case["x"]], size[case["y"]], 1 if case["residual"] else 0
        ids = n * size[case["ids"]] if case["masked"] else 0
        if case["op"] == "layer_norm":
            return {"bytes": n * d * (x * (seen + more * seen + more) + y) + 2 * d * size[case["param"]] + ids, "flops": 8 * seen * n * d}
        moved = n * d * (seen * (x + y + more * x) + x) + d * size[case["param"]] + ids
        return {"bytes": moved + case["workers"] * 2 * d * 4 * (2 if case["accumulate"] else 1), "flops": 16 * seen * n * d}
    n = case["workers"] * sum(math.prod(s) for s in _shapes(case))
    moved = size[case["src"]] + (size[case["dst"]] if case["op"] == "clip" else 0)
    return {"bytes": n * moved + 4 * case["workers"], "flops": (3 if case["op"] == "clip" else 2) * n}


def exact(case, seed):
    s = prepare(case, seed)
    f = torch.float64
    if case["op"] in ("layer_norm", "layer_norm_grad"):
        w, t, d = s["x"].shape
        x = s["x"].reshape(w * t, d)
        keep = torch.ones((w * t,), dtype=torch.bool, device="cuda") if s["ids"] is None else s["ids"].reshape(-1) >= 0
        weight = s["weight"].to(f)
        out = torch.zeros((w * t, d), dtype=f, device="cuda")
        total = torch.zeros((w * t, d), dtype=f, device="cuda") if case["residual"] else None
        sums = torch.zeros((w, 2 * d), dtype=f, device="cuda")
        for i in range(0, w * t, 4096):
            part = torch.nonzero(keep[i:i + 4096]).reshape(-1) + i
            u = x[part].to(f)
            if case["op"] == "layer_norm" and case["residual"]:
                total[part] = u + s["add"].reshape(w * t, d)[part].to(f)
                u = (u + s["add"].reshape(w * t, d)[part].to(f)).to(x.dtype).to(f)   # what later layers read is the rounded sum
            z = (u - u.mean(1, keepdim=True)) / torch.sqrt(u.var(1, unbiased=False, keepdim=True) + EPS)
            if case["op"] == "layer_norm":
                out[part] = z * weight + s["bias"].to(f)
                continue
            dy = s["dy"].reshape(w * t, d)[part].to(f)
            # the Jacobian of a row: (I - 1 1^T / d - z z^T / d) / sigma
            v = dy * weight
            v = v - v.sum(1, keepdim=True) / d - z * torch.einsum("td,td->t", v, z).unsqueeze(1) / d
            out[part] = v / torch.sqrt(u.var(1, unbiased=False, keepdim=True) + EPS)
            if case["residual"]:
                out[part] += s["dtotal"].reshape(w * t, d)[part].to(f)
            sums.index_add_(0, part // t, torch.cat([dy * z, dy], 1))
        out = out.view(w, t, d)
        if case["op"] == "layer_norm":
            return {"y": out, "total": total.view(w, t, d)} if case["residual"] else out
        return {"dx": out, "grads": s["grads"].to(f) + sums if case["accumulate"] else sums}
    w = case["workers"]
    norm = torch.stack([torch.sqrt(sum(torch.dot(r, r) for r in (g[m].reshape(-1).to(f) for g in s["grads"]))) for m in range(w)])
    if case["op"] == "grad_norm":
        return norm
    rows = torch.empty(s["rows"].shape, dtype=f, device="cuda")
    for m in range(w):
        c = min(1.0, MAX_NORM / (float(norm[m]) + CLIP_EPS))
        torch.cat([g[m].reshape(-1).to(f) for g in s["grads"]], out=rows[m])
        rows[m] *= c
    return {"rows": rows, "norm": norm}
