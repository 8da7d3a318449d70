"""Cases that time the operators for a language model's parameters: orthogonalised updates and the embedding table.

Four operators.  `orthogonalise`: Newton-Schulz products on a (batch of) matrices.  `step`: momentum, orthogonalise, update
of the parameters, in place.  `lookup`: rows of an embedding table by token, scaled.  `grad`: the table's gradient, summed
per token, written into (or added to) the workers' rows of a gradient buffer.

run() computes a case once: in elementary torch operations in 32 bits, or, where `own` is true, through the package's calls.
"""
import math

import torch

own = False

COEFFS = (3.4445, -4.7750, 2.0315)
EPS = 1e-7
MU, LR, DECAY = 0.95, 2e-3, 0.1
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "i8": torch.int8, "i32": torch.int32, "i64": torch.int64}


def _ortho(name, batch, rows, cols, src, dst, steps=5):
    return {"name": name, "op": "orthogonalise", "batch": batch, "rows": rows, "cols": cols, "src": src, "dst": dst, "steps": steps}


def _step(name, batch, rows, cols, src, dst, nesterov, steps=5):
    return {"name": name, "op": "step", "batch": batch, "rows": rows, "cols": cols, "src": src, "dst": dst, "nesterov": nesterov,
            "steps": steps}


def _lookup(name, tokens, vocab, dim, src, dst, ids, masked=0.0):
    return {"name": name, "op": "lookup", "workers": 1, "tokens": tokens, "vocab": vocab, "dim": dim, "src": src, "dst": dst, "ids": ids,
            "masked": masked}


def _grad(name, workers, tokens, vocab, dim, src, dst, ids, masked=0.0, accumulate=False):
    return {"name": name, "op": "grad", "workers": workers, "tokens": tokens, "vocab": vocab, "dim": dim, "src": src, "dst": dst, "ids": ids,
            "masked": masked, "accumulate": accumulate}


def listed():
    return [
        # the projections of 32 attention heads, each orthogonalised by itself: many small matrices, latency counts
        _ortho("ortho_heads_32x64x128", 32, 64, 128, "f32", "f32"),
        # a square projection of a small model, result in full precision
        _ortho("ortho_1024_f32", 1, 1024, 1024, "f32", "f32"),
        # a tall matrix with odd sides (a fused projection cut unevenly), low-precision gradients
        _ortho("ortho_2731x1000_bf16", 1, 2731, 1000, "bf16", "bf16"),
        # the largest: a square projection of a large model
        _ortho("ortho_8192_bf16", 1, 8192, 8192, "bf16", "bf16"),
        # the deepest convolution of ResNet-18 (512 x 512 x 3 x 3) as a matrix, fp32 parameters
        _step("step_conv_512x4608_f32", 1, 512, 4608, "f32", "f32", True),
        # a wide projection moved by the workers' majority vote: the int8 vote is the gradient
        _step("step_vote_1024x4096", 1, 1024, 4096, "i8", "f32", False),
        # the same projection of four layers at once, low-precision parameters and gradients
        _step("step_4x2048x2048_bf16", 4, 2048, 2048, "bf16", "bf16", True),
        # one token of a generating model: latency
        _lookup("lookup_1_token", 1, 32000, 1024, "bf16", "bf16", "i64"),
        # a training batch, an odd width, full-precision table read for low-precision activations
        _lookup("lookup_65536_f32", 65536, 50021, 1000, "f32", "bf16", "i32", 0.05),
        # a few tokens of a fine-tuning step added to a gradient that the tied output layer left behind
        _grad("grad_add_200", 1, 200, 8000, 768, "f32", "f32", "i64", 0.0, True),
        # eight simulated workers, each with tokens of its own, into their rows of the gradient buffer
        _grad("grad_8_workers_4096", 8, 4096, 16000, 512, "f32", "f32", "i64", 0.05),
        # a long batch over a large vocabulary: few words take a large part of the tokens
        _grad("grad_131072_bf16", 1, 131072, 65536, 2048, "bf16", "f32", "i32", 0.02),
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 1))) - 0.5))))


def draw(rng):
    op = rng.choice(("orthogonalise", "step", "lookup", "grad"))
    if op in ("orthogonalise", "step"):
        short = _log_int(rng, 16, 4096)
        long = int(short * rng.uniform(1.0, 4.0))
        rows, cols = (short, long) if rng.random() < 0.5 else (long, short)
        batch = 1 if rng.random() < 0.5 else _log_int(rng, 1, min(64, max(1, (1 << 25) // (short * long))))
        dst = rng.choice(("f32", "bf16"))
        if op == "orthogonalise":
            return {k: v for k, v in _ortho("", batch, rows, cols, rng.choice(("f32", "bf16", "i8")), dst).items() if k != "name"}
        return {k: v for k, v in _step("", batch, rows, cols, rng.choice(("f32", "bf16", "i8")), dst, rng.random() < 0.5).items() if k != "name"}
    vocab, dim = _log_int(rng, 500, 130000), _log_int(rng, 64, 4096)
    src, dst, ids, masked = rng.choice(("f32", "bf16")), rng.choice(("f32", "bf16")), rng.choice(("i32", "i64")), rng.choice((0.0, 0.05, 0.4))
    if op == "lookup":
        vocab = min(vocab, (1 << 27) // dim)
        return {k: v for k, v in _lookup("", min(_log_int(rng, 1, 130000), (1 << 27) // dim), vocab, dim, src, dst, ids, masked).items() if k != "name"}
    workers = rng.choice((1, 1, 2, 5, 10))
    vocab = max(500, min(vocab, (1 << 27) // (dim * workers)))
    tokens = min(_log_int(rng, 1, 130000 // workers), (1 << 28) // (dim * workers))
    return {k: v for k, v in _grad("", workers, tokens, vocab, dim, src, dst, ids, masked, rng.random() < 0.3).items() if k != "name"}


def _tokens(case, gen):
    """Token ids with the frequencies of a language (the r-th word about 1 / r), in no order of frequency; some are masked (-1)."""
    shape, vocab = (case["workers"], case["tokens"]), case["vocab"]
    cdf = torch.cumsum(1.0 / (torch.arange(vocab, device="cuda", dtype=torch.float64) + 2.7), 0)
    u = torch.rand(shape, generator=gen, device="cuda", dtype=torch.float64) * cdf[-1]
    ids = torch.randperm(vocab, generator=gen, device="cuda")[torch.searchsorted(cdf, u).clamp(max=vocab - 1)]
    ids = torch.where(torch.rand(shape, generator=gen, device="cuda") < case["masked"], torch.full_like(ids, -1), ids)
    return ids.to(DTYPES[case["ids"]])


def _gradient(case, gen):
    """A matrix's gradient: a part of low rank that the batch agrees on, and noise; for int8 the vote on it, with zeros where too few voted."""
    b, m, n = case["batch"], case["rows"], case["cols"]
    r = min(16, m, n)
    g = torch.randn((b, m, r), generator=gen, device="cuda") @ torch.randn((b, r, n), generator=gen, device="cuda") / math.sqrt(r)
    g += 0.5 * torch.randn((b, m, n), generator=gen, device="cuda")
    if case["src"] == "i8":
        return torch.where(g.abs() > 1.0, torch.sign(g), torch.zeros_like(g)).to(torch.int8)
    return (1e-3 * g).to(DTYPES[case["src"]])


def prepare(case, seed):
    gen = torch.Generator("cuda").manual_seed(seed)
    src, dst = DTYPES[case["src"]], DTYPES[case["dst"]]
    state = {"case": case}
    if case["op"] in ("orthogonalise", "step"):
        shape = (case["batch"], case["rows"], case["cols"])
        state["g"] = _gradient(case, gen)
        if case["op"] == "orthogonalise":
            state["out"] = torch.empty(shape, dtype=dst, device="cuda")
        else:
            state["x"] = (0.02 * torch.randn(shape, generator=gen, device="cuda")).to(dst)
            state["v"] = state["g"].float() * 4 + torch.randn(shape, generator=gen, device="cuda") * (1.0 if src == torch.int8 else 1e-3)
            state["scale"] = 0.2 * math.sqrt(max(case["rows"], case["cols"]))
        return state
    w, t, v, d = case["workers"], case["tokens"], case["vocab"], case["dim"]
    state["ids"] = _tokens(case, gen)
    state["scale"] = math.sqrt(d)
    if case["op"] == "lookup":
        state["table"] = (0.02 * torch.randn((v, d), generator=gen, device="cuda")).to(src)
        state["out"] = torch.empty((w, t, d), dtype=dst, device="cuda")
    else:
        state["dout"] = (1e-3 * torch.randn((w, t, d), generator=gen, device="cuda")).to(src)
        state["grads"] = torch.empty((w, v * d), dtype=dst, device="cuda")
        if case["accumulate"]:
            state["grads"].copy_(1e-2 * torch.randn((w, v * d), generator=gen, device="cuda"))
    return state


def _newton_schulz(u, steps):
    tall = u.shape[-2] > u.shape[-1]
    x = u.mT if tall else u
    x = x / (torch.sqrt((x * x).sum(dim=(-2, -1), keepdim=True)) + EPS)
    a, b, c = COEFFS
    for _ in range(steps):
        s = x @ x.mT
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.mT if tall else x


def _plain(state):
    case = state["case"]
    if case["op"] == "orthogonalise":
        state["out"].copy_(_newton_schulz(state["g"].float(), case["steps"]))
        return state["out"]
    if case["op"] == "step":
        g, x, v = state["g"].float(), state["x"], state["v"]
        v.mul_(MU).add_(g)
        u = g + MU * v if case["nesterov"] else v
        x.copy_(x.float() * (1 - LR * DECAY) - (LR * state["scale"]) * _newton_schulz(u, case["steps"]))
        return {"x": x, "v": v}
    ids, scale = state["ids"], state["scale"]
    there = (ids >= 0).unsqueeze(-1)
    if case["op"] == "lookup":
        rows = state["table"][ids.clamp(min=0).long()].float() * scale
        state["out"].copy_(torch.where(there, rows, torch.zeros_like(rows)))
        return state["out"]
    w, v, d = case["workers"], case["vocab"], case["dim"]
    at = ids.clamp(min=0).long() + v * torch.arange(w, device=ids.device).unsqueeze(-1)
    rows = torch.where(there, state["dout"].float(), torch.zeros((), device=ids.device)) * scale
    total = state["grads"].float().reshape(w * v, d) if case["accumulate"] else torch.zeros((w * v, d), device=ids.device)
    total.index_add_(0, at.reshape(-1), rows.reshape(-1, d))
    state["grads"].copy_(total.reshape(w, v * d))
    return state["grads"]


def run(state):
    if not own:
        return _plain(state)
    import paper_2302_07475_b200 as S
    case = state["case"]
    if case["op"] == "orthogonalise":
        if "ws" not in state:
            state["ws"] = S.alloc_ortho_workspace(case["batch"], case["rows"], case["cols"], state["g"].device)
        S.s3gd_orthogonalise(state["g"], state["out"], state["ws"], steps=case["steps"], coeffs=COEFFS, eps=EPS)
        return state["out"]
    if case["op"] == "step":
        if "ws" not in state:
            state["ws"] = S.alloc_ortho_workspace(case["batch"], case["rows"], case["cols"], state["g"].device)
        S.s3gd_step_ortho(state["x"], state["g"], LR, state["ws"], v=state["v"], mu=MU, nesterov=case["nesterov"], weight_decay=DECAY,
                          scale=state["scale"], steps=case["steps"], coeffs=COEFFS, eps=EPS)
        return {"x": state["x"], "v": state["v"]}
    if case["op"] == "lookup":
        S.s3gd_embed(state["table"], state["ids"], state["out"], scale=state["scale"])
        return state["out"]
    if "ws" not in state:
        state["ws"] = S.alloc_embed_workspace(case["workers"], case["tokens"], case["vocab"], case["dim"], state["ids"].device)
    S.s3gd_embed_grad(state["dout"], state["ids"], state["grads"], case["vocab"], state["ws"], scale=state["scale"],
                      accumulate=case["accumulate"])
    return state["grads"]


def work(case):
    size = {k: torch.empty((), dtype=t).element_size() for k, t in DTYPES.items()}
    if case["op"] in ("orthogonalise", "step"):
        n = case["batch"] * case["rows"] * case["cols"]
        short, long = sorted((case["rows"], case["cols"]))
        # per iteration: two symmetric products (half of their entries) and the product with the matrix itself
        flops = case["batch"] * case["steps"] * (short * short * long + short ** 3 + 2 * short * short * long)
        moved = size[case["src"]] + (size[case["dst"]] if case["op"] == "orthogonalise" else 2 * size[case["dst"]] + 8)
        return {"bytes": n * moved, "flops": flops}
    t, d = case["workers"] * case["tokens"], case["dim"]
    seen = t * (1 - case["masked"])
    moved = t * size[case["ids"]]
    if case["op"] == "lookup":
        return {"bytes": moved + min(seen, case["vocab"]) * d * size[case["src"]] + t * d * size[case["dst"]], "flops": t * d}
    moved += seen * d * size[case["src"]]
    table = case["workers"] * case["vocab"]
    moved += (2 * min(seen, table) if case["accumulate"] else table) * d * size[case["dst"]]
    return {"bytes": moved, "flops": 2 * seen * d}


def exact(case, seed):
    s = prepare(case, seed)
    f = torch.float64
    if case["op"] in ("orthogonalise", "step"):
        g = s["g"].to(f)
        u = g
        if case["op"] == "step":
            v = MU * s["v"].to(f) + g
            u = g + MU * v if case["nesterov"] else v
        y = u / (torch.linalg.vector_norm(u, dim=(1, 2)).view(-1, 1, 1) + EPS)
        a, b, c = COEFFS
        for _ in range(case["steps"]):  # on the side that is shorter; a y + b (y y') y + c (y y')^2 y either way
            if case["rows"] <= case["cols"]:
                p = torch.bmm(y, y.transpose(1, 2))
                z = torch.bmm(p, y)
                y = a * y + b * z + c * torch.bmm(p, z)
            else:
                p = torch.bmm(y.transpose(1, 2), y)
                z = torch.bmm(y, p)
                y = a * y + b * z + c * torch.bmm(z, p)
        if case["op"] == "orthogonalise":
            return y
        return {"x": s["x"].to(f) - LR * DECAY * s["x"].to(f) - LR * s["scale"] * y, "v": v}
    ids = s["ids"].long()
    if case["op"] == "lookup":
        out = torch.zeros((1, case["tokens"], case["dim"]), dtype=f, device="cuda")
        out[ids >= 0] = s["table"][ids[ids >= 0]].to(f) * s["scale"]
        return out
    total = s["grads"].to(f) if case["accumulate"] else torch.zeros(s["grads"].shape, dtype=f, device="cuda")
    for w in range(case["workers"]):
        keep = torch.nonzero(ids[w] >= 0).reshape(-1)
        table = total[w].view(case["vocab"], case["dim"])
        for part in keep.split(1 << 14):
            table.index_add_(0, ids[w][part], s["dout"][w][part].to(f) * s["scale"])
    return total
