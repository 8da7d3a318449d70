"""s3gd_orthogonalise and s3gd_step_ortho on the GPU against the 64-bit statement.

Tolerances (relative, in the Frobenius norm of one matrix).  A step stores three matrices, each rounded independently to p
bits; what one rounding brings is amplified at most about threefold by the products that follow, and independent errors add
in squares, so `steps` steps held in p bits give 3 * sqrt(3 * steps) * 2^-(p+1).  Two 16-bit pieces hold 22 bits, one 11.
fp32 accumulation adds a few 2^-24 per product of the same kind: another 3 * sqrt(3 * steps) * 2^-22.  The result's own
rounding in bf16 is at most 2^-8 of an entry, spread evenly below that: less than 2^-9 in the norm.  A part of low rank that is `ratio` times stronger than the rest makes every error relative
to the rest larger by `ratio`.
"""
import numpy as np
import pytest
import torch

import paper_2302_07475_b200 as S
from oracle import operators_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda"
C = (3.4445, -4.7750, 2.0315)
EPS = 1e-7


def tolerance(dtype, steps=5, split=None, ratio=1.0):
    split = (steps if dtype == torch.float32 else min(2, steps)) if split is None else split
    inner = 3 * np.sqrt(3 * steps) * (2.0 ** -23 + 2.0 ** -22) * ratio
    if split < steps:
        inner += 3 * np.sqrt(3 * (steps - split)) * 2.0 ** -12 * (ratio if split == 0 else 1.0)
    return inner + (2.0 ** -9 if dtype == torch.bfloat16 else 0.0)


def rand(shape, dtype, seed, scale=1.0):
    g = torch.Generator(DEV).manual_seed(seed)
    t = torch.randn(shape, generator=g, device=DEV) * scale
    return torch.sign(t).mul_(t.abs() > 0.4).to(torch.int8) if dtype == torch.int8 else t.to(dtype)


def workspace(shape):
    b = shape[0] if len(shape) == 3 else 1
    ws = S.alloc_ortho_workspace(b, shape[-2], shape[-1], DEV)
    ws.fill_(255)                                   # NaN in every format: nothing may be read before it is written
    return ws


def ortho(g, dtype, **kw):
    out, ws = torch.full(g.shape, 7.0, dtype=dtype, device=DEV), workspace(g.shape)
    S.s3gd_orthogonalise(g, out, ws, **kw)
    S.s3gd_device_status(ws)
    return out


def near(got, want, tol):
    got, want = got.double().cpu().numpy(), np.asarray(want)
    got, want = (a.reshape((-1,) + a.shape[-2:]) for a in (got, want))
    for k in range(got.shape[0]):
        size = np.linalg.norm(want[k])
        off = np.linalg.norm(got[k] - want[k])
        assert off <= tol * size, f"matrix {k}: off by {off / max(size, 1e-300):.3g}, allowed {tol:.3g}"


SHAPES = [(1, 1), (1, 7), (7, 1), (2, 2), (3, 5), (16, 16), (17, 40), (64, 64), (64, 128), (128, 64), (65, 130), (127, 127), (128, 128),
          (128, 256), (128, 300), (129, 129), (129, 257), (100, 1000), (1000, 100), (30, 2000), (256, 256), (300, 300), (513, 700), (640, 511)]


@pytest.mark.parametrize("src", [torch.float32, torch.bfloat16, torch.int8])
@pytest.mark.parametrize("dst", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", SHAPES)
def test_against_the_statement(shape, src, dst):
    g = rand(shape, src, 1 + shape[0])
    near(ortho(g, dst), O.orthogonalise(g.double().cpu().numpy(), 5, C, EPS), tolerance(dst))


@pytest.mark.parametrize("dst", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(5, 33, 48), (3, 48, 33), (70, 64, 64), (3, 130, 200), (2, 300, 140)])
def test_batches(shape, dst):
    g = rand(shape, torch.float32, 3) * torch.logspace(-6, 6, shape[0], device=DEV)[:, None, None]   # each with a norm of its own
    near(ortho(g, dst), O.orthogonalise(g.double().cpu().numpy(), 5, C, EPS), tolerance(dst))


@pytest.mark.parametrize("split", [0, 1, 3, 5])
@pytest.mark.parametrize("shape", [(60, 90), (200, 333)])
def test_split_steps(shape, split):
    g = rand(shape, torch.float32, 5)
    near(ortho(g, torch.float32, split_steps=split), O.orthogonalise(g.double().cpu().numpy(), 5, C, EPS), tolerance(torch.float32, 5, split))


@pytest.mark.parametrize("shape", [(60, 90), (333, 200)])
@pytest.mark.parametrize("dst", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("steps,coeffs", [(1, C), (2, C), (7, C), (12, (1.5, -0.5, 0.0)), (3, (1.0, 0.0, 0.0))])
def test_steps_and_coefficients(shape, dst, steps, coeffs):
    g = rand(shape, torch.float32, 6)
    near(ortho(g, dst, steps=steps, coeffs=coeffs), O.orthogonalise(g.double().cpu().numpy(), steps, coeffs, EPS), tolerance(dst, steps))


@pytest.mark.parametrize("shape", [(100, 128), (256, 384)])
@pytest.mark.parametrize("dst", [torch.float32, torch.bfloat16])
def test_low_rank_signal_above_noise(shape, dst):
    ratio = 10.0
    g = rand((shape[0], 8), torch.float32, 7) @ rand((8, shape[1]), torch.float32, 8) / 8 ** 0.5 + rand(shape, torch.float32, 9) / ratio
    near(ortho(g, dst), O.orthogonalise(g.double().cpu().numpy(), 5, C, EPS), tolerance(dst, ratio=ratio))


@pytest.mark.parametrize("shape", [(1500, 2100), (4096, 300)])
@pytest.mark.parametrize("dst", [torch.float32, torch.bfloat16])
def test_larger_matrices(shape, dst):
    g = rand(shape, torch.float32, 10)
    near(ortho(g, dst), O.orthogonalise(g.double().cpu().numpy(), 5, C, EPS), tolerance(dst))


@pytest.mark.parametrize("scale", [2.0 ** -100, 2.0 ** 100])
@pytest.mark.parametrize("shape", [(40, 50), (200, 150)])
def test_any_magnitude(shape, scale):
    """Squares of these pass fp32's range; a power of two leaves nothing but the exponents changed (eps aside, here 0)."""
    g = rand(shape, torch.float32, 11)
    assert torch.equal(ortho(g * scale, torch.float32, eps=0.0), ortho(g, torch.float32, eps=0.0))


@pytest.mark.parametrize("shape", [(3, 40, 50), (3, 200, 150)])
@pytest.mark.parametrize("dst", [torch.float32, torch.bfloat16])
def test_zeros_and_non_finite_matrices_stay_by_themselves(shape, dst):
    g = rand(shape, torch.float32, 12)
    alone = ortho(g, dst)
    for bad in (float("nan"), float("inf"), -float("inf")):
        h = g.clone()
        h[1, 3, 5] = bad
        got = ortho(h, dst)
        assert torch.equal(got[0], alone[0]) and torch.equal(got[2], alone[2]) and torch.isnan(got[1]).all()
    g[1] = 0
    got = ortho(g, dst)
    assert torch.equal(got[0], alone[0]) and not got[1].any() and torch.equal(got[2], alone[2])


@pytest.mark.parametrize("shape", [(60, 90), (90, 60), (200, 330), (330, 200)])
@pytest.mark.parametrize("src,dst", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.int8, torch.float32)])
def test_strides(shape, src, dst):
    g = rand(shape, src, 13)
    want = ortho(g, dst)
    # columns cut out of wider buffers, at odd offsets; what lies around the result stays
    wide = rand((shape[0], shape[1] + 11), src, 14)
    wide[:, 5:5 + shape[1]] = g
    room = torch.full((shape[0] + 2, shape[1] + 9), 3.0, dtype=dst, device=DEV)
    to, ws = room[1:-1, 3:3 + shape[1]], workspace(shape)
    S.s3gd_orthogonalise(wide[:, 5:5 + shape[1]], to, ws)
    assert torch.equal(to, want)
    to.fill_(3.0)
    assert (room == 3.0).all()
    # columns contiguous in both: the transposed problem
    out = torch.empty((shape[1], shape[0]), dtype=dst, device=DEV).mT
    S.s3gd_orthogonalise(g.mT.contiguous().mT, out, ws)
    assert torch.equal(out, want)
    # a batch whose matrices lie interleaved, and one that is broadcast
    pair = torch.empty((shape[0], 2, shape[1]), dtype=src, device=DEV)
    pair[:, 0], pair[:, 1] = g, g
    got = torch.empty((shape[0], 2, shape[1]), dtype=dst, device=DEV)
    ws = workspace((2,) + shape)
    S.s3gd_orthogonalise(pair.transpose(0, 1), got.transpose(0, 1), ws)
    assert torch.equal(got[:, 0], want) and torch.equal(got[:, 1], want)
    S.s3gd_orthogonalise(g.unsqueeze(0).expand(2, -1, -1), got.transpose(0, 1), ws)
    assert torch.equal(got[:, 0], want) and torch.equal(got[:, 1], want)


@pytest.mark.parametrize("shape", [(64, 100), (300, 200)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_in_place_repeatable_and_on_another_stream(shape, dtype):
    g = rand(shape, dtype, 15)
    want, ws = ortho(g, dtype), workspace(shape)
    side = torch.cuda.Stream()
    h = g.clone()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        S.s3gd_orthogonalise(h, h, ws)
    side.synchronize()
    assert torch.equal(h, want)
    graph = torch.cuda.CUDAGraph()
    h = torch.empty_like(g)
    with torch.cuda.graph(graph):
        S.s3gd_orthogonalise(g, h, ws)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(h, want)


def f32_bits(a):
    return a.cpu().numpy().view(np.uint32)


@pytest.mark.parametrize("shape", [(40, 64), (64, 40), (150, 220), (260, 130), (3, 50, 70), (2, 170, 140)])
@pytest.mark.parametrize("g_dtype", [torch.float32, torch.bfloat16, torch.int8])
@pytest.mark.parametrize("x_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("mode", ["plain", "momentum", "nesterov"])
def test_step(shape, g_dtype, x_dtype, mode):
    x, g = rand(shape, x_dtype, 16, 0.02), rand(shape, g_dtype, 17, 1e-3)
    v = None if mode == "plain" else rand(shape, torch.float32, 18, 1e-3 if g_dtype != torch.int8 else 1.0)
    mu, lr, wd, scale = 0.9, 0.01, 0.1, 0.2 * max(shape[-2:]) ** 0.5
    x1, ws = x.clone(), workspace(shape)
    v1 = None if v is None else v.clone()
    S.s3gd_step_ortho(x1, g, lr, ws, v=v1, mu=mu, nesterov=mode == "nesterov", weight_decay=wd, scale=scale)
    S.s3gd_device_status(ws)
    # the momentum is two fp32 operations, bit for bit
    if v is not None:
        want_v = np.float32(mu) * v.cpu().numpy() + g.float().cpu().numpy()
        assert np.array_equal(f32_bits(v1), want_v.view(np.uint32))
    want, _ = O.step(x.double().cpu().numpy(), None if v is None else v.double().cpu().numpy(), g.double().cpu().numpy(), mu,
                     mode == "nesterov", lr, wd, scale, 5, C, EPS)
    got, x0 = x1.double().cpu().numpy(), x.double().cpu().numpy()
    # x: a few fp32 roundings of its own size, plus its share of the orthogonalised matrix's error; bf16: one more of 2^-9
    moved = np.abs(want - (1 - lr * wd) * x0)
    for k in range(got.reshape((-1,) + shape[-2:]).shape[0]):
        sel = (k,) if len(shape) == 3 else ()
        tol = 4 * 2.0 ** -24 * np.linalg.norm(x0[sel]) + tolerance(torch.float32 if x_dtype == torch.float32 else torch.bfloat16) * np.linalg.norm(moved[sel])
        tol += 2.0 ** -9 * np.linalg.norm(want[sel]) if x_dtype == torch.bfloat16 else 0.0
        assert np.linalg.norm(got[sel] - want[sel]) <= tol


def test_step_takes_the_vote_of_the_workers():
    M, rows, cols = 5, 96, 160
    d = rows * cols
    grads = rand((M, d), torch.float32, 19)
    vote, x = torch.empty(d, dtype=torch.int8, device=DEV), torch.zeros(d, device=DEV)
    ws = S.alloc_workspace(M, d, d // 10, DEV)
    S.s3gd_step(x, grads, d // 10, 0.1, ws, opt_vote=vote)
    w, v = rand((rows, cols), torch.float32, 20), torch.zeros((rows, cols), device=DEV)
    w1, ws = w.clone(), workspace((rows, cols))
    S.s3gd_step_ortho(w1, vote.view(rows, cols), 0.1, ws, v=v, mu=0.9, nesterov=False)
    assert torch.equal(v, vote.view(rows, cols).float())
    want, _ = O.step(w.double().cpu().numpy(), None, vote.view(rows, cols).double().cpu().numpy(), 0.9, False, 0.1, 0.0, 1.0, 5, C, EPS)
    assert np.abs(w1.double().cpu().numpy() - want).max() <= 1e-5


def test_binding_refusals():
    g, out, ws = rand((8, 12), torch.float32, 1), torch.empty((8, 12), device=DEV), workspace((8, 12))
    with pytest.raises(ValueError):
        S.s3gd_orthogonalise(g, out[:4], ws)                       # another shape
    with pytest.raises(ValueError):
        S.s3gd_orthogonalise(g, torch.empty((12, 8), device=DEV).mT, ws)   # rows here, columns there
    with pytest.raises(ValueError):
        S.s3gd_orthogonalise(g[0], out[0], ws)
    with pytest.raises(TypeError):
        S.s3gd_orthogonalise(g.double(), out, ws)
    with pytest.raises(TypeError):
        S.s3gd_orthogonalise(g, out.to(torch.int8), ws)
    with pytest.raises(TypeError):
        S.s3gd_step_ortho(g, g, 0.1, ws, v=torch.zeros((8, 12), dtype=torch.bfloat16, device=DEV))
    with pytest.raises(S.S3gdError) as e:
        S.s3gd_orthogonalise(g, out, ws[:256])
    assert e.value.code == 2
    with pytest.raises(S.S3gdError) as e:
        S.s3gd_orthogonalise(g, out, ws, steps=0)
    assert e.value.code == 1


# ------------------------------------------------------------------ many tiles: pairs of CTAs on 256 x 256 tiles
def exact_on_gpu(g, steps=5):
    """The statement in fp64 on the GPU, for sizes that take numpy minutes."""
    y = g.double()
    y = y / (torch.linalg.vector_norm(y, dim=(-2, -1), keepdim=True) + EPS)
    tall = y.shape[-2] > y.shape[-1]
    a, b, c = C
    for _ in range(steps):
        p = y.mT @ y if tall else y @ y.mT
        q = b * p + c * (p @ p)
        y = a * y + (y @ q if tall else q @ y)
    return y


WIDE = [(2500, 2600), (2601, 2307), (12, 1030, 1025), (5, 1400, 2000), (3, 1300, 1290), (1, 2048, 2560), (20, 520, 700)]


@pytest.mark.parametrize("shape", WIDE)
@pytest.mark.parametrize("src,dst", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.int8, torch.float32)])
def test_many_tiles(shape, src, dst):
    g = rand(shape, src, 21)
    near(ortho(g, dst), exact_on_gpu(g).cpu().numpy(), tolerance(dst))


@pytest.mark.parametrize("shape", [(2500, 2600), (2601, 2307), (5, 1400, 1500)])
@pytest.mark.parametrize("x_dtype", [torch.float32, torch.bfloat16])
def test_many_tiles_step(shape, x_dtype):
    x, g, v = rand(shape, x_dtype, 22, 0.02), rand(shape, torch.bfloat16, 23, 1e-3), rand(shape, torch.float32, 24, 1e-3)
    mu, lr, wd, scale = 0.9, 0.01, 0.1, 0.2 * max(shape[-2:]) ** 0.5
    # rows of x that are not a multiple of four entries apart, so that no wide access fits
    room = torch.zeros(shape[:-1] + (shape[-1] + 3,), dtype=x_dtype, device=DEV)
    for x1 in (x.clone(), room[..., 1:1 + shape[-1]]):
        x1.copy_(x)
        v1, ws = v.clone(), workspace(shape)
        S.s3gd_step_ortho(x1, g, lr, ws, v=v1, mu=mu, nesterov=True, weight_decay=wd, scale=scale)
        S.s3gd_device_status(ws)
        want_v = (torch.tensor(mu, device=DEV) * v) + g.float()
        assert torch.equal(v1, want_v)
        moved = lr * scale * exact_on_gpu(g.double() + float(np.float32(mu)) * want_v.double())
        want = (1 - lr * wd) * x.double() - moved
        tol = 4 * 2.0 ** -24 * x.double().norm() + tolerance(x_dtype) * moved.norm()
        tol += 2.0 ** -9 * want.norm() if x_dtype == torch.bfloat16 else 0.0
        assert (x1.double() - want).norm() <= tol
    room[..., 1:1 + shape[-1]] = 0
    assert not room.any()


def test_many_tiles_keep_matrices_apart():
    shape, dst = (5, 1400, 1500), torch.bfloat16
    g = rand(shape, torch.float32, 25)
    alone = ortho(g, dst)
    assert torch.equal(alone, ortho(g, dst))
    h = g.clone()
    h[1, 3, 5], h[3] = float("inf"), 0.0
    got = ortho(h, dst)
    for k in (0, 2, 4):
        assert torch.equal(got[k], alone[k])
    assert torch.isnan(got[1]).all() and not got[3].any()
