"""s3gd_layer_norm and s3gd_layer_norm_grad on the GPU against the 64-bit statement.

Tolerances, in u = 2^-24.  A row's sums are taken over at most 16 entries in turn, 5 rounds of lanes and 16 warps: with the
division no more than 40 u of the sum of magnitudes.  The centred entry is off by 3 u of itself and by 40 u of the mean
magnitude (at most sigma), rstd by (40 / 2 + 3) u, which gives xhat an error of (28 |xhat| + 40) u; y adds the product's and the
sum's roundings.  Put through the gradient's formula, with mg = mean |g| and mgx = mean |g xhat|:
    rstd u (28 |g| + 68 mg + 40 |xhat| mg + (124 |xhat| + 40) mgx).
A sum of T terms in any grouping is within T u of the sum of magnitudes.  16-bit results add half a step, 2^-8 of the value.
"""
import numpy as np
import pytest
import torch

import paper_2302_07475_b200 as S
from oracle import operators_oracle as O

pytestmark = pytest.mark.gpu
DEV, U, EPS = "cuda", 2.0 ** -24, 1e-5
F32, BF16 = torch.float32, torch.bfloat16


def rand(shape, dtype, seed, scale=1.0, offset=0.0):
    return (torch.randn(shape, generator=torch.Generator(DEV).manual_seed(seed), device=DEV) * scale + offset).to(dtype)


def places(shape, masked, seed, dtype=torch.int64):
    g = torch.Generator(DEV).manual_seed(seed)
    ids = torch.randint(0, 1000, shape, generator=g, device=DEV)
    return torch.where(torch.rand(shape, generator=g, device=DEV) < masked, -ids - 1, ids).to(dtype)


def host(t):
    return None if t is None else t.double().cpu().numpy()


def half(t):
    return 2.0 ** -8 if t.dtype == BF16 else U


def check_y(y, x, weight, bias, ids=None, eps=EPS):
    want, xhat = O.layer_norm(host(x), host(weight), host(bias), eps, None if ids is None else ids.cpu().numpy())
    w = 1.0 if weight is None else np.abs(host(weight))
    off = U * (w * (29 * np.abs(xhat) + 40) + np.abs(want)) * (1 + 2.0 ** -8)
    have = host(y)
    over = np.abs(have - want) - off - half(y) * np.abs(want)
    there = np.ones(have.shape[:-1], dtype=bool) if ids is None else ids.cpu().numpy() >= 0
    assert np.isfinite(have).all() and not have[~there].any()
    assert not there.any() or over[there].max() <= 1e-30, f"worst {over[there].max():.3g}"


def run_grad(dy, x, weight, ids=None, dtotal=None, dst=F32, before=None, eps=EPS, dx=None):
    M, T, dim = x.shape
    dx = torch.full_like(x, float("nan")) if dx is None else dx
    grads = torch.full((M, 2 * dim + 3), float("nan"), dtype=dst, device=DEV) if before is None else before.clone()
    ws = S.alloc_layer_norm_workspace(M, T, dim, DEV)
    ws.fill_(255)
    S.s3gd_layer_norm_grad(dy, x, dx, weight, grads[:, 1:dim + 1], grads[:, dim + 2:2 * dim + 2], ws, eps=eps, ids=ids, dtotal=dtotal,
                           accumulate=before is not None)
    S.s3gd_device_status(ws)
    kept = torch.full_like(grads, float("nan")) if before is None else before
    for at in (0, dim + 1, 2 * dim + 2):
        assert torch.equal(grads[:, at].isnan(), kept[:, at].isnan())
    return dx, grads[:, 1:dim + 1], grads[:, dim + 2:2 * dim + 2]


def check_grad(got, dy, x, weight, ids=None, dtotal=None, before=None, eps=EPS):
    dx, dw, db = got
    there = None if ids is None else ids.cpu().numpy()
    want_x, want_w, want_b, (size, size_h, size_w, size_b) = O.layer_norm_grad(host(dy), host(x), host(weight), eps, there, host(dtotal))
    T, dim = x.shape[1:]
    if dx is not None:
        off = U * (size + 2 * np.abs(want_x)) * (1 + 2.0 ** -8) + half(dx) * np.abs(want_x)
        assert np.isfinite(host(dx)).all() and (np.abs(host(dx) - want_x) <= off + 1e-37).all(), f"{(np.abs(host(dx) - want_x) - off).max():.3g}"
        if ids is not None:
            assert not host(dx)[there < 0].any()
    for have, want, off, at in ((dw, want_w, U * (size_h + (T + 3) * size_w), slice(1, dim + 1)), (db, want_b, U * (T + 3) * size_b, slice(dim + 2, 2 * dim + 2))):
        if have is None:
            continue
        if before is not None:
            want = want + host(before[:, at])
        off = (off + U * np.abs(want)) * (1 + 2.0 ** -8) + (half(have) * np.abs(want) if have.dtype == BF16 else 0)
        assert np.isfinite(host(have)).all() and (np.abs(host(have) - want) <= off + 1e-37).all(), f"{(np.abs(host(have) - want) - off).max():.3g}"


SHAPES = [(1, 1, 1), (1, 1, 7), (1, 3, 1024), (3, 2, 33), (2, 5, 128), (1, 700, 64), (4, 37, 512), (2, 9, 513), (1, 33, 768), (5, 3, 1001), (1, 17, 2048),
          (2, 4, 2047), (1, 5, 4096), (3, 2, 4100), (1, 3, 8192), (1, 2, 8191), (1, 2, 8196), (1, 2, 20001), (1, 2, 40000), (200, 1, 16), (1, 5000, 12)]


@pytest.mark.parametrize("M,T,dim", SHAPES)
@pytest.mark.parametrize("src,dst", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
def test_forward(M, T, dim, src, dst):
    x, param = rand((M, T, dim), src, 1, 2.0, 0.3), BF16 if dim % 3 == 0 else F32
    w, b = rand((dim,), param, 2, 0.3, 1.0), rand((dim,), param, 3)
    ids = places((M, T), 0.3, 4, torch.int32 if dim % 2 else torch.int64) if T > 1 else None
    y = torch.full((M, T, dim), float("nan"), dtype=dst, device=DEV)
    S.s3gd_layer_norm(x, y, w, b, ids=ids)
    check_y(y, x, w, b, ids)
    add, total = rand((M, T, dim), src, 5), torch.full_like(x, float("nan"))
    y.fill_(float("nan"))
    S.s3gd_layer_norm(x, y, w, None, ids=ids, add=add, total=total)
    summed = (x.float() + add.float()).to(src)
    if ids is not None:
        summed = torch.where((ids >= 0)[..., None], summed, torch.zeros_like(summed))
    assert torch.equal(total, summed)
    check_y(y, summed, w, None, ids)


@pytest.mark.parametrize("M,T,dim", SHAPES)
@pytest.mark.parametrize("src,dst,grad", [(F32, F32, F32), (F32, BF16, BF16), (BF16, F32, F32), (BF16, BF16, F32)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient(M, T, dim, src, dst, grad, accumulate):
    x, dy, w = rand((M, T, dim), src, 6, 2.0, 0.3), rand((M, T, dim), dst, 7), rand((dim,), BF16 if dim % 3 == 0 else F32, 8, 0.3, 1.0)
    ids = places((M, T), 0.3, 9, torch.int32 if dim % 2 else torch.int64) if T > 1 else None
    dtotal = rand((M, T, dim), src, 10) if accumulate else None
    before = rand((M, 2 * dim + 3), grad, 11) if accumulate else None
    check_grad(run_grad(dy, x, w, ids, dtotal, grad, before), dy, x, w, ids, dtotal, before)


def test_many_rows_and_workers():
    for M, T, dim in ((1, 30000, 40), (3, 7001, 96), (300, 40, 64), (7, 1500, 260)):
        x, dy, w = rand((M, T, dim), F32, 12), rand((M, T, dim), F32, 13), rand((dim,), F32, 14, 0.3, 1.0)
        ids = places((M, T), 0.1, 15)
        got = run_grad(dy, x, w, ids)
        check_grad(got, dy, x, w, ids)
        again = run_grad(dy, x, w, ids)
        assert all(torch.equal(a, b) for a, b in zip(got, again))          # no result depends on the run


@pytest.mark.parametrize("M,T,dim", [(200, 100, 40), (100, 333, 96), (160, 37, 512), (9, 20, 768), (8, 64, 768), (8, 65, 768), (2, 1025, 33), (37, 150, 264),
                                     (400, 3, 1030), (1, 9, 4096), (5, 900, 1024)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_dealt_in_all_ways(M, T, dim, dtype):
    x, dy, w = rand((M, T, dim), dtype, 62, 1.5), rand((M, T, dim), dtype, 63), rand((dim,), F32, 64, 0.3, 1.0)
    ids, before = places((M, T), 0.1, 65), rand((M, 2 * dim + 3), F32, 66)
    got = run_grad(dy, x, w, ids, before=before)
    check_grad(got, dy, x, w, ids, before=before)
    assert all(torch.equal(a, b) for a, b in zip(got, run_grad(dy, x, w, ids, before=before)))


@pytest.mark.parametrize("dim", [64, 100, 1001, 2048, 9000])
def test_rows_far_from_zero(dim):
    x = rand((1, 6, dim), F32, 16, 1.0, 1e4)
    y, w = torch.empty_like(x), rand((dim,), F32, 17)
    S.s3gd_layer_norm(x, y, w, None)
    check_y(y, x, w, None)
    dy = rand((1, 6, dim), F32, 18)
    check_grad(run_grad(dy, x, w), dy, x, w)


def test_constant_rows_and_outliers():
    x = rand((1, 5, 300), F32, 19)
    x[0, 0] = 3.7
    x[0, 1] = 0.0
    x[0, 2, 0] = 1e6
    x[0, 3, 299] = -1e5
    y, w, b = torch.empty_like(x), rand((300,), F32, 20), rand((300,), F32, 21)
    S.s3gd_layer_norm(x, y, w, b)
    check_y(y, x, w, b)
    assert torch.equal(y[0, 0], b) and torch.equal(y[0, 1], b)
    dy = rand((1, 5, 300), F32, 22)
    check_grad(run_grad(dy, x, w), dy, x, w)


@pytest.mark.parametrize("dim", [24, 1000, 1001, 9000])
def test_what_is_not_finite_stays_in_its_row(dim):
    x, dy = rand((2, 5, dim), F32, 23), rand((2, 5, dim), F32, 24)
    ids = torch.zeros((2, 5), dtype=torch.int64, device=DEV)
    x[0, 1, 3], x[0, 2, 4], dy[0, 3, 5] = float("nan"), float("inf"), float("nan")
    y, clean = torch.empty_like(x), torch.ones((2, 5), dtype=torch.bool, device=DEV)
    clean[0, 1:4] = False
    S.s3gd_layer_norm(x, y)
    assert y[0, 1].isnan().all() and y[0, 2].isnan().any() and y[0, 3].isfinite().all() and y[clean].isfinite().all()
    dx, dw, db = run_grad(dy, x, None)
    assert dx[clean].isfinite().all() and dx[0, 1].isnan().all() and dw[1].isfinite().all() and db[1].isfinite().all() and dw[0].isnan().any()
    ids[0, 1:4] = -1                                     # the same rows as empty places: nothing of them is seen
    S.s3gd_layer_norm(x, y, ids=ids)
    assert y.isfinite().all() and not y[0, 1:4].any()
    got = run_grad(dy, x, None, ids, dtotal=torch.where((ids >= 0)[..., None], 0.0, float("nan")).expand(2, 5, dim).contiguous())
    assert all(t.isfinite().all() for t in got)
    check_grad(got, dy, torch.where((ids >= 0)[..., None], x, torch.zeros_like(x)), None, ids)


def test_all_places_empty_and_no_rows():
    x, ids = torch.full((2, 3, 40), float("nan"), device=DEV), torch.full((2, 3), -7, device=DEV)
    dx, dw, db = run_grad(x, x, None, ids)
    assert not dx.any() and not dw.any() and not db.any()
    none = torch.empty((2, 0, 40), device=DEV)
    dx, dw, db = run_grad(none, none, None)
    assert not dw.any() and not db.any()
    before = rand((2, 83), F32, 25)
    _, dw, db = run_grad(none, none, None, before=before)
    assert torch.equal(dw, before[:, 1:41]) and torch.equal(db, before[:, 42:82])
    S.s3gd_layer_norm(none, none.clone())
    S.s3gd_layer_norm(torch.empty((0, 40), device=DEV), torch.empty((0, 40), device=DEV))


@pytest.mark.parametrize("dim", [40, 41, 1024, 8200])
def test_strides_and_repeated_rows(dim):
    M, T = 3, 5
    big = rand((T, M, dim + 9), F32, 26)
    x = big[:, :, 2:dim + 2].transpose(0, 1)             # tokens first, workers inside; rows that begin anywhere
    dy = rand((1, 1, dim), F32, 27).expand(M, T, dim)    # one row for all
    room = torch.full((M, T + 1, dim + 5), 5.0, device=DEV)
    y = room[:, :T, 3:dim + 3]
    w = rand((dim + 1,), F32, 28)[1:]
    S.s3gd_layer_norm(x, y, w)
    check_y(y, x, w, None)
    assert (room[:, :, :3] == 5).all() and (room[:, :, dim + 3:] == 5).all() and (room[:, T] == 5).all()
    inner = torch.full((T, M, dim + 4), 5.0, device=DEV)
    got = run_grad(dy, x, w, dx=inner[:, :, 4:].transpose(0, 1))
    check_grad(got, dy, x, w)
    assert (inner[:, :, :4] == 5).all()
    flat, out = x[0], torch.empty((T, dim), dtype=BF16, device=DEV)   # one worker: [T, dim], gradients [dim]
    S.s3gd_layer_norm(flat, out, w)
    check_y(out, flat, w, None)
    four = rand((2, 2, 3, dim), F32, 29)
    out = torch.empty_like(four)
    S.s3gd_layer_norm(four, out, w)
    check_y(out, four, w, None)


@pytest.mark.parametrize("dim", [40, 1001, 2048, 8200])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_in_place(dim, dtype):
    x, add, dy, w = rand((2, 9, dim), dtype, 30), rand((2, 9, dim), dtype, 31), rand((2, 9, dim), dtype, 32), rand((dim,), F32, 33)
    y, total = torch.empty_like(x), torch.empty_like(x)
    S.s3gd_layer_norm(x, y, w, add=add, total=total)
    for target in ("x", "add"):
        a, b, o = x.clone(), add.clone(), torch.empty_like(x)
        S.s3gd_layer_norm(a, o, w, add=b, total=a if target == "x" else b)
        assert torch.equal(o, y) and torch.equal(a if target == "x" else b, total)
    a, o = x.clone(), torch.empty_like(x)
    S.s3gd_layer_norm(x, o, w)
    S.s3gd_layer_norm(a, a, w)
    assert torch.equal(a, o)
    dx, dw, db = run_grad(dy, x, w, dtotal=add)
    for target in ("dy", "x", "dtotal"):
        t = {"dy": dy.clone(), "x": x.clone(), "dtotal": add.clone()}
        got = run_grad(t["dy"], t["x"], w, dtotal=t["dtotal"], dx=t[target])
        assert torch.equal(got[0], dx) and torch.equal(got[1], dw) and torch.equal(got[2], db)


@pytest.mark.parametrize("dim", [96, 333, 8200])
def test_parts_of_the_gradient(dim):
    x, dy, w = rand((2, 30, dim), F32, 34), rand((2, 30, dim), F32, 35), rand((dim,), F32, 36)
    dx, dw, db = run_grad(dy, x, w)
    ws = S.alloc_layer_norm_workspace(2, 30, dim, DEV)
    only = torch.empty_like(x)
    S.s3gd_layer_norm_grad(dy, x, only, w, None, None, ws)
    assert torch.equal(only, dx)
    a, b = torch.empty((2, dim), device=DEV), torch.empty((2, dim), device=DEV)
    S.s3gd_layer_norm_grad(dy, x, None, w, a, None, ws)
    S.s3gd_layer_norm_grad(dy, x, None, w, None, b, ws)
    assert torch.equal(a, dw) and torch.equal(b, db)
    one = torch.empty((dim,), device=DEV)                # one worker
    S.s3gd_layer_norm_grad(dy[0], x[0], only[0], w, one, None, ws)
    check_grad((only[:1], one[None], None), dy[:1], x[:1], w)
    S.s3gd_device_status(ws)


@pytest.mark.parametrize("dim", [12, 130, 1024])
def test_gradient_against_autograd_and_differences(dim):
    x, dy, w, b = (rand(s, F32, 40 + i).double() for i, s in enumerate(((1, 4, dim), (1, 4, dim), (dim,), (dim,))))
    leaves = [t.clone().requires_grad_() for t in (x, w, b)]
    d = leaves[0] - leaves[0].mean(-1, keepdim=True)
    (dy * (d / torch.sqrt((d * d).mean(-1, keepdim=True) + EPS) * leaves[1] + leaves[2])).sum().backward()
    dx, dw, db = run_grad(dy.float(), x.float(), w.float())
    for have, leaf in ((dx, leaves[0]), (dw[0], leaves[1]), (db[0], leaves[2])):
        assert (have.double() - leaf.grad).norm() <= 1e-5 * leaf.grad.norm()

    def loss(t):
        return float((host(dy) * O.layer_norm(t, host(w), host(b), EPS)[0]).sum())

    for at in ((0, 0, 0), (0, 3, dim - 1), (0, 1, dim // 2)):
        up, down, h = host(x), host(x), 1e-4
        up[at] += h
        down[at] -= h
        assert abs((loss(up) - loss(down)) / (2 * h) - float(dx[at])) <= 1e-5 * float(dx.abs().max())   # h^2 and 1e-16 / h beside 40 u


def test_streams_graphs_and_workspaces():
    x, dy, w = rand((2, 200, 512), F32, 50), rand((2, 200, 512), F32, 51), rand((512,), F32, 52)
    y, (dx, dw, db) = torch.empty_like(x), run_grad(dy, x, w)
    S.s3gd_layer_norm(x, y, w)
    large = S.alloc_layer_norm_workspace(5, 4000, 9000, DEV)           # serves smaller calls
    outs = [torch.zeros_like(x), torch.zeros_like(x), torch.zeros((2, 512), device=DEV), torch.zeros((2, 512), device=DEV)]

    def calls():
        S.s3gd_layer_norm(x, outs[0], w)
        S.s3gd_layer_norm_grad(dy, x, outs[1], w, outs[2], outs[3], large)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, (y, dx, dw, db)))
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for graph in graphs:                                               # two graphs that share the workspace
        with torch.cuda.graph(graph):
            calls()
    for o in outs:
        o.zero_()
    x.mul_(1.5)
    want_y, want = torch.empty_like(x), run_grad(dy, x, w)
    S.s3gd_layer_norm(x, want_y, w)
    for k in (0, 1, 0):
        graphs[k].replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, (want_y, *want)))


@pytest.mark.skipif(torch.cuda.is_available() and torch.cuda.get_device_properties(0).total_memory < 60e9, reason="needs 40 GB of device memory")
def test_offsets_past_32_bits():
    T, dim = 1 << 16, 64                                                # rows 40,000 entries apart: 2.6e9 entries
    room = torch.empty((T, 40000), dtype=BF16, device=DEV)
    x = room[:, 39000:39000 + dim]
    x.copy_(rand((T, dim), BF16, 60))
    y, w = torch.empty((T, dim), device=DEV), rand((dim,), F32, 61)
    S.s3gd_layer_norm(x, y, w)
    check_y(y[-50:], x[-50:], w, None)
    dx, dw, ws = room[:, 100:100 + dim], torch.empty((dim,), device=DEV), S.alloc_layer_norm_workspace(1, T, dim, DEV)
    S.s3gd_layer_norm_grad(y, x, dx, w, dw, None, ws)
    tail = run_grad(y[None, -50:].contiguous(), x[None, -50:].contiguous(), w)[0]
    assert torch.equal(dx[-50:], tail[0])
