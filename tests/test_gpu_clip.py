"""s3gd_grad_norm and s3gd_clip on the GPU against the 64-bit statement.

Tolerances, in u = 2^-24.  Squares of at most eight neighbours may be added in 32 bits (8 u of their sum), all else in 64: the norm
is within 4 u, and a rounding: 6 u.  The factor adds a division and a rounding, the product another: 8 u, and half a step of the
result's type where that is bf16 (2^-8).
"""
import numpy as np
import pytest
import torch

import paper_2302_07475_b200 as S
from oracle import operators_oracle as O

pytestmark = pytest.mark.gpu
DEV, U = "cuda", 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16


def rand(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator(DEV).manual_seed(seed), device=DEV) * scale).to(dtype)


def host(t):
    return t.double().cpu().numpy()


def workspace(M):
    ws = S.alloc_clip_workspace(M, DEV)
    ws.fill_(255)
    return ws


def check(outs, norm, grads, max_norm, eps=1e-6):
    want, want_norm = O.clip([host(g) for g in grads], max_norm, eps)
    assert (np.abs(host(norm) - want_norm) <= 6 * U * want_norm).all()
    for o, w in zip(outs or (), want):
        off = (8 * U + (2.0 ** -8 * (1 + 8 * U) if o.dtype == BF16 else 0)) * np.abs(w) + 2.0 ** -133
        assert o.shape == w.shape and (np.abs(host(o) - w) <= off).all()


LISTS = [[(1,)], [(3,), (1,), (7, 5)], [(8191,), (8192,), (8193,)], [(1000, 33), (33,), (64, 3, 3, 3), (16,)], [(100003,)], [(2,)] * 70, [(5, 4)] * 700 + [(30000,)]]


@pytest.mark.parametrize("shapes", LISTS, ids=lambda s: f"{len(s)}x{s[0]}")
@pytest.mark.parametrize("M", [1, 3, 40])
@pytest.mark.parametrize("src,dst", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
def test_norm_and_clip_into_rows(shapes, M, src, dst):
    grads = [rand((M,) + s, src, i, 0.1 * (1 + i % 3)) for i, s in enumerate(shapes)]
    norm, ws = torch.full((M,), float("nan"), device=DEV), workspace(M)
    S.s3gd_grad_norm(grads, norm, ws)
    S.s3gd_device_status(ws)
    check(None, norm, grads, 1.0)
    sizes = [int(np.prod(s)) for s in shapes]
    d = sum(sizes)
    rows = torch.full((M, d + 3), 7.0, dtype=dst, device=DEV)              # rows that lie in all ways to their tensors
    outs = [p.unflatten(1, s) for p, s in zip(rows[:, 2:d + 2].split(sizes, 1), shapes)]
    for max_norm in (float(norm.median()), 1e9, 0.0):                      # some, none, all to nothing
        norm.fill_(float("nan"))
        S.s3gd_clip(grads, max_norm, norm, ws, out=outs)
        S.s3gd_device_status(ws)
        check(outs, norm, grads, max_norm)
        assert (rows[:, :2] == 7).all() and (rows[:, d + 2:] == 7).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_in_place_and_one_norm_for_everything(dtype):
    grads = [rand(s, dtype, i) for i, s in enumerate(((400, 31), (77,), (5, 6, 7), (), (90001,)))]
    norm, ws = torch.empty((), device=DEV), workspace(1)
    kept = [g.clone() for g in grads]
    S.s3gd_clip(grads, 1e6, norm, ws)
    assert all(torch.equal(a, b) for a, b in zip(grads, kept))            # below the limit: untouched
    S.s3gd_clip(grads, 0.5, norm, ws)
    check([g[None] for g in grads], norm[None], [g[None] for g in kept], 0.5)
    single = rand((3, 1000), dtype, 9)
    S.s3gd_grad_norm(single, norm, ws)
    check(None, norm[None], [single[None]], 1.0)
    part = rand((4, 3000), dtype, 10)
    rows, before = part[:, 5:2900], part.clone()                          # columns of a buffer, per worker
    each = torch.empty((4,), device=DEV)
    ws = workspace(4)
    S.s3gd_clip(rows, 20.0, each, ws)
    check([rows], each, [before[:, 5:2900]], 20.0)
    assert torch.equal(part[:, :5], before[:, :5]) and torch.equal(part[:, 2900:], before[:, 2900:])


def test_other_orders_of_axes_and_refusals_of_gaps():
    norm, ws = torch.empty((), device=DEV), workspace(1)
    g = rand((40, 60), F32, 1).t()
    o = torch.empty((40, 60), dtype=BF16, device=DEV).t()
    S.s3gd_clip([g], 2.0, norm, ws, out=[o])
    check([o[None]], norm[None], [g[None]], 2.0)
    h = rand((2, 8, 5, 3), F32, 2).permute(0, 3, 1, 2)                    # channels last
    S.s3gd_grad_norm([h, g], norm, ws)
    assert abs(float(norm) - float(torch.sqrt(h.double().square().sum() + g.double().square().sum()))) <= 6 * U * float(norm)
    with pytest.raises(ValueError):
        S.s3gd_clip([g], 2.0, norm, ws, out=[torch.empty((60, 40), device=DEV)])   # another order
    with pytest.raises(ValueError):
        S.s3gd_grad_norm([rand((10, 10), F32, 3)[:, ::2]], norm, ws)
    with pytest.raises(ValueError):
        S.s3gd_grad_norm([rand((10, 1), F32, 3).expand(10, 10)], norm, ws)


def test_empty_tensors_and_lists():
    norm, ws = torch.full((2,), 9.0, device=DEV), workspace(2)
    S.s3gd_grad_norm([], norm, ws)
    assert not norm.any()
    g = rand((2, 5), F32, 1)
    S.s3gd_clip([torch.empty((2, 0), device=DEV), g, torch.empty((2, 3, 0), dtype=BF16, device=DEV)], 1e-3, norm, ws)
    check([g], norm, [rand((2, 5), F32, 1)], 1e-3)
    zero = torch.zeros((2, 100), device=DEV)
    S.s3gd_clip([zero], 0.0, norm, ws, eps=0.0)
    assert not zero.any() and not norm.any()


@pytest.mark.parametrize("scale", [1e-42, 1e-30, 1e-20, 1e18, 1e19, 1e30, 3e38])
def test_ends_of_the_range(scale):
    g = (rand((2, 5000), torch.float64, 1).clamp(-1, 1) * scale).float()
    g[1, ::3] = 0
    norm, ws = torch.empty((2,), device=DEV), workspace(2)
    S.s3gd_grad_norm([g], norm, ws)
    want = np.sqrt((host(g) ** 2).sum(1))
    fits = want < 3.4e38
    assert (np.abs(host(norm) - want)[fits] <= 6 * U * want[fits] + 2.0 ** -149).all() and np.isinf(host(norm)[~fits]).all()
    out = torch.empty_like(g)
    S.s3gd_clip([g], float(np.float32(min(scale, 1e30) * 0.25)), norm, ws, out=[out], eps=0.0)
    c = np.float32(min(scale, 1e30) * 0.25) / want
    assert (np.abs(host(out) - host(g) * c[:, None]) <= 8 * U * np.abs(host(g)) * c[:, None] + 2.0 ** -149).all()


def test_what_is_not_finite_stays_with_its_worker():
    g = rand((4, 20000), F32, 1)
    g[1, 777], g[2, 15000] = float("nan"), float("-inf")
    norm, ws, out = torch.empty((4,), device=DEV), workspace(4), torch.empty((4, 20000), device=DEV)
    S.s3gd_clip([g], 1.0, norm, ws, out=[out])
    assert norm[1].isnan() and norm[2].isinf() and norm[0].isfinite() and norm[3].isfinite()
    assert out[1].isnan().all() and out[2, 15000].isnan() and not out[2, :15000].any() and not out[2, 15001:].any()
    check([out[::3]], norm[::3], [g[::3]], 1.0)


@pytest.mark.parametrize("tiles", [1, 8, 9, 16, 17, 40])
@pytest.mark.parametrize("M", [1, 8, 9])
def test_few_and_many_tiles(tiles, M):
    n = 8192 * tiles - 8                                                  # tiles of 8192 entries, wherever the first one lies
    g, out = rand((M, n + 3), F32, 1)[:, 1:n + 1], torch.full((M, n + 7), 5.0, dtype=BF16, device=DEV)
    norm, ws = torch.empty((M,), device=DEV), workspace(M)
    S.s3gd_clip([g], 3.0, norm, ws, out=[out[:, 4:n + 4]])
    S.s3gd_device_status(ws)
    check([out[:, 4:n + 4]], norm, [g], 3.0)
    assert (out[:, :4] == 5).all() and (out[:, n + 4:] == 5).all()
    norm.zero_()
    S.s3gd_grad_norm(g, norm, ws)
    check(None, norm, [g], 3.0)


def test_types_mixed_in_one_list():
    shapes, kinds = [(3000,), (40, 5), (9000,), (7,), (123,), (20000,)], [(F32, F32), (BF16, F32), (F32, BF16), (BF16, BF16), (BF16, F32), (F32, F32)]
    grads = [rand((4,) + s, src, i) for i, (s, (src, _)) in enumerate(zip(shapes, kinds))]
    outs = [torch.empty((4,) + s, dtype=dst, device=DEV) for s, (_, dst) in zip(shapes, kinds)]
    norm, ws = torch.empty((4,), device=DEV), workspace(4)
    S.s3gd_clip(grads, 2.0, norm, ws, out=outs)
    check(outs, norm, grads, 2.0)
    kept = [g.clone() for g in grads]
    S.s3gd_clip(grads, 2.0, norm, ws, out=[g if i % 2 else o for i, (g, o) in enumerate(zip(grads, outs))])   # every other one in place
    check([g if i % 2 else o for i, (g, o) in enumerate(zip(grads, outs))], norm, kept, 2.0)
    assert all(torch.equal(a, b) for a, b in zip(grads[::2], kept[::2]))


def test_values_equal_for_any_place_in_memory():
    base = rand((70000,), F32, 1)
    norms, ws = [], workspace(1)
    for shift in range(5):
        room = torch.zeros((70010,), device=DEV)
        room[shift:shift + 70000] = base
        norm = torch.empty((), device=DEV)
        S.s3gd_clip([room[shift:shift + 70000]], 1.0, norm, ws)
        check([room[None, shift:shift + 70000]], norm[None], [base[None]], 1.0)
        assert not room[:shift].any() and not room[shift + 70000:].any()
        norms.append(float(norm))
    assert max(norms) - min(norms) <= 12 * U * norms[0]


def test_large_rows_streams_and_graphs():
    M, d = 6, 3_000_001                                                   # rows that lie in all ways
    g, out = rand((M, d), F32, 1), torch.empty((M, d), device=DEV)
    norm, ws = torch.empty((M,), device=DEV), workspace(M)
    S.s3gd_clip([g], 100.0, norm, ws, out=[out])
    want = g.double().square().sum(1).sqrt()
    assert ((norm.double() - want).abs() <= 6 * U * want).all()
    exact = g.double() * (100.0 / (want + 1e-6))[:, None]
    assert ((out.double() - exact).abs() <= 8 * U * exact.abs()).all()
    again, n2 = torch.zeros_like(out), torch.zeros_like(norm)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        S.s3gd_clip([g], 100.0, n2, ws, out=[again])
    side.synchronize()
    assert torch.equal(again, out) and torch.equal(n2, norm)
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for k, graph in enumerate(graphs):                                    # two graphs that share the workspace; the lists are gone by the replay
        with torch.cuda.graph(graph):
            S.s3gd_clip([g[:, :1000], g[:, 1000:]], 100.0 * (k + 1), n2, ws, out=[again[:, :1000], again[:, 1000:]])
    for k in (0, 1, 0):
        again.zero_()
        graphs[k].replay()
        torch.cuda.synchronize()
        exact = g.double() * (100.0 * (k + 1) / (want + 1e-6))[:, None]
        assert ((again.double() - exact).abs() <= 8 * U * exact.abs()).all()


@pytest.mark.skipif(torch.cuda.is_available() and torch.cuda.get_device_properties(0).total_memory < 60e9, reason="needs 40 GB of device memory")
def test_offsets_past_32_bits():
    n = (1 << 32) + 1000
    g = torch.zeros((n,), dtype=BF16, device=DEV)
    g[-3:] = 3.0
    g[5] = 4.0
    norm, ws = torch.empty((), device=DEV), workspace(1)
    S.s3gd_clip([g], 1.0, norm, ws)
    assert abs(float(norm) - 43 ** 0.5) <= 6 * U * 43 ** 0.5
    assert float(g[5]) == float(torch.tensor(4 / (43 ** 0.5 + 1e-6)).to(BF16)) and float(g[-1]) == float(torch.tensor(3 / (43 ** 0.5 + 1e-6)).to(BF16))
    assert int((g != 0).sum()) == 4
