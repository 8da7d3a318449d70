"""s3gd_clip and s3gd_grad_norm at the ends of their ranges.

Tolerances are those of test_gpu_clip.py; what is below fp32's normal range is off by the factor's and the product's rounding there, two
steps of 2^-149 at most.
"""
import numpy as np
import pytest
import torch

import paper_2302_07475_b200 as S
from test_gpu_clip import BF16, DEV, F32, U, host, rand, workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale,max_norm", [(1e30, 1.0), (1e36, 1e-2), (3e38, 1.0), (3e38, 1e-3), (3e38, 1e-30), (3e38, 1e-38), (3e38, 0.0), (1e20, 1e-20)])
@pytest.mark.parametrize("n", [5, 5000, 300001])                          # one launch, and two
@pytest.mark.parametrize("dst", [F32, BF16])
def test_factors_below_the_normal_range(scale, max_norm, n, dst):
    g = (rand((2, n), torch.float64, 1).clamp(-1, 1) * scale).float()
    g[1] *= 1e-3
    g[0, ::7] *= 1e-9                                                     # some whose product is below the normal range
    g[1, 2] = 0
    want = np.sqrt((host(g) ** 2).sum(1))
    c = float(np.float32(max_norm)) / want
    assert scale < 1e36 or (c < 2.0 ** -100).any()
    exact, norm, ws = host(g) * c[:, None], torch.empty((2,), device=DEV), workspace(2)
    off = (8 * U + (2.0 ** -8 * (1 + 8 * U) if dst == BF16 else 0)) * np.abs(exact) + (2.0 ** -148 if dst == F32 else 2.0 ** -133)
    out = torch.full((2, n + 3), 7.0, dtype=dst, device=DEV)
    S.s3gd_clip([g], max_norm, norm, ws, out=[out[:, 1:n + 1]], eps=0.0)
    assert (np.abs(host(out[:, 1:n + 1]) - exact) <= off).all() and (out[:, 0] == 7).all() and (out[:, n + 1:] == 7).all()
    if dst == F32:
        S.s3gd_clip([g], max_norm, norm, ws, eps=0.0)                     # in place
        assert (np.abs(host(g) - exact) <= off).all()


def test_a_small_factor_that_is_held_as_one():
    g = torch.tensor([[2.0 ** 126, 0.0, 2.0 ** 100]], device=DEV)         # c = 2^-126 - a step of it, and 2^-127: times 2^126 no 1 and a half
    norm, ws = torch.empty((1,), device=DEV), workspace(1)
    for max_norm in (1.0 - 2.0 ** -24, 0.5):
        t, o = g.clone(), torch.empty_like(g)
        S.s3gd_clip([t], max_norm, norm, ws, out=[o], eps=0.0)
        S.s3gd_clip([t], max_norm, norm, ws, eps=0.0)
        assert torch.equal(t, o) and abs(float(t[0, 0]) - max_norm) <= 8 * U and not t[0, 1] and float(t[0, 2]) <= 2.0 ** -26


def test_long_lists_in_a_captured_graph():
    M, shapes = 2, [(7,)] * 300 + [(33, 5)] * 300 + [(20001,)] + [(3,)] * 100           # two groups of up to 640 tensors
    grads = [rand((M,) + s, BF16 if i % 3 else F32, i) for i, s in enumerate(shapes)]
    sizes = [int(np.prod(s)) for s in shapes]
    rows, norm, ws = torch.zeros((M, sum(sizes)), device=DEV), torch.zeros((M,), device=DEV), workspace(M)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.s3gd_clip(grads, 2.0, norm, ws, out=[p.unflatten(1, s) for p, s in zip(rows.split(sizes, 1), shapes)])
    for turn in range(2):                                                               # the list is gone; the gradients are others
        for g in grads:
            g.mul_(-3)
        graph.replay()
        S.s3gd_device_status(ws)
        flat = np.concatenate([host(g).reshape(M, -1) for g in grads], 1)
        want = np.sqrt((flat ** 2).sum(1))
        exact = flat * (2.0 / (want + 1e-6))[:, None]
        assert (np.abs(host(norm) - want) <= 6 * U * want).all() and (np.abs(host(rows) - exact) <= 8 * U * np.abs(exact)).all()
