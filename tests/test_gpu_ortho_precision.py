"""A bf16 result or parameter is the fp32-accurate value rounded once.

Bound.  Let y be the exact value and z = y + e what is rounded, |e| in the Frobenius norm at most the tolerance of an fp32
result.  The distance to the nearest bf16 number changes by no more than its argument does, so |rn(z) - z| <= |rn(y) - y| + |e|
entry by entry, and |rn(z) - y| <= |rn(y) - y| + 2 |e|: the result is off by what rounding the exact value costs, plus 2 |e|.
"""
import numpy as np
import pytest
import torch

import paper_2302_07475_b200 as S
from test_gpu_ortho import DEV, exact_on_gpu, ortho, rand, tolerance, workspace

pytestmark = pytest.mark.gpu
SHAPES = [(20, 300), (40, 60), (100, 128), (256, 128), (128, 300), (300, 300), (1000, 731), (3, 130, 200), (2500, 2600), (12, 1030, 1025)]


@pytest.mark.parametrize("src", [torch.float32, torch.bfloat16, torch.int8])
@pytest.mark.parametrize("shape", SHAPES)
def test_result(shape, src):
    g = rand(shape, src, 31)
    want = exact_on_gpu(g)
    rounding = (want.to(torch.bfloat16).double() - want).norm()
    off = (ortho(g, torch.bfloat16).double() - want).norm()
    assert off <= rounding + 2 * tolerance(torch.float32) * want.norm(), f"off by {off:.6g}, rounding alone {rounding:.6g}"


@pytest.mark.parametrize("shape", [(100, 128), (2, 300, 200), (2500, 2600)])
def test_step(shape):
    x, g, v = rand(shape, torch.bfloat16, 32, 0.02), rand(shape, torch.float32, 33, 1e-3), rand(shape, torch.float32, 34, 1e-3)
    mu, lr, wd, scale = 0.9, 0.05, 0.1, 0.2 * max(shape[-2:]) ** 0.5
    x1, v1 = x.clone(), v.clone()
    S.s3gd_step_ortho(x1, g, lr, workspace(shape), v=v1, mu=mu, nesterov=True, weight_decay=wd, scale=scale)
    moved = lr * scale * exact_on_gpu(g.double() + float(np.float32(mu)) * v1.double())
    want = (1 - lr * wd) * x.double() - moved
    rounding = (want.to(torch.bfloat16).double() - want).norm()
    e = 4 * 2.0 ** -24 * x.double().norm() + tolerance(torch.float32) * moved.norm()     # a few fp32 roundings, and the matrix's own
    assert (x1.double() - want).norm() <= rounding + 2 * e
