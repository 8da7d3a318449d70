"""Matrices at the ends of fp32's range.  Entries are small whole numbers times a power of two, so nothing but exponents
changes between a matrix and its multiple: with eps = 0 the results are equal bit for bit."""
import numpy as np
import pytest
import torch

import paper_2302_07475_b200 as S
from test_gpu_ortho import DEV, ortho, workspace

pytestmark = pytest.mark.gpu


def whole(shape, exponent, seed=41):
    n = np.random.default_rng(seed).integers(-7, 8, shape).astype(np.float32)
    return torch.from_numpy(np.ldexp(n, exponent)).to(DEV)


@pytest.mark.parametrize("exponent", [-149, -140, -126, 124])
@pytest.mark.parametrize("shape", [(40, 50), (60, 30), (200, 150), (150, 200), (1500, 2100)])
@pytest.mark.parametrize("dst", [torch.float32, torch.bfloat16])
def test_smallest_and_largest_entries(shape, exponent, dst):
    want = ortho(whole(shape, 0), dst, eps=0.0)
    assert torch.isfinite(want).all()
    assert torch.equal(ortho(whole(shape, exponent), dst, eps=0.0), want)


@pytest.mark.parametrize("eps", [1e-45, 1e-38, 1e-37])
@pytest.mark.parametrize("shape", [(40, 50), (200, 150)])
def test_zeros_stay_zeros_for_any_positive_eps(shape, eps):
    assert not ortho(torch.zeros(shape, device=DEV), torch.float32, eps=eps).any()


@pytest.mark.parametrize("shape", [(40, 50), (200, 150)])
@pytest.mark.parametrize("nesterov", [False, True])
def test_step_of_a_vanishing_momentum(shape, nesterov):
    out = []
    for exponent in (0, -140):                       # mu = 1: the momentum's sums are whole numbers too
        x, v = torch.zeros(shape, device=DEV), whole(shape, exponent, 42)
        S.s3gd_step_ortho(x, whole(shape, exponent), 1.0, workspace(shape), v=v, mu=1.0, nesterov=nesterov, eps=0.0)
        out.append(x)
    assert torch.isfinite(out[0]).all() and torch.equal(out[0], out[1])
