"""s3gd_layer_norm and s3gd_layer_norm_grad where the definition divides by nothing, or entries are as large as the header allows.

Tolerances are those of test_gpu_layer_norm.py.
"""
import pytest
import torch

import paper_2302_07475_b200 as S
from test_gpu_layer_norm import BF16, DEV, F32, check_grad, check_y, rand, run_grad

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [1, 7, 16, 41, 47, 97, 300, 1000, 1001, 2048, 8191, 9000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_equal_entries_without_eps_are_nan(dim, dtype):
    T = 300                                              # a number to a row: 3.7, 1.3, 0 and others of all sizes and signs
    size = rand((T,), F32, 1) * 10.0 ** torch.linspace(-6, 6, T, device=DEV)
    size[:3] = torch.tensor([3.7, 1.3, 0.0])
    x = size.to(dtype)[None, :, None].expand(1, T, dim).contiguous()
    mixed = rand((1, T, dim), dtype, 2)
    if dim > 1:
        x[0, ::5] = mixed[0, ::5]                        # rows of other entries between them
        x[0, ::5, 0] += 3
    y, w, b = torch.empty_like(x, dtype=F32), rand((dim,), F32, 3, 0.1, 1.0), rand((dim,), F32, 4)
    S.s3gd_layer_norm(x, y, w, b, eps=0.0)
    equal = torch.ones(T, dtype=torch.bool, device=DEV)
    equal[::5] = dim == 1
    assert y[0, equal].isnan().all()
    dy = rand((1, T, dim), F32, 5)
    dx, dw, db = run_grad(dy, x, w, eps=0.0)
    assert dx[0, equal].isnan().all() and dw.isnan().all() and db.isfinite().all()
    if dim > 1:
        check_y(y[:, ~equal], x[:, ~equal], w, b, eps=0.0)
        rest = [t[:, ~equal].contiguous() for t in (dy, x)]
        check_grad(run_grad(*rest, w, eps=0.0), *rest, w, eps=0.0)
