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


@pytest.mark.parametrize("dim", [1, 16, 41, 512, 1001, 2047, 4096, 8192, 9000])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size,eps", [(1e17, 1e-5), (1e18, 1e-5), (1e18, 0.0), (1e-16, 0.0), (1e-16, 1e-32)])
def test_large_and_small_entries(dim, dtype, size, eps):
    x, dy, w = rand((2, 5, dim), dtype, 6, size), rand((2, 5, dim), F32, 7), rand((dim,), F32, 8, 0.1, 1.0)
    if dim == 1 and eps < 1e-6:
        pytest.skip("one entry is its own mean")
    y = torch.empty_like(x, dtype=F32)
    S.s3gd_layer_norm(x, y, w, None, eps=eps)
    check_y(y, x, w, None, eps=eps)
    check_grad(run_grad(dy, x, w, eps=eps), dy, x, w, eps=eps)


@pytest.mark.parametrize("dim", [16, 41, 512, 1001, 8192])
def test_beyond_the_limits(dim):
    x, dy, y = rand((2, 3, dim), F32, 9), rand((2, 3, dim), F32, 10), torch.empty((2, 3, dim), device=DEV)
    x[0, 1] *= 1e21                                      # squares pass fp32's range: its row, and its worker's weight gradients
    S.s3gd_layer_norm(x, y)
    dx, dw, db = run_grad(dy, x, None)
    for t in (y, dx):
        assert t[0, 1].isnan().all() and t[0, ::2].isfinite().all() and t[1].isfinite().all()
    assert dw[0].isnan().all() and dw[1].isfinite().all() and db.isfinite().all()
    x[0, 1] *= 1e-41                                     # a variance that counts as zero, with nothing beside it
    S.s3gd_layer_norm(x, y, eps=0.0)
    assert not y[0, 1].isfinite().any() and y[0, ::2].isfinite().all() and y[1].isfinite().all()


@pytest.mark.parametrize("T,dim", [(1, 8), (1, 1001), (1, 9000), (900, 40)])
def test_weight_gradients_in_16_bits_are_rounded_once(T, dim):
    # 1 + 2^-8 lies half way between two bf16 numbers: with 2^-31 on top the upper one is nearer, but 32 bits do not hold that
    dy, x = torch.zeros((2, T, dim), device=DEV), rand((2, T, dim), F32, 11)
    dy[0, 0], dy[1, T - 1] = 2.0 ** -8 + 2.0 ** -31, -2.0 ** -8 - 2.0 ** -31
    before = torch.ones((2, 2 * dim + 3), dtype=BF16, device=DEV)
    before[1] = -1.0
    db = run_grad(dy, x, None, dst=BF16, before=before)[2]
    assert (db[0] == 1 + 2.0 ** -7).all() and (db[1] == -1 - 2.0 ** -7).all()


def guarded_workspace(M, T, dim):
    """A workspace of the stated size, and the bytes behind it."""
    n = S.s3gd_layer_norm_grad_workspace_bytes(M, T, dim)
    room = torch.full((n + 4096,), 165, dtype=torch.uint8, device=DEV)
    return room[:n], room[n:]


# 148 runs of 4096 rows are not enough: more runs, that go on from worker to worker or end with one
@pytest.mark.parametrize("M,T", [(1, 700001), (3, 300007), (4, 500003), (300, 2500), (20000, 31)])
def test_more_rows_than_148_long_runs_hold(M, T):
    dim = 16
    x, dy, w = rand((M, T, dim), F32, 12, 2.0, 0.3), rand((M, T, dim), F32, 13), rand((dim,), F32, 14, 0.3, 1.0)
    grads, dx, (ws, behind) = torch.empty((M, 2 * dim), device=DEV), torch.empty_like(x), guarded_workspace(M, T, dim)
    S.s3gd_layer_norm_grad(dy, x, dx, w, grads[:, :dim], grads[:, dim:], ws)
    S.s3gd_device_status(ws)
    assert (behind == 165).all()
    check_grad((dx, grads[:, :dim], grads[:, dim:]), dy, x, w)
    y = torch.empty_like(x)
    S.s3gd_layer_norm(x, y, w)
    check_y(y, x, w, None)


@pytest.mark.parametrize("dim", [5, 24, 300, 1000, 1001, 8192, 9000])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_what_is_not_finite_takes_its_whole_row(dim, value):
    x, dy, y = rand((2, 4, dim), F32, 15), rand((2, 4, dim), F32, 16), torch.empty((2, 4, dim), device=DEV)
    x[0, 1, dim // 2], x[1, 3, dim - 1] = value, value
    S.s3gd_layer_norm(x, y)
    dx, dw, db = run_grad(dy, x, None)
    for t in (y, dx):
        assert t[0, 1].isnan().all() and t[1, 3].isnan().all() and t[0, [0, 2, 3]].isfinite().all() and t[1, :3].isfinite().all()
    assert dw.isnan().all() and db.isfinite().all()
