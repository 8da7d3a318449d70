"""The last product's epilogue in tiles of which a warp finishes 64 columns after 64 columns: the matrix that is added arrives in
one buffer for both halves.  Whole 256 x 256 tiles (216 of them, no multiple of what runs at a time that would be cut in two), the
last rows of each matrix filling a warp's 32 only in part, and rows that allow no wide access, so that lanes part ways."""
import pytest
import torch

import paper_2302_07475_b200 as S
from test_gpu_ortho import DEV, exact_on_gpu, rand, tolerance, workspace

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(3, 1990, 2301), (3, 2301, 1990)])
@pytest.mark.parametrize("dtype,split", [(torch.float32, -1), (torch.bfloat16, -1), (torch.bfloat16, 0)])
def test_many_whole_tiles_with_ragged_ends(shape, dtype, split):
    x, g = rand(shape, dtype, 71, 0.02), rand(shape, torch.float32, 72)
    lr, scale, ws = 0.5, 3.0, workspace(shape)
    moved = lr * scale * exact_on_gpu(g)
    want = x.double() - moved
    room = torch.zeros(shape[:-1] + (shape[-1] + 2,), dtype=dtype, device=DEV)
    first = None
    for k in range(8):
        x1 = x.clone() if k % 2 else room[..., 1:1 + shape[-1]]
        x1.copy_(x)
        S.s3gd_step_ortho(x1, g, lr, ws, scale=scale, split_steps=split)
        S.s3gd_device_status(ws)
        if first is None:
            first = x1.clone()
        assert torch.equal(x1, first)
    for m in range(shape[0]):
        off = tolerance(torch.float32, split=None if split else 0) * moved[m].norm() + 4 * 2.0 ** -24 * x[m].double().norm()
        off += 2.0 ** -8 * want[m].norm() if dtype == torch.bfloat16 else 0.0
        assert (first[m].double() - want[m]).norm() <= off
