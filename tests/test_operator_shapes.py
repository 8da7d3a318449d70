"""Shapes that no call takes are refused by name, whatever their number of axes (stand-ins: no GPU needed)."""
import pytest
import torch

import paper_2302_07475_b200 as S
from test_operator_devices import lib, stand  # noqa: F401 -- the fixture builds the library


@pytest.mark.parametrize("shape", [(), (1,), (40,), (5, 5), (1, 40), (2, 19), (1, 5, 4), (2, 4, 5), (2, 5, 4, 1)])
def test_gradients(shape):
    with pytest.raises(ValueError, match="grads"):
        S.s3gd_embed_grad(stand((2, 3, 4)), stand((2, 3), torch.int32), stand(shape), 5, stand((64,), torch.uint8))


@pytest.mark.parametrize("ids,out", [((), ()), ((3,), ()), ((), (3, 4)), ((3,), (3,)), ((3,), (4, 4)), ((1, 3), (3, 4)), ((3,), (1, 3, 4))])
def test_lookups(ids, out):
    with pytest.raises(ValueError, match="out"):
        S.s3gd_embed(stand((5, 4)), stand(ids, torch.int32), stand(out))
