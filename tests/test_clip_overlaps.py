"""Outputs of s3gd_clip that are read as other gradients: refused (no GPU)."""
import pytest
import torch

import paper_2302_07475_b200 as S
from paper_2302_07475_b200 import binding, build as B


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    return binding.load()


class Stand(torch.Tensor):
    """A CPU tensor that says it lies on a GPU."""

    is_cuda = True
    get_device = lambda self: 0  # noqa: E731


def stand(*shape):
    return torch.zeros(shape).as_subclass(Stand)


@pytest.mark.parametrize("several", [False, True])
@pytest.mark.parametrize("others", [0, 4])                                    # short lists and long ones are looked at in different ways
def test_an_output_that_is_read_as_another_gradient_is_refused(several, others):
    a, b, c, none = stand(2, 6), stand(2, 6), stand(2, 6), stand(2, 0)
    more, norm = [stand(2, 3) for _ in range(others)], stand(2) if several else stand(1)[0]
    ws = torch.zeros(64, dtype=torch.uint8).as_subclass(Stand)
    for grads, outs in (([a, a], [a, b]), ([a, b], [b, c]), ([a, b], [b, a]), ([none, a, b], [none, c, a])):
        with pytest.raises(ValueError, match="read"):
            S.s3gd_clip(grads + more, 1.0, norm, ws, out=outs + more)
    for grads, outs in (([a, a], [b, c]), ([a, b], [a, c]), ([a, b], [a, b]), ([none, a, none], [none, a, none])):
        binding._parts(grads + more, outs + more, 0, 2 if several else 1, several, True, True)
