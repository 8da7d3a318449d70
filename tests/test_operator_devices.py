"""Tensors of one call have to lie on one device: a pointer into another GPU's memory would fault there.

No GPU is needed: the stand-ins are CPU tensors that say they lie on a GPU and whose pointer is null, which the library refuses
where a call gets that far."""
import pytest
import torch

import paper_2302_07475_b200 as S
from paper_2302_07475_b200 import build as B


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()


class Stand(torch.Tensor):
    is_cuda = True
    device = property(lambda self: torch.device("cuda", self.index))
    get_device = lambda self: self.index  # noqa: E731
    data_ptr = lambda self: 0  # noqa: E731


def stand(shape, dtype=torch.float32, index=0):
    t = torch.zeros(shape, dtype=dtype).as_subclass(Stand)
    t.index = index
    return t


M, T, V, D, N = 2, 3, 5, 4, 40


def ws(index=0):
    return stand((64,), torch.uint8, index)


def i32(*shape):
    return lambda index=0: stand(shape, torch.int32, index)


def f32(*shape):
    return lambda index=0: stand(shape, torch.float32, index)


CALLS = {
    "s3gd_embed": (S.s3gd_embed, {"table": f32(V, D), "ids": i32(T), "out": f32(T, D), "opt_bad_count": i32(1)}, {}),
    "s3gd_embed_grad": (S.s3gd_embed_grad, {"dout": f32(M, T, D), "ids": i32(M, T), "grads": f32(M, V * D), "ws": ws, "opt_bad_count": i32(1)},
                        {"vocab": V}),
    "s3gd_orthogonalise": (S.s3gd_orthogonalise, {"g": f32(V, D), "out": f32(V, D), "ws": ws}, {}),
    "s3gd_step_ortho": (S.s3gd_step_ortho, {"x": f32(V, D), "g": f32(V, D), "v": f32(V, D), "ws": ws}, {"lr": 0.1}),
}


@pytest.mark.parametrize("name,moved", [(n, k) for n, (_, tensors, _) in CALLS.items() for k in tensors])
def test_a_tensor_on_another_device_is_refused(name, moved):
    call, tensors, rest = CALLS[name]
    with pytest.raises(TypeError, match="device"):
        call(**{k: make(1 if k == moved else 0) for k, make in tensors.items()}, **rest)
