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


M, T, V, D, N, K = 2, 3, 5, 4, 40, 3


def ws(index=0):
    return stand((64,), torch.uint8, index)


def i32(*shape):
    return lambda index=0: stand(shape, torch.int32, index)


def f32(*shape):
    return lambda index=0: stand(shape, torch.float32, index)


def i8(*shape):
    return lambda index=0: stand(shape, torch.int8, index)


STEP = {"x": f32(N), "grads": f32(M, N), "ws": ws, "opt_idx": i32(M, K), "opt_signbits": i32(M, 1), "opt_vote": i8(N)}
CALLS = {
    "s3gd_embed": (S.s3gd_embed, {"table": f32(V, D), "ids": i32(T), "out": f32(T, D), "opt_bad_count": i32(1)}, {}),
    "s3gd_embed_grad": (S.s3gd_embed_grad, {"dout": f32(M, T, D), "ids": i32(M, T), "grads": f32(M, V * D), "ws": ws, "opt_bad_count": i32(1)},
                        {"vocab": V}),
    "s3gd_orthogonalise": (S.s3gd_orthogonalise, {"g": f32(V, D), "out": f32(V, D), "ws": ws}, {}),
    "s3gd_step_ortho": (S.s3gd_step_ortho, {"x": f32(V, D), "g": f32(V, D), "v": f32(V, D), "ws": ws}, {"lr": 0.1}),
    "s3gd_topk_sign": (S.s3gd_topk_sign, {"grads": f32(M, N), "out_idx": i32(M, K), "out_signbits": i32(M, 1), "ws": ws}, {"K": K}),
    "s3gd_debug_topk_sign": (S.s3gd_debug_topk_sign, {"grads": f32(M, N), "out_idx": i32(M, K), "out_signbits": i32(M, 1), "ws": ws},
                             {"K": K, "sample_rank": 0}),
    "s3gd_randk_sign": (S.s3gd_randk_sign, {"grads": f32(M, N), "out_idx": i32(M, K), "out_signbits": i32(M, 1), "ws": ws},
                        {"K": K, "seed": 0, "step": 0}),
    "s3gd_majority_vote": (S.s3gd_majority_vote, {"idx": i32(M, K), "signbits": i32(M, 1), "out_vote": i8(N), "ws": ws}, {"M": M, "K": K, "d": N}),
    "s3gd_majority_vote_noalloc": (S.s3gd_majority_vote_noalloc, {"idx": i32(M, K), "signbits": i32(M, 1), "out_vote": i8(N),
                                                                 "opt_bad_count": i32(1)}, {"M": M, "K": K, "d": N}),
    "s3gd_apply": (S.s3gd_apply, {"x": f32(N), "vote": i8(N)}, {"lr": 0.1}),
    "s3gd_apply_momentum": (S.s3gd_apply_momentum, {"x": f32(N), "v": f32(N), "vote": i8(N)}, {"mu": 0.9, "lr": 0.1}),
    "s3gd_step": (S.s3gd_step, STEP, {"K": K, "lr": 0.1}),
    "s3gd_debug_step": (S.s3gd_debug_step, STEP, {"K": K, "lr": 0.1, "sample_rank": 0}),
    "s3gd_step_randk": (S.s3gd_step_randk, STEP, {"K": K, "lr": 0.1, "seed": 0, "step": 0}),
    "s3gd_step_ex": (S.s3gd_step_ex, {**STEP, "err": f32(M, N), "v": f32(N)}, {"K": K, "lr": 0.1}),
    "s3gd_vote_apply": (S.s3gd_vote_apply, {"x": f32(N), "msg": i32(M * (K + 1)), "ws": ws, "opt_vote": i8(N)},
                        {"n_groups": 1, "group_stride": 0, "M_group": M, "K": K, "lr": 0.1}),
    "s3gd_vote_counts": (S.s3gd_vote_counts, {"idx": i32(M, K), "signbits": i32(M, 1), "out_counts": i32(N), "opt_bad_count": i32(1)},
                         {"M": M, "K": K, "d": N}),
    "s3gd_encode_vote2": (S.s3gd_encode_vote2, {"src": i32(N), "out_words": i32(N)}, {}),
    "s3gd_apply_vote2": (S.s3gd_apply_vote2, {"x": f32(N), "words2": i32(N), "opt_vote": i8(N)}, {"lr": 0.1}),
    "s3gd_encode_vote_sparse": (S.s3gd_encode_vote_sparse, {"src": i32(N), "out_piece": i32(N), "ws": ws}, {"cap": K}),
    "s3gd_apply_vote_sparse": (S.s3gd_apply_vote_sparse, {"x": f32(N), "pieces": i32(N), "opt_bad_count": i32(1)},
                               {"n_pieces": 1, "piece_stride": 0, "cap": K, "lr": 0.1}),
}


@pytest.mark.parametrize("name,moved", [(n, k) for n, (_, tensors, _) in CALLS.items() for k in tensors])
def test_a_tensor_on_another_device_is_refused(name, moved):
    call, tensors, rest = CALLS[name]
    with pytest.raises(TypeError, match="device"):
        call(**{k: make(1 if k == moved else 0) for k, make in tensors.items()}, **rest)
