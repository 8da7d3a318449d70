"""Routes of the operators that only their size or number opens: sort tiles of long rows, chunks of more than 32 places, three
and four digits of a sort key, small matrices that share an SM.

Gradient sums are of small whole numbers: exact in fp32 in any order, so that one lost or doubled token shows.
"""
import pytest
import torch

import paper_2302_07475_b200 as S
from test_gpu_ortho import DEV, exact_on_gpu, near, ortho, rand, tolerance, workspace

pytestmark = pytest.mark.gpu


def whole_numbers(shape, dtype, seed):
    return torch.randint(-4, 5, shape, generator=torch.Generator(DEV).manual_seed(seed), device=DEV).to(dtype)


def check_whole(dout, ids, vocab, accumulate=False):
    M, T, dim = dout.shape
    want = torch.zeros((M, vocab, dim), dtype=torch.float64, device=DEV)
    grads = torch.full((M, vocab * dim), float("nan"), device=DEV)
    if accumulate:
        grads = whole_numbers((M, vocab * dim), torch.float32, 51)
        want += grads.view(want.shape).double()
    for m in range(M):
        keep = (ids[m] >= 0) & (ids[m] < vocab)
        want[m].index_add_(0, ids[m][keep].long(), dout[m][keep].double())
    ws = S.alloc_embed_workspace(M, T, vocab, dim, DEV)
    ws.fill_(255)
    S.s3gd_embed_grad(dout, ids, grads, vocab, ws, accumulate=accumulate)
    S.s3gd_device_status(ws)
    assert torch.equal(grads.view(want.shape).double(), want)


def with_counts(counts, T, rest_from, vocab, seed):
    """T ids: word i counts[i] times, the other places over [rest_from, vocab) evenly; shuffled."""
    g = torch.Generator(DEV).manual_seed(seed)
    head = torch.repeat_interleave(torch.arange(len(counts), device=DEV), torch.tensor(counts, device=DEV))
    rest = torch.randint(rest_from, vocab, (T - head.numel(),), generator=g, device=DEV)
    return torch.cat([head, rest])[torch.randperm(T, generator=g, device=DEV)]


@pytest.mark.parametrize("src", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [131_072, 131_073, 262_145, 300_000])
def test_long_rows(T, src):
    """Words that take 0 to 79 places, among them 32 (a chunk at the shorter lengths), 33, 36 and 37 (a chunk of 300000), and a few
    that take a tenth of all."""
    vocab, dim = 9_001, 8
    counts = list(range(80)) + [T // 10, T // 10 + 1, 4096, 4097]
    ids = with_counts(counts, T, 100, vocab, 52)
    check_whole(whole_numbers((1, T, dim), src, 53), ids[None], vocab)


@pytest.mark.parametrize("accumulate", [False, True])
def test_long_rows_of_two_workers_with_empty_places(accumulate):
    T, vocab, dim = 140_001, 3_000, 12
    ids = torch.stack([with_counts(list(range(70)) + [30_000], T, 80, vocab, 54 + m) for m in range(2)]).int()
    ids[0, ::7] = -1
    ids[1, 5::1000] = vocab
    check_whole(whole_numbers((2, T, dim), torch.float32, 56), ids, vocab, accumulate)


@pytest.mark.parametrize("T", [4096, 4097, 9000])
@pytest.mark.parametrize("vocab,dim", [((1 << 18) - 1, 3), ((1 << 18) + 1, 3), ((1 << 27) + 3, 1)])
def test_keys_of_three_and_four_digits(T, vocab, dim):
    ids = with_counts([40, 1, 500], T, 3, vocab, 57)
    ids[:2] = vocab - 1
    check_whole(whole_numbers((1, T, dim), torch.float32, 58), ids[None], vocab)


MANY = [(300, 48, 64), (300, 64, 48), (333, 33, 47), (200, 64, 64), (150, 7, 90), (160, 100, 128)]


@pytest.mark.parametrize("shape", MANY)
@pytest.mark.parametrize("src,dst", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.int8, torch.float32)])
def test_more_small_matrices_than_sms(shape, src, dst):
    g = rand(shape, src, 59)
    near(ortho(g, dst), exact_on_gpu(g).cpu().numpy(), tolerance(dst))
    wide = rand((shape[0], shape[1], shape[2] + 5), src, 60)             # rows at odd offsets
    wide[..., 3:3 + shape[2]] = g
    assert torch.equal(ortho_into(wide[..., 3:3 + shape[2]], shape, dst), ortho(g, dst))


def ortho_into(g, shape, dst):
    room = torch.full((shape[0], shape[1] + 1, shape[2] + 3), 3.0, dtype=dst, device=DEV)
    out, ws = room[:, :-1, 1:1 + shape[2]], workspace(shape)
    S.s3gd_orthogonalise(g, out, ws)
    S.s3gd_device_status(ws)
    got = out.clone()
    out.fill_(3.0)
    assert (room == 3.0).all()
    return got


@pytest.mark.parametrize("shape", [(300, 48, 64), (333, 47, 33)])
def test_steps_of_more_small_matrices_than_sms(shape):
    x, g, v = rand(shape, torch.float32, 61, 0.02), rand(shape, torch.float32, 62, 1e-3), rand(shape, torch.float32, 63, 1e-3)
    x1, v1, ws = x.clone(), v.clone(), workspace(shape)
    S.s3gd_step_ortho(x1, g, 0.01, ws, v=v1, mu=0.5, nesterov=False, weight_decay=0.1, scale=2.0)
    S.s3gd_device_status(ws)
    assert torch.equal(v1, 0.5 * v + g)
    moved = 0.02 * exact_on_gpu(v1)
    want = (1 - 0.01 * 0.1) * x.double() - moved
    for k in range(shape[0]):
        assert (x1[k].double() - want[k]).norm() <= 4 * 2.0 ** -24 * x[k].double().norm() + tolerance(torch.float32) * moved[k].norm()
