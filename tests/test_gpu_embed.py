"""s3gd_embed and s3gd_embed_grad on the GPU against the 64-bit statement.

Tolerances.  The lookup is one fp32 product, rounded once more where the result is bf16: compared bit for bit with the same
two operations in numpy / torch.  A sum of n terms in fp32, in whatever grouping, is within n 2^-24 of the exact one relative
to the sum of magnitudes; the products with the scale and the last addition of `accumulate` add two roundings; bf16 results
add half a unit of their 8 bits, 2^-8 of the result.
"""
import numpy as np
import pytest
import torch

import paper_2302_07475_b200 as S
from oracle import operators_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda"


def rand(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator(DEV).manual_seed(seed), device=DEV).to(dtype)


def tokens(shape, vocab, seed, dtype=torch.int64, masked=0.2, few=0):
    """Ids with a few very common ones among them, empty places, and (few > 0) only that many different ones."""
    g = torch.Generator(DEV).manual_seed(seed)
    ids = (torch.rand(shape, generator=g, device=DEV) ** 4 * (few or vocab)).long().clamp(max=vocab - 1)
    return torch.where(torch.rand(shape, generator=g, device=DEV) < masked, torch.full_like(ids, -1), ids).to(dtype)


@pytest.mark.parametrize("src", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dst", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("idt", [torch.int32, torch.int64])
@pytest.mark.parametrize("n,vocab,dim", [(1, 1, 1), (1, 50, 64), (7, 3, 3), (33, 100, 100), (1000, 77, 8), (257, 1000, 768), (64, 20, 1030),
                                         (5, 9, 4099), (5000, 300, 36)])
def test_lookup(n, vocab, dim, src, dst, idt):
    table, ids = rand((vocab, dim), src, 1), tokens((n,), vocab, 2, idt)
    out = torch.full((n, dim), 7.0, dtype=dst, device=DEV)
    S.s3gd_embed(table, ids, out, scale=1.7)
    rows = table[ids.clamp(min=0).long()].float() * torch.tensor(1.7, device=DEV)
    assert torch.equal(out, torch.where((ids >= 0)[:, None], rows, torch.zeros_like(rows)).to(dst))


def test_lookup_places_strides_and_ids_out_of_range():
    table = rand((40, 50), torch.float32, 3)[:, 3:24]
    ids = torch.tensor([0, -1, 39, 40, 5, 2 ** 31 + 5, -2 ** 40], device=DEV)
    room, bad = torch.full((7, 30), 5.0, device=DEV), torch.full((1,), -1, dtype=torch.int32, device=DEV)
    S.s3gd_embed(table, ids, room[:, 2:23], opt_bad_count=bad)
    want = O.embed(table.cpu().numpy(), ids.cpu().numpy(), 1.0)
    assert np.array_equal(room[:, 2:23].double().cpu().numpy(), want) and int(bad) == 2
    assert (room[:, :2] == 5.0).all() and (room[:, 23:] == 5.0).all()
    out = torch.empty((2, 3, 21), device=DEV)                     # ids of more than one axis
    S.s3gd_embed(table, ids[:6].view(2, 3), out)
    assert np.array_equal(out.view(6, 21).double().cpu().numpy(), want[:6])
    S.s3gd_embed(table, ids[:0], torch.empty((0, 21), device=DEV), opt_bad_count=bad)
    assert int(bad) == 0


def test_lookup_keeps_what_is_not_finite_to_its_own_row():
    table = rand((4, 16), torch.float32, 4)
    table[2] = float("nan")
    table[3] = float("inf")
    out = torch.empty((4, 16), device=DEV)
    S.s3gd_embed(table, torch.tensor([0, 2, -1, 3], device=DEV), out, scale=2.0)
    assert torch.equal(out[0], 2 * table[0]) and torch.isnan(out[1]).all() and not out[2].any() and torch.isinf(out[3]).all()


def run_grad(dout, ids, vocab, dst=torch.float32, scale=1.3, before=None, grads=None):
    M, T, dim = dout.shape
    if grads is None:
        grads = torch.full((M, vocab * dim), float("nan"), dtype=dst, device=DEV) if before is None else before.clone()
    ws = S.alloc_embed_workspace(M, T, vocab, dim, DEV)
    ws.fill_(255)
    bad = torch.full((1,), -1, dtype=torch.int32, device=DEV)
    S.s3gd_embed_grad(dout, ids, grads, vocab, ws, scale=scale, accumulate=before is not None, opt_bad_count=bad)
    S.s3gd_device_status(ws)
    assert int(bad) == int((ids >= vocab).sum())
    return grads


def check_grad(got, dout, ids, vocab, scale=1.3, before=None):
    M, T, dim = dout.shape
    want, size = O.embed_grad(dout.float().cpu().numpy(), ids.cpu().numpy(), vocab, scale)
    counts = np.stack([np.bincount(r[(r >= 0) & (r < vocab)], minlength=vocab) for r in ids.cpu().numpy().astype(np.int64)])
    off = (counts[:, :, None] + 3) * 2.0 ** -24 * size
    if before is not None:
        old = before.double().cpu().numpy().reshape(want.shape)
        want = want + old
        off = off + 2.0 ** -24 * np.abs(want)
    if got.dtype == torch.bfloat16:
        off = off * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)
    have = got.double().cpu().numpy().reshape(want.shape)
    assert np.isfinite(have).all()
    assert (np.abs(have - want) <= off).all(), f"worst {np.max(np.abs(have - want) - off):.3g}"
    if before is not None:
        assert np.array_equal(have[counts == 0], before.double().cpu().numpy().reshape(want.shape)[counts == 0])
    else:
        assert not have[counts == 0].any()


CASES = [(1, 0, 5, 8), (1, 1, 1, 1), (1, 1, 300, 65), (2, 3, 5, 3), (1, 33, 7, 64), (3, 100, 50, 100), (1, 700, 40, 768), (1, 1000, 5000, 36),
         (2, 2100, 900, 24), (1, 5000, 64, 130), (4, 1500, 3000, 16), (1, 9000, 20000, 8), (1, 300, 3, 4100), (70, 40, 20, 12)]


@pytest.mark.parametrize("M,T,vocab,dim", CASES)
@pytest.mark.parametrize("src,dst", [(torch.float32, torch.float32), (torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16),
                                     (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_grad(M, T, vocab, dim, src, dst, accumulate):
    dout, ids = rand((M, T, dim), src, 5), tokens((M, T), vocab, 6, torch.int32 if dim % 2 else torch.int64)
    before = rand((M, vocab * dim), dst, 7) if accumulate else None
    check_grad(run_grad(dout, ids, vocab, dst, before=before), dout, ids, vocab, before=before)


@pytest.mark.parametrize("M,T,few,dim", [(1, 600, 1, 20), (1, 20000, 1, 12), (2, 6000, 2, 64), (1, 30000, 3, 8), (1, 4097, 40, 20)])
def test_grad_where_few_words_take_the_tokens(M, T, few, dim):
    vocab = 1000
    dout, ids = rand((M, T, dim), torch.float32, 8), tokens((M, T), vocab, 9, few=few)
    check_grad(run_grad(dout, ids, vocab), dout, ids, vocab)


@pytest.mark.parametrize("T", [50, 6000])
def test_grad_with_nothing_left(T):
    dout = torch.full((2, T, 16), float("nan"), device=DEV)       # masked places may hold anything
    ids = torch.full((2, T), -1, device=DEV)
    assert not run_grad(dout, ids, 30).any()
    before = rand((2, 30 * 16), torch.float32, 10)
    assert torch.equal(run_grad(dout, ids, 30, before=before), before)
    ids[1] = 30                                                   # and so may places whose id is out of range
    assert not run_grad(dout, ids, 30).any()


@pytest.mark.parametrize("T", [60, 7000])
def test_grad_does_not_leak_masked_or_foreign_rows(T):
    vocab, dim = 90, 20
    dout, ids = rand((1, T, dim), torch.float32, 11), tokens((1, T), vocab, 12)
    dout[ids < 0] = float("nan")
    ids[0, 3] = 17
    dout[0, 3] = float("inf")
    got = run_grad(dout, ids, vocab).view(vocab, dim)
    assert not torch.isnan(got).any() and torch.isinf(got[17]).all() and torch.isfinite(got[:17]).all() and torch.isfinite(got[18:]).all()


@pytest.mark.parametrize("T", [100, 5000])
def test_grad_strides_and_its_part_of_a_row(T):
    M, vocab, dim = 3, 70, 21
    wide, ids = rand((T, M, dim + 6), torch.bfloat16, 13), tokens((M, T), vocab, 14)
    dout = wide.transpose(0, 1)[..., 5:5 + dim]
    room = torch.full((M, 40 + vocab * dim + 9), 2.0, device=DEV)   # the table is one part of a model's coordinates
    run_grad(dout, ids, vocab, grads=room[:, 37:37 + vocab * dim])
    check_grad(room[:, 37:37 + vocab * dim], dout.contiguous(), ids, vocab)
    room[:, 37:37 + vocab * dim] = 2.0
    assert (room == 2.0).all()
    table = torch.empty((M, vocab, dim), device=DEV)
    run_grad(dout, ids, vocab, grads=table)
    check_grad(table, dout.contiguous(), ids, vocab)
    one = torch.empty((vocab, dim), device=DEV)
    ws = S.alloc_embed_workspace(1, T, vocab, dim, DEV)
    S.s3gd_embed_grad(dout[0], ids[0].contiguous(), one, vocab, ws, scale=1.3)
    assert torch.equal(one, table[0])
    # one gradient for every token (a sum's): stride 0
    ones = rand((dim,), torch.float32, 15).expand(M, T, dim)
    check_grad(run_grad(ones, ids, vocab), ones.contiguous(), ids, vocab)


@pytest.mark.parametrize("M,T,vocab,dim", [(1, 300, 100, 64), (2, 30000, 500, 40), (1, 20000, 70000, 16)])
def test_grad_is_the_same_in_every_run_on_any_stream(M, T, vocab, dim):
    dout, ids = rand((M, T, dim), torch.float32, 16), tokens((M, T), vocab, 17)
    want = run_grad(dout, ids, vocab)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = run_grad(dout, ids, vocab)
    side.synchronize()
    assert torch.equal(want, again)
    ws, grads = S.alloc_embed_workspace(M, T, vocab, dim, DEV), torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.s3gd_embed_grad(dout, ids, grads, vocab, ws, scale=1.3)
    for _ in range(3):
        grads.fill_(-1.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(want, grads)


def test_grad_is_the_derivative_of_the_lookup():
    """sum(w * lookup(table)) is linear in the table: its difference between two tables is the gradient's product with theirs."""
    vocab, dim, T = 200, 48, 3000
    ids, w = tokens((1, T), vocab, 18), rand((1, T, dim), torch.float32, 19)
    grad = run_grad(w, ids, vocab, scale=0.5).view(vocab, dim).double()
    table, way = rand((vocab, dim), torch.float32, 20), rand((vocab, dim), torch.float32, 21)
    value = []
    for t in (table + way, table - way):
        out = torch.empty((1, T, dim), device=DEV)
        S.s3gd_embed(t, ids, out, scale=0.5)
        value.append((out.double() * w.double()).sum())
    want, scale = (value[0] - value[1]) / 2, (w.double().abs().sum() * 4)
    assert abs(float((grad * way.double()).sum() - want)) <= float(scale) * 2.0 ** -22


def test_offsets_past_32_bits():
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    vocab, dim = 140_000, 32_768                                   # 4.6e9 entries
    table = torch.zeros((vocab, dim), dtype=torch.bfloat16, device=DEV)
    table[139_990] = 3.0
    table[7] = 2.0
    ids = torch.tensor([[139_990, 7, -1, 139_990]], device=DEV)
    out = torch.empty((1, 4, dim), dtype=torch.bfloat16, device=DEV)
    S.s3gd_embed(table, ids, out)
    assert [float(r.float().mean()) for r in out[0]] == [3.0, 2.0, 0.0, 3.0]
    table.fill_(5.0)
    ws = S.alloc_embed_workspace(1, 4, vocab, dim, DEV)
    S.s3gd_embed_grad(out, ids, table.unsqueeze(0), vocab, ws)
    assert (table[139_990] == 6.0).all() and (table[7] == 2.0).all()
    table[139_990], table[7] = 0.0, 0.0
    assert not any(bool(part.any()) for part in table.split(10_000))


def test_binding_refusals():
    table, ids, out = rand((9, 8), torch.float32, 1), torch.zeros(4, dtype=torch.int64, device=DEV), torch.empty((4, 8), device=DEV)
    with pytest.raises(TypeError):
        S.s3gd_embed(table, ids.float(), out)
    with pytest.raises(TypeError):
        S.s3gd_embed(table.double(), ids, out)
    with pytest.raises(ValueError):
        S.s3gd_embed(table, ids, out[:3])
    with pytest.raises(ValueError):
        S.s3gd_embed(table, ids, torch.empty((4, 9), device=DEV))
    with pytest.raises(ValueError):
        S.s3gd_embed(table.mT, ids, out)
    ws, grads = S.alloc_embed_workspace(1, 4, 9, 8, DEV), torch.empty((1, 72), device=DEV)
    with pytest.raises(ValueError):
        S.s3gd_embed_grad(out.unsqueeze(0), ids, grads, 9, ws)
    with pytest.raises(ValueError):
        S.s3gd_embed_grad(out, ids, grads, 10, ws)
    with pytest.raises(ValueError):
        S.s3gd_embed_grad(out.mT.contiguous().mT, ids, grads, 9, ws)
    with pytest.raises(S.S3gdError) as e:
        S.s3gd_embed_grad(out, ids, grads, 9, ws[:0])
    assert e.value.code == 2
