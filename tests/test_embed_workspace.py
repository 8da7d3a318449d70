"""A workspace for some number of tokens, workers, rows or columns serves every smaller one: callers size it once for the most."""
import random

import pytest

import paper_2302_07475_b200 as S
from paper_2302_07475_b200 import build as B


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()


def size(M, T, vocab, dim):
    return S.s3gd_embed_grad_workspace_bytes(M, T, vocab, dim)


@pytest.mark.parametrize("M", [1, 3, 1000])
@pytest.mark.parametrize("vocab,dim", [(100, 1), (32_000, 4096), (1 << 30, 8)])
def test_grows_with_the_tokens(M, vocab, dim):
    edges = [0, 1, 512, 513, 4096, 4097, 1 << 17, 1 << 18, 1 << 19, 3 << 18, (1 << 20) - 1, 1 << 20]
    edges = sorted({t + o for t in edges for o in (-1, 0, 1, 2, 500, 5000)} - {-1})
    sizes = [size(M, t, vocab, dim) for t in edges]
    assert all(sizes) and sizes == sorted(sizes)


def test_grows_with_everything():
    r = random.Random(0)
    for _ in range(3000):                       # M T stays below 2^31, the limit of a call
        a = [r.randint(1, 40), int(2 ** r.uniform(0, 20)), int(2 ** r.uniform(0, 30)), int(2 ** r.uniform(0, 13))]
        b = list(a)
        b[r.randrange(4)] += r.choice((1, 1, 7, 1000))
        assert size(*a) <= size(*b), (a, b)
