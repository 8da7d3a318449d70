"""Operators on a language model's parameters: refusals, workspace sizes and the 64-bit statements themselves (no GPU)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2302_07475_b200 as S
from oracle import operators_oracle as O
from paper_2302_07475_b200 import binding, build as B

INV, WS = 1, 2
F32, BF16, I8, I32, I64 = range(5)
C = (3.4445, -4.7750, 2.0315)


@pytest.fixture(scope="module")
def lib():
    B.build()
    return binding.load()


def mat(ptr=256 * 1024, dtype=F32, row=8, batch=64):
    return binding.Matrix(ptr, dtype, row, batch)


FAKE = ctypes.c_void_p(256 * 1024)      # never dereferenced: every call below is refused first


def ortho(lib, g=None, out=None, batch=1, rows=8, cols=8, steps=5, coeffs=C, eps=1e-7, split=-1, ws=FAKE, size=1 << 40):
    g, out = g or mat(), out or mat()
    return lib.s3gd_orthogonalise(g, out, batch, rows, cols, steps, *coeffs, eps, split, ws, size, None)


def test_orthogonalise_refusals(lib):
    assert lib.s3gd_orthogonalise(None, mat(), 1, 8, 8, 5, *C, 1e-7, -1, FAKE, 1 << 40, None) == INV
    assert lib.s3gd_orthogonalise(mat(), None, 1, 8, 8, 5, *C, 1e-7, -1, FAKE, 1 << 40, None) == INV
    assert ortho(lib, g=mat(ptr=None)) == INV
    assert ortho(lib, g=mat(ptr=256 * 1024 + 2)) == INV                       # not aligned to its type
    assert ortho(lib, g=mat(dtype=I32)) == INV and ortho(lib, g=mat(dtype=9)) == INV
    assert ortho(lib, out=mat(dtype=I8)) == INV                               # no integer result
    assert ortho(lib, g=mat(row=7)) == INV                                    # rows run into each other
    assert ortho(lib, g=mat(batch=-1), batch=2) == INV
    assert ortho(lib, out=mat(batch=0), batch=2) == INV                       # results on top of each other
    for kw in ({"batch": 0}, {"batch": 65536}, {"rows": 0}, {"cols": 0}, {"rows": 1 << 24}, {"steps": 0}, {"steps": 33}, {"split": -2},
               {"split": 6}, {"eps": -1e-9}, {"eps": float("nan")}, {"coeffs": (float("inf"), 0, 0)},
               {"coeffs": (3.4445, 4.7750, 2.0315)}):                         # a quintic that blows up
        assert ortho(lib, **kw) == INV, kw
    assert ortho(lib, ws=None) == WS and ortho(lib, size=8) == WS and ortho(lib, ws=ctypes.c_void_p(256 * 1024 + 8)) == WS


def test_step_ortho_refusals(lib):
    def call(x=None, v=None, g=None, ws=FAKE, size=1 << 40, **kw):
        a = {"batch": 1, "rows": 8, "cols": 8, "mu": 0.9, "nesterov": 1, "lr": 0.1, "wd": 0.0, "scale": 1.0, "steps": 5, "split": -1, **kw}
        return lib.s3gd_step_ortho(x or mat(), v, g or mat(), a["batch"], a["rows"], a["cols"], a["mu"], a["nesterov"], a["lr"], a["wd"],
                                   a["scale"], a["steps"], *C, 1e-7, a["split"], ws, size, None)

    assert call(x=mat(dtype=I8)) == INV
    assert call(v=mat(dtype=BF16)) == INV                                     # momentum is fp32
    assert call(v=mat(row=4)) == INV
    assert call(g=mat(dtype=I64)) == INV
    assert call(steps=0) == INV and call(split=9) == INV
    assert call(ws=None) == WS and call(size=1) == WS


def test_embed_refusals(lib):
    def call(table=FAKE, td=F32, ts=8, vocab=10, dim=8, ids=FAKE, idt=I32, n=4, out=FAKE, od=F32, os=8):
        return lib.s3gd_embed(table, td, ts, vocab, dim, ids, idt, n, 1.0, out, od, os, None, None)

    odd = ctypes.c_void_p(256 * 1024 + 1)
    for kw in ({"table": None}, {"td": I8}, {"ts": 7}, {"vocab": 0}, {"dim": 0}, {"ids": None}, {"idt": F32}, {"out": None}, {"od": I64},
               {"os": 7}, {"table": odd}, {"ids": odd}, {"out": odd}, {"vocab": 1 << 31}, {"n": 1 << 40}):
        assert call(**kw) == INV, kw
    assert call(n=0, ids=None, out=None) == 0                                 # nothing to do, nothing enqueued


def test_embed_grad_refusals(lib):
    def call(dout=FAKE, dt=F32, ts=8, wstride=32, ids=FAKE, idt=I64, M=2, T=4, vocab=10, dim=8, grads=FAKE, gd=F32, gs=80, ws=FAKE, size=1 << 40):
        return lib.s3gd_embed_grad(dout, dt, ts, wstride, ids, idt, M, T, vocab, dim, 1.0, grads, gd, gs, 0, None, ws, size, None)

    for kw in ({"dout": None}, {"dt": I8}, {"ids": None}, {"idt": BF16}, {"M": 0}, {"M": 65536}, {"vocab": 0}, {"dim": 0}, {"grads": None},
               {"gd": I8}, {"gs": 79}, {"ts": -1}, {"T": 1 << 31}, {"M": 60000, "T": 60000}):
        assert call(**kw) == INV, kw
    assert call(ws=None) == WS and call(size=8) == WS and call(ws=ctypes.c_void_p(256 * 1024 + 16)) == WS


def test_workspace_sizes(lib):
    assert S.s3gd_orthogonalise_workspace_bytes(0, 8, 8) == 0 and S.s3gd_orthogonalise_workspace_bytes(1, 0, 8) == 0
    assert S.s3gd_orthogonalise_workspace_bytes(1, 8, 1 << 24) == 0
    assert S.s3gd_orthogonalise_workspace_bytes(1, 100, 300) == S.s3gd_orthogonalise_workspace_bytes(1, 300, 100) > 0
    assert S.s3gd_embed_grad_workspace_bytes(0, 1, 1, 1) == 0 and S.s3gd_embed_grad_workspace_bytes(1, 1, 0, 1) == 0
    assert S.s3gd_embed_grad_workspace_bytes(1, 0, 1, 1) > 0
    for f in (S.alloc_ortho_workspace, S.alloc_embed_workspace):
        with pytest.raises(ValueError):
            f(0, 8, 8, *((8,) if f is S.alloc_embed_workspace else ()), device="cpu")


def test_binding_refuses_cpu_tensors(lib):
    a, ws = torch.zeros(4, 4), torch.zeros(64, dtype=torch.uint8)
    with pytest.raises(TypeError):
        S.s3gd_orthogonalise(a, a, ws)
    with pytest.raises(TypeError):
        S.s3gd_step_ortho(a, a, 0.1, ws)
    with pytest.raises(TypeError):
        S.s3gd_embed(a, torch.zeros(2, dtype=torch.int64), torch.zeros(2, 4))
    with pytest.raises(TypeError):
        S.s3gd_embed_grad(torch.zeros(2, 4), torch.zeros(2, dtype=torch.int64), a, 4, ws)


# ------------------------------------------------------------------ the statements themselves
@pytest.mark.parametrize("shape", [(5, 9), (9, 5), (6, 6)])
def test_orthogonalise_moves_singular_values_only(shape):
    g = np.random.default_rng(1).standard_normal(shape)
    u, s, vt = np.linalg.svd(g, full_matrices=False)
    want = u @ np.diag(O.singular_map(s / np.sqrt((s * s).sum()), 5, C)) @ vt
    np.testing.assert_allclose(O.orthogonalise(g, 5, C, 0.0), want, atol=1e-12)
    assert not O.orthogonalise(np.zeros(shape), 5, C, 1e-7).any()


def test_five_steps_bring_singular_values_near_one():
    s = O.singular_map(np.linspace(0.02, 1.0, 500), 5, C)
    assert 0.6 < s.min() and s.max() < 1.25


def test_embed_grad_is_the_derivative_of_embed():
    r = np.random.default_rng(2)
    table, ids, w = r.standard_normal((7, 3)), np.array([[3, -1, 3, 6, 0, 9]]), r.standard_normal((1, 6, 3))
    grad, _ = O.embed_grad(w, ids, 7, 1.5)
    for v in range(7):
        for j in range(3):
            up, down = table.copy(), table.copy()
            up[v, j] += 0.5
            down[v, j] -= 0.5
            assert np.isclose(grad[0, v, j], (w * O.embed(up, ids, 1.5)).sum() - (w * O.embed(down, ids, 1.5)).sum())
