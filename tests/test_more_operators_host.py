"""Layer norm, its gradient, the norm over many gradients and clipping: refusals, workspace sizes and the 64-bit statements (no GPU)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2302_07475_b200 as S
from oracle import operators_oracle as O
from paper_2302_07475_b200 import binding, build as B

INV, WS = 1, 2
F32, BF16, I8, I32, I64 = range(5)
AT = 256 * 1024                          # never dereferenced: every call below is refused first


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    return binding.load()


def forward(lib, **kw):
    a = {"x": AT, "xd": F32, "xs": 8, "xw": 32, "add": None, "as": 8, "aw": 32, "total": None, "ts": 8, "tw": 32, "weight": AT, "bias": AT, "pd": F32,
         "ids": AT, "idt": I64, "M": 2, "T": 4, "dim": 8, "eps": 1e-5, "y": AT, "yd": BF16, "ys": 8, "yw": 32, **kw}
    return lib.s3gd_layer_norm(*a.values(), None)


@pytest.mark.parametrize("kw", [{"x": None}, {"y": None}, {"xd": I8}, {"yd": I32}, {"pd": I64}, {"idt": F32}, {"M": 0}, {"M": 65536}, {"dim": 0},
                                {"dim": 1 << 24}, {"T": 1 << 31}, {"M": 60000, "T": 60000}, {"eps": -1e-9}, {"eps": float("nan")},
                                {"eps": float("inf")}, {"add": AT}, {"total": AT}, {"x": AT + 2}, {"y": AT + 1}, {"weight": AT + 2},
                                {"bias": AT + 2}, {"ids": AT + 4}, {"xs": -1}, {"xw": -1}, {"ys": 7}, {"ys": 0}, {"yw": 31}, {"yw": 0},
                                {"add": AT, "total": AT, "ts": 4}, {"add": AT + 2, "total": AT}, {"add": AT, "total": AT + 2},
                                {"add": AT, "total": AT, "as": -8}], ids=str)
def test_layer_norm_refusals(lib, kw):
    assert forward(lib, **kw) == INV


def test_layer_norm_of_nothing(lib):
    assert forward(lib, T=0, x=None, y=None, ids=None) == 0


def backward(lib, ws=AT, size=1 << 40, **kw):
    a = {"dy": AT, "dyd": F32, "ds": 8, "dw": 32, "x": AT, "xd": F32, "xs": 8, "xw": 32, "dtotal": None, "ts": 8, "tw": 32, "weight": AT, "wd": F32,
         "ids": AT, "idt": I64, "M": 2, "T": 4, "dim": 8, "eps": 1e-5, "dx": AT, "os": 8, "ow": 32, "dweight": AT, "dbias": AT, "gd": F32, "gs": 16,
         "acc": 0, **kw}
    return lib.s3gd_layer_norm_grad(*a.values(), ws, size, None)


@pytest.mark.parametrize("kw", [{"dy": None}, {"x": None}, {"dyd": I8}, {"xd": I64}, {"wd": I32}, {"gd": I8}, {"idt": BF16}, {"M": 0}, {"M": 65536},
                                {"dim": 0}, {"dim": 1 << 24}, {"T": 1 << 31}, {"M": 60000, "T": 60000}, {"eps": -1.0}, {"eps": float("nan")},
                                {"dx": None, "dweight": None, "dbias": None}, {"dx": None, "dtotal": AT}, {"gs": 7}, {"gs": -16}, {"dy": AT + 2},
                                {"x": AT + 1}, {"dtotal": AT + 2}, {"dx": AT + 2}, {"weight": AT + 1}, {"ids": AT + 4}, {"dweight": AT + 2},
                                {"dbias": AT + 2}, {"ds": -1}, {"xw": -1}, {"os": 7}, {"ow": 31}], ids=str)
def test_layer_norm_grad_refusals(lib, kw):
    assert backward(lib, **kw) == INV


def test_workspace_refusals_and_sizes(lib):
    assert backward(lib, ws=None) == WS and backward(lib, size=100) == WS and backward(lib, ws=AT + 16) == WS
    assert norms(lib, ws=None) == WS and norms(lib, size=100) == WS and norms(lib, ws=AT + 16) == WS
    assert clips(lib, ws=None) == WS and clips(lib, size=100) == WS and clips(lib, ws=AT + 16) == WS
    size = S.s3gd_layer_norm_grad_workspace_bytes
    assert size(0, 1, 1) == size(1, 1, 0) == size(65536, 1, 1) == size(1, 1, 1 << 24) == size(60000, 60000, 1) == 0 and size(1, 0, 1) > 0
    assert S.s3gd_clip_workspace_bytes(0) == S.s3gd_clip_workspace_bytes(65536) == 0 and S.s3gd_clip_workspace_bytes(1) > 0
    for args in ((0, 8, 8), (1, 8, 0)):
        with pytest.raises(ValueError):
            S.alloc_layer_norm_workspace(*args, device="cpu")
    with pytest.raises(ValueError):
        S.alloc_clip_workspace(0, device="cpu")


def test_a_workspace_for_more_serves_less(lib):
    r = np.random.default_rng(1)
    for _ in range(3000):
        M, T, dim = (int(np.exp(r.uniform(0, np.log(n)))) for n in (2000, 100000, 20000))
        if M * T >= 1 << 31:
            continue
        less = tuple(int(r.integers(1, n + 1)) for n in (M, T, dim))
        assert S.s3gd_layer_norm_grad_workspace_bytes(*less) <= S.s3gd_layer_norm_grad_workspace_bytes(M, T, dim)
    sizes = [S.s3gd_clip_workspace_bytes(M) for M in range(1, 5000)]
    assert sizes == sorted(sizes)


def part(data=AT, out=AT, n=10, stride=10, out_stride=10, dtype=F32, out_dtype=F32):
    return [data or 0, out or 0, n, stride & (1 << 64) - 1, out_stride & (1 << 64) - 1, dtype | out_dtype << 32]


def packed(parts):
    flat = [v for p in parts for v in p]
    return (ctypes.c_uint64 * len(flat))(*flat)


def norms(lib, parts=None, count=None, M=2, norm=AT, ws=AT, size=1 << 40):
    parts = [part()] if parts is None else parts
    return lib.s3gd_grad_norm(packed(parts), len(parts) if count is None else count, M, norm, ws, size, None)


def clips(lib, parts=None, M=2, max_norm=1.0, eps=1e-6, norm=AT, ws=AT, size=1 << 40):
    parts = [part()] if parts is None else parts
    return lib.s3gd_clip(packed(parts), len(parts), M, max_norm, eps, norm, ws, size, None)


def test_grad_norm_refusals(lib):
    for p in (part(data=None), part(data=AT + 2), part(dtype=I8), part(dtype=7), part(n=1 << 40), part(stride=-1)):
        assert norms(lib, [p]) == INV and norms(lib, [part(), p]) == INV
    assert norms(lib, M=0) == INV and norms(lib, M=65536) == INV and norms(lib, norm=None) == INV and norms(lib, norm=AT + 2) == INV
    assert norms(lib, count=-1) == INV
    assert lib.s3gd_grad_norm(None, 1, 1, AT, AT, 1 << 40, None) == INV


def test_clip_refusals(lib):
    for p in (part(out=None), part(out=AT + 2), part(out_dtype=I32), part(out_stride=9, out=AT + 400), part(out_stride=-10, out=AT + 400),
              part(out_dtype=BF16), part(out_stride=12)):                  # the last two: in place, but not the same entries
        assert clips(lib, [p]) == INV and clips(lib, [part(), p]) == INV
    for kw in ({"max_norm": -1.0}, {"max_norm": float("inf")}, {"max_norm": float("nan")}, {"eps": -1.0}, {"eps": float("inf")}, {"M": 0}, {"norm": None}):
        assert clips(lib, **kw) == INV, kw


def test_binding_refuses_cpu_tensors():
    a, ws = torch.zeros(4, 4), torch.zeros(64, dtype=torch.uint8)
    for call in (lambda: S.s3gd_layer_norm(a, a), lambda: S.s3gd_layer_norm_grad(a, a, a, None, None, None, ws), lambda: S.s3gd_grad_norm(a, torch.zeros(4), ws),
                 lambda: S.s3gd_clip([a], 1.0, torch.zeros(4), ws)):
        with pytest.raises(TypeError):
            call()


class Stand(torch.Tensor):
    """A CPU tensor that says it lies on a GPU and whose pointer is null."""

    is_cuda = True
    device = property(lambda self: torch.device("cuda", self.index))
    get_device = lambda self: self.index  # noqa: E731
    data_ptr = lambda self: 0  # noqa: E731


def stand(shape, dtype=torch.float32, index=0):
    t = torch.zeros(shape, dtype=dtype).as_subclass(Stand)
    t.index = index
    return t


M, T, D = 2, 3, 5
CALLS = {
    "s3gd_layer_norm": (S.s3gd_layer_norm, {k: ((M, T, D), torch.float32) for k in ("x", "y", "add", "total")} | {"weight": ((D,), torch.float32),
                        "bias": ((D,), torch.float32), "ids": ((M, T), torch.int64)}, {}),
    "s3gd_layer_norm_grad": (S.s3gd_layer_norm_grad, {k: ((M, T, D), torch.float32) for k in ("dy", "x", "dx", "dtotal")} | {
                             "weight": ((D,), torch.float32), "dweight": ((M, D), torch.float32), "dbias": ((M, D), torch.float32),
                             "ids": ((M, T), torch.int64), "ws": ((64,), torch.uint8)}, {}),
    "s3gd_grad_norm": (S.s3gd_grad_norm, {"grads": ((M, D), torch.float32), "norm": ((M,), torch.float32), "ws": ((64,), torch.uint8)}, {}),
    "s3gd_clip": (S.s3gd_clip, {"grads": ((M, D), torch.float32), "norm": ((M,), torch.float32), "ws": ((64,), torch.uint8),
                                "out": ((M, D), torch.float32)}, {"max_norm": 1.0}),
}


def given(name, changed=None, shape=None, dtype=None, index=0):
    call, tensors, rest = CALLS[name]
    made = {k: stand(s, t) for k, (s, t) in tensors.items()}
    if changed:
        s, t = tensors[changed]
        made[changed] = stand(s if shape is None else shape, dtype or t, index)
    return lambda: call(**made, **rest)


@pytest.mark.parametrize("name,moved", [(n, k) for n, (_, tensors, _) in CALLS.items() for k in tensors])
def test_a_tensor_on_another_device_is_refused(name, moved):
    with pytest.raises(TypeError, match="device"):
        given(name, moved, index=1)()


@pytest.mark.parametrize("name,changed", [(n, k) for n, (_, tensors, _) in CALLS.items() for k in tensors])
def test_another_type_is_refused(name, changed):
    with pytest.raises(TypeError):
        given(name, changed, dtype=torch.float64)()


@pytest.mark.parametrize("name,changed,shape", [
    ("s3gd_layer_norm", "x", ()), ("s3gd_layer_norm", "y", (M, T, D + 1)), ("s3gd_layer_norm", "add", (T, D)), ("s3gd_layer_norm", "total", (M, T)),
    ("s3gd_layer_norm", "weight", (D + 1,)), ("s3gd_layer_norm", "bias", (1, D)), ("s3gd_layer_norm", "ids", (M * T,)),
    ("s3gd_layer_norm_grad", "x", (D,)), ("s3gd_layer_norm_grad", "dy", (M, T + 1, D)), ("s3gd_layer_norm_grad", "dx", (M * T, D)),
    ("s3gd_layer_norm_grad", "weight", (M, D)), ("s3gd_layer_norm_grad", "dweight", (D,)), ("s3gd_layer_norm_grad", "dbias", (M, D + 1)),
    ("s3gd_layer_norm_grad", "ids", (T,)), ("s3gd_grad_norm", "grads", (M + 1, D)), ("s3gd_grad_norm", "norm", (0,)), ("s3gd_clip", "out", (M, D + 1)),
    ("s3gd_clip", "grads", ())])
def test_another_shape_is_refused(name, changed, shape):
    with pytest.raises(ValueError):
        given(name, changed, shape=shape)()


def test_binding_refusals_of_combinations():
    x, w16 = stand((M, T, D)), stand((D,), torch.bfloat16)
    ws, rows = stand((64,), torch.uint8), stand((M, D))
    apart = stand((M, 2 * D))[:, :D]
    apart.index = 0
    with pytest.raises(ValueError):
        S.s3gd_layer_norm(x, x, add=x)
    with pytest.raises(TypeError):
        S.s3gd_layer_norm(x, x, stand((D,)), w16)
    with pytest.raises(TypeError):
        S.s3gd_layer_norm(x, x, add=stand((M, T, D), torch.bfloat16), total=x)
    with pytest.raises(TypeError):
        S.s3gd_layer_norm_grad(x, x, stand((M, T, D), torch.bfloat16), None, rows, rows, ws)
    with pytest.raises(TypeError):
        S.s3gd_layer_norm_grad(x, x, x, None, rows, stand((M, D), torch.bfloat16), ws)
    with pytest.raises(ValueError):
        S.s3gd_layer_norm_grad(x, x, x, None, rows, apart, ws)         # other distances between workers
    with pytest.raises(ValueError):
        S.s3gd_layer_norm_grad(x, x, None, None, None, None, ws)                          # nothing wanted
    with pytest.raises(ValueError):
        S.s3gd_layer_norm_grad(x, x, None, None, rows, rows, ws, dtotal=x)                # nothing to add it to
    with pytest.raises(ValueError):
        S.s3gd_clip([rows, rows], 1.0, stand((M,)), ws, out=[rows])
    with pytest.raises(TypeError):
        S.s3gd_clip([rows, None], 1.0, stand((M,)), ws)
    with pytest.raises(TypeError):
        S.s3gd_grad_norm([rows], stand((M, 1)), ws)


@pytest.mark.parametrize("several", [False, True])
@pytest.mark.parametrize("others", [0, 4])                                    # short lists and long ones are looked at in different ways
def test_an_output_that_is_named_twice_is_refused(several, others):
    a, b, none = torch.zeros(2, 6), torch.zeros(2, 6), torch.zeros(2, 0)
    more, M = [torch.zeros(2, 3) for _ in range(others)], 2 if several else 1
    for grads, outs in (([a, a], None), ([a, b], [b, b]), ([a, b, a], None)):
        with pytest.raises(ValueError, match="twice"):
            binding._parts(grads + more, outs and outs + more, -1, M, several, True)
    for grads, outs, writes, n in (([a, a], None, False, 2), ([a, a], [a, b], True, 2), ([none, a, none], None, True, 1)):   # read twice, or empty: fine
        packed, count = binding._parts(grads + more, outs and outs + more, -1, M, several, writes)
        assert sum(1 for k in range(count) if packed[6 * k + 2]) == n + others


# ------------------------------------------------------------------ the statements themselves
def test_layer_norm_statement():
    r = np.random.default_rng(3)
    x = r.standard_normal((2, 3, 50)) * 4 + 7
    y, xhat = O.layer_norm(x, None, None, 0.0)
    np.testing.assert_allclose(y.mean(-1), 0, atol=1e-13)
    np.testing.assert_allclose((y * y).mean(-1), 1, atol=1e-13)
    np.testing.assert_allclose(O.layer_norm(5 * x - 3, None, None, 0.0)[0], y, atol=1e-12)      # shifts and scales of a row do not matter
    ids = np.array([[0, -1, 2], [-5, 1, 1]])
    y, _ = O.layer_norm(x, np.full(50, 2.0), np.full(50, 1.0), 0.0, ids)
    assert not y[ids < 0].any()
    np.testing.assert_allclose(y[ids >= 0], 2 * xhat[ids >= 0] + 1)


def test_layer_norm_grad_is_the_derivative_of_layer_norm():
    r = np.random.default_rng(4)
    x, dy, w, b = r.standard_normal((2, 3, 6)), r.standard_normal((2, 3, 6)), r.standard_normal(6), r.standard_normal(6)
    ids = np.array([[0, -1, 2], [3, 1, 1]])
    dx, dw, db, _ = O.layer_norm_grad(dy, x, w, 1e-3, ids)

    def loss(x, w, b):
        return (dy * O.layer_norm(x, w, b, 1e-3, ids)[0]).sum((1, 2))

    h = 1e-5
    for at in np.ndindex(2, 3, 6):
        e = np.zeros_like(x)
        e[at] = h
        assert np.isclose((loss(x + e, w, b) - loss(x - e, w, b)).sum() / (2 * h), dx[at], atol=1e-8)
    for j in range(6):
        e = np.zeros(6)
        e[j] = h
        np.testing.assert_allclose((loss(x, w + e, b) - loss(x, w - e, b)) / (2 * h), dw[:, j], atol=1e-8)
        np.testing.assert_allclose((loss(x, w, b + e) - loss(x, w, b - e)) / (2 * h), db[:, j], atol=1e-8)


def test_clip_statement():
    g = [np.array([[3.0], [0.3]]), np.array([[[4.0, 0.0]], [[0.0, 0.4]]])]
    out, norm = O.clip(g, 1.0, 0.0)
    np.testing.assert_allclose(norm, [5.0, 0.5])
    np.testing.assert_allclose(out[0], [[0.6], [0.3]])
    np.testing.assert_allclose(out[1], [[[0.8, 0.0]], [[0.0, 0.4]]])
