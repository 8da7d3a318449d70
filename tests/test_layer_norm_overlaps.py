"""Outputs of s3gd_layer_norm and s3gd_layer_norm_grad that lie over one another, or over an input in another way: refused (no GPU)."""
import pytest

from paper_2302_07475_b200 import binding, build as B

F32, BF16, I64 = 0, 1, 4
INV = 1
X, Y, A, B_, DX, DW, WS = (1 << 20, 2 << 20, 3 << 20, 4 << 20, 5 << 20, 6 << 20, 7 << 20)      # never dereferenced: all calls are refused


@pytest.fixture(scope="module", autouse=True)
def lib():
    B.build()
    return binding.load()


def forward(lib, **kw):
    a = {"x": X, "xd": F32, "xs": 8, "xw": 32, "add": A, "as": 8, "aw": 32, "total": B_, "ts": 8, "tw": 32, "weight": None, "bias": None, "pd": F32,
         "ids": None, "idt": I64, "M": 2, "T": 4, "dim": 8, "eps": 1e-5, "y": Y, "yd": F32, "ys": 8, "yw": 32, **kw}
    return lib.s3gd_layer_norm(*a.values(), None)


@pytest.mark.parametrize("kw", [{"y": B_}, {"y": X, "total": X}, {"y": X, "yd": BF16}, {"y": X, "ys": 10, "yw": 40}, {"y": X, "yw": 40}, {"y": X, "xs": 0},
                                {"total": X, "ts": 9, "tw": 40}, {"total": X, "tw": 33}, {"total": A, "aw": 0}, {"total": A, "as": 16}], ids=str)
def test_forward(lib, kw):
    assert forward(lib, **kw) == INV


def backward(lib, **kw):
    a = {"dy": Y, "dyd": F32, "ds": 8, "dw": 32, "x": X, "xd": F32, "xs": 8, "xw": 32, "dtotal": A, "ts": 8, "tw": 32, "weight": None, "wd": F32,
         "ids": None, "idt": I64, "M": 2, "T": 4, "dim": 8, "eps": 1e-5, "dx": DX, "os": 8, "ow": 32, "dweight": DW, "dbias": DW + 32, "gd": F32, "gs": 16,
         "acc": 0, **kw}
    return lib.s3gd_layer_norm_grad(*a.values(), WS, 1 << 40, None)


@pytest.mark.parametrize("kw", [{"dx": X, "xs": 16, "xw": 64}, {"dx": X, "xw": 33}, {"dx": Y, "dyd": BF16}, {"dx": Y, "ds": 0}, {"dx": Y, "dw": 0},
                                {"dx": A, "ts": 12, "tw": 64}, {"dbias": DW}, {"dbias": DW + 28}, {"dbias": DW - 28}, {"dbias": DW + 64},
                                {"dbias": DW + 36}, {"dbias": DW - 36}, {"dbias": DW + 64 - 28}, {"dbias": DW + 92}, {"dbias": DW - 92},
                                {"M": 1, "dbias": DW + 28}, {"T": 0, "dbias": DW}, {"gd": BF16, "dbias": DW + 14}], ids=str)
def test_backward(lib, kw):
    assert backward(lib, **kw) == INV
