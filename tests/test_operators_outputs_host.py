"""Outputs that share memory are refused: no GPU needed."""
import pytest
import torch

from paper_2006_16668_b200 import binding as B
from paper_2006_16668_b200.build import build_library

INVALID = B.GSHARD_ERR_INVALID_ARG
X, W, DY, PRE, DX, DW, DB, WS = (0x10000 * i for i in range(1, 9))


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_library()


def _linear_backward(dx=DX, dw=DW, db=DB, n=64, dtype=0):
    return B.load().gshard_linear_backward(n, 64, 64, dtype, dtype, 0, X, W, PRE, DY, dx, dw, db, WS, 1 << 30, None)


@pytest.mark.parametrize("dtype", [0, 1])
def test_linear_backward_refuses_one_address_for_two_gradients(dtype):
    for kw in (dict(dx=DW), dict(dw=DX), dict(db=DX), dict(db=DW), dict(dx=DW, db=DW), dict(dx=DB, dw=None), dict(dw=DB, dx=None)):
        assert _linear_backward(dtype=dtype, **kw) == INVALID, kw
    assert _linear_backward(dx=DW, n=0) == INVALID           # and where there are no rows, which clears dw and dbias
    assert _linear_backward(dw=DB, n=0) == INVALID
    if not torch.cuda.is_available():                        # absent gradients are no clash
        for kw in ({}, dict(dx=None, dw=None), dict(dw=None, db=None), dict(dx=None, db=None), dict(dx=None, dw=None, db=None)):
            assert _linear_backward(dtype=dtype, **kw) in (B.GSHARD_ERR_CUDA, B.GSHARD_ERR_ARCH), kw


def test_layer_norm_refuses_one_tensor_for_two_outputs():
    x, g, s, y = torch.zeros(4, 64), torch.zeros(64), torch.zeros(4), torch.zeros(4, 64)
    with pytest.raises(ValueError, match="mean and rstd"):
        B.gshard_layer_norm_forward(x, g, None, y, s, s)
    with pytest.raises(ValueError, match="dgamma and dbeta"):
        B.gshard_layer_norm_backward(x, g, s, torch.ones(4), y, torch.zeros(4, 64), g, g)
