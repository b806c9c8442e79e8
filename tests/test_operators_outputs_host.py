"""Outputs that share memory, and sizes that the library's 32-bit arguments cannot hold, are refused: no GPU needed."""
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


def test_sizes_beyond_31_bits_are_refused():
    """A size of 2^32 + 1024 must not be taken for 1024."""
    big = (1 << 32) + 1024
    bf, f32 = torch.bfloat16, torch.float32
    e = lambda *s, dtype=bf: torch.empty(*s, dtype=dtype, device="meta")
    with pytest.raises(ValueError, match="2\\*\\*31"):
        B.gshard_layer_norm_forward(e(1, big), e(big, dtype=f32), None, e(1, big))
    with pytest.raises(ValueError, match="2\\*\\*31"):
        B.gshard_layer_norm_backward(e(1, big), e(big, dtype=f32), e(1, dtype=f32), e(1, dtype=f32), e(1, big), e(1, big))
    with pytest.raises(ValueError, match="2\\*\\*31"):
        B.gshard_linear_forward(e(1, big), e(big, 8), e(1, 8))
    with pytest.raises(ValueError, match="2\\*\\*31"):
        B.gshard_linear_forward(e(1, 8), e(8, big), e(1, big))
    with pytest.raises(ValueError, match="2\\*\\*31"):
        B.gshard_linear_backward(e(1, big), e(big, 8), e(1, 8), e(1, big))
    for call in (lambda: B.gshard_layer_norm_workspace_bytes(4, big), lambda: B.gshard_linear_workspace_bytes(4, big, 64, bf),
                 lambda: B.gshard_linear_workspace_bytes(4, 64, big, bf), lambda: B.make_route(G=1, S=big, E=8, k=2),
                 lambda: B.make_route(G=1, S=8, E=8, k=(1 << 32) + 2)):
        with pytest.raises(ValueError, match="2\\*\\*31"):
            call()
