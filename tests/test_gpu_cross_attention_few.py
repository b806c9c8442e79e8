"""Cross attention of few rows (queries times the heads of a key head), in every form of the kernel that streams the source: eight rows with
wide heads, lanes beyond the head's dimensions, several blocks per key head, and on both sides of where sources are cut into parts instead.
Bounds in decoder_reference."""
import pytest
import torch

import test_gpu_cross_attention as attn

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32

LONG = [(1, 1, 9000, 1, 1, 128, None), (1, 1, 30000, 1, 1, 128, [29990]), (1, 1, 30000, 1, 1, 64, None), (1, 2, 20000, 2, 2, 72, None),
        (2, 4, 8200, 2, 2, 128, [8200, 77]), (1, 8, 3000, 1, 1, 128, None), (1, 8, 9001, 1, 1, 128, [9000]), (1, 7, 12000, 4, 4, 40, None),
        (1, 1, 20000, 8, 1, 128, None), (3, 1, 17000, 8, 1, 64, [17000, 0, 1]), (2, 3, 6000, 16, 8, 128, [5999, 1])]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("size", LONG)
def test_long_sources(size, dtype):
    t = attn.make(*size[:6], dtype, size[6])
    o, lse = attn.forward(t)
    attn.check_forward(t, o, lse)
    only, _ = attn.forward(t, lse=False)
    assert torch.equal(only, o)


FEW = [(2, 8, 150, 2, 2, 128, None), (1, 2, 200, 4, 1, 120, None), (1, 1, 1030, 2, 2, 72, None), (3, 4, 250, 2, 1, 96, [250, 0, 5]),
       (2, 7, 260, 1, 1, 104, [259, 130]), (1, 3, 2000, 1, 1, 80, [1999]), (1, 5, 300, 1, 1, 24, None), (4, 1, 700, 16, 2, 128, [700, 1, 0, 650])]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("size", FEW)
def test_few_rows(size, dtype):
    t = attn.make(*size[:6], dtype, size[6])
    o, lse = attn.forward(t)
    attn.check_forward(t, o, lse)
    attn.check_backward(t, o, lse, attn.backward(t, o, lse))
