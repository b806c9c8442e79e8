"""Cross attention with lengths far outside of [0, k_len], which are taken into it, where a source is cut into parts and where it is whole."""
import pytest
import torch

import test_gpu_cross_attention as attn

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
LOWEST, HIGHEST = -2 ** 31, 2 ** 31 - 1


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lengths", [[LOWEST, 3000, LOWEST + 700, 1], [2900, LOWEST + 1, HIGHEST, -3000], [LOWEST] * 4])
@pytest.mark.parametrize("Tq", [1, 40, 700])
def test_lengths_far_outside(Tq, lengths, dtype):
    t = attn.make(4, Tq, 3000, 2, 1, 64, dtype, lengths)
    o, lse = attn.forward(t)
    attn.check_forward(t, o, lse)
    grads = attn.backward(t, o, lse)
    attn.check_backward(t, o, lse, grads)
    for b, n in enumerate(lengths):
        if n <= 0:
            assert not o[b].any() and not grads[0][b].any()
