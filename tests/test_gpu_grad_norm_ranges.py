"""Clipping where the factor leaves the range of fp32; bounds as for the other tests of the norm."""
import pytest
import torch

import test_gpu_grad_norm as norms

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("max_norm", [1e-2, 1e-3, 1e-8])
def test_factors_below_the_normal_numbers(max_norm, dtype):
    """A norm of 3e37 brought to max_norm: the factor has no normal fp32 value, the clipped gradients do."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    g = (torch.randn(1001, generator=gen, device="cuda") * 1e36).to(dtype)
    for outs in ([g], [torch.empty_like(g)], [torch.empty(1002, dtype=dtype, device="cuda")[1:]]):
        grads = [g.clone()] if outs[0] is g else [g]
        target = grads if outs[0] is g else outs
        norms.check(grads, [g], target, max_norm, *norms.clip(grads, max_norm, target))
