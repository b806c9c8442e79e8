"""Clipping where the factor or the norm leaves the range of fp32; bounds as for the other tests of the norm."""
import math

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


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_norm_beyond_fp32_leaves_the_gradients(dtype):
    """Finite gradients whose norm, 1e39, fp32 has no number for: the norm is reported as infinite, and the gradients are left."""
    g = [torch.full((100,), 1e38, device="cuda").to(dtype), torch.ones(7, device="cuda")]
    before = [x.clone() for x in g]
    outs = [torch.zeros_like(x) for x in g]
    sumsq, norm = norms.clip(g, 1.0, outs)
    assert math.isfinite(sumsq) and norm == math.inf
    assert all(torch.equal(o, b) for o, b in zip(outs, before))
    norms.clip(g, 1.0)
    assert all(torch.equal(x, b) for x, b in zip(g, before))
