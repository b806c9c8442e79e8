"""Infinities, NaN and very large values under the linear operator's activations and in its gradient, against the
definition in 64 bits.  They are put into the pre-activations through the bias (one of each per column), so that every
type and every kernel meets them."""
import math

import pytest
import torch

import test_gpu_linear as L
from operator_reference import HALF, activation, slope

pytestmark = pytest.mark.gpu

BF, F32 = L.BF, L.F32
ODD = (math.inf, -math.inf, math.nan, 1e20, -1e20, 1e30, -1e30, 3e38, -3e38)

# one or two rows, up to 8 of fp32, one launch, pairs of CTAs, one CTA per tile, runs of a cut contraction
SIZES = [(1, 256, 512), (8, 256, 512), (300, 256, 512), (3000, 256, 512), (100, 264, 37888), (130, 40000, 64)]


@pytest.mark.parametrize("dtype,out", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("act", L.ACTS)
@pytest.mark.parametrize("n,K,cols", SIZES)
def test_activation_of_infinity_nan_and_huge_values(n, K, cols, act, dtype, out):
    t = L._make(n, K, cols, dtype, out)
    t["bias"][:len(ODD)] = torch.tensor(ODD, device="cuda")
    t["bias"][-len(ODD):] = torch.tensor(ODD, device="cuda")
    y, kept = L._forward(t, act, pre=True)
    pre = t["x"].double() @ t["w"].double() + t["bias"].double()
    for what, got, want in (("pre", kept, pre), ("y", y, activation(pre, act))):
        got = got.double()
        assert torch.equal(torch.isnan(got), torch.isnan(want)), what
        assert torch.equal(torch.isinf(got), torch.isinf(want)), what
        assert torch.equal(got[torch.isinf(got)], want[torch.isinf(want)]), what
        there = torch.isfinite(want)
        # x . w is about 1, far from its neighbours in size: the columns of huge values have two roundings and the exp
        # of an activation, the others are held by the general tests
        huge = there & (pre.abs() > 1e10)
        bound = (HALF[out] * 1.01 + 8 * L.U32) * want.abs() + 1e-30
        assert ((got - want).abs() <= bound)[huge].all(), what
    rest = slice(len(ODD), cols - len(ODD))
    u = {k: (v[..., rest].contiguous() if k in ("w", "bias", "dy") else v) for k, v in t.items()}
    L._check_forward(u, y[:, rest], kept[:, rest], act)


@pytest.mark.parametrize("dtype,out", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("act", L.ACTS[1:])
def test_slope_far_from_zero(act, dtype, out):
    """dbias of a single row is dy times the slope: 0 or 1 however large the pre-activation is."""
    far = [s * v for v in (100.0, 1e4, 1e10, 1e19, 2e19, 1e25, 1e30, 3e38) for s in (1, -1)]
    cols = len(far)
    t = L._make(1, 64, cols, dtype, out)
    t["pre"] = torch.tensor([far], device="cuda").to(out)
    gx, gw, gb = L._backward(t, act)
    want = t["dy"].double()[0] * slope(t["pre"].double(), act)[0]
    assert torch.isfinite(want).all()
    assert ((gb.double() - want).abs() <= 8 * L.U32 * t["dy"].double()[0].abs()).all(), gb
    assert torch.isfinite(gx).all() and torch.isfinite(gw).all()
