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


@pytest.mark.parametrize("n,K,cols", [(5, 64, 64), (300, 264, 520), (2100, 1024, 1032)])
@pytest.mark.parametrize("act", L.ACTS)
@pytest.mark.parametrize("out", [BF, F32])
def test_infinite_gradient(out, act, n, K, cols):
    """An infinite dy reaches its row of dx, its column of dw and its dbias as an infinity, in products of every size."""
    t = L._make(n, K, cols, BF, out)
    t["pre"][2, 3] = 1.0
    t["dy"][2, 3], t["dy"][4, 5] = math.inf, -math.inf
    t["pre"][4, 5] = 2.0
    t["w"][:, 3] = torch.where(t["w"][:, 3].abs() < 1e-3, torch.full_like(t["w"][:, 3], 0.5), t["w"][:, 3])
    t["w"][:, 5] = t["w"][:, 3]
    t["x"][2] = torch.where(t["x"][2].abs() < 1e-3, torch.full_like(t["x"][2], 0.5), t["x"][2])
    t["x"][4] = t["x"][2]
    gx, gw, gb = L._backward(t, act)
    inf = torch.full((), math.inf, device="cuda")
    assert torch.equal(gx[2].float(), torch.sign(t["w"][:, 3].float()) * inf)
    assert torch.equal(gx[4].float(), -torch.sign(t["w"][:, 5].float()) * inf)
    assert torch.equal(gw[:, 3].float(), torch.sign(t["x"][2].float()) * inf)
    assert torch.equal(gw[:, 5].float(), -torch.sign(t["x"][4].float()) * inf)
    assert gb[3] == math.inf and gb[5] == -math.inf
    keep_rows = [i for i in range(n) if i not in (2, 4)]
    keep_cols = [i for i in range(cols) if i not in (3, 5)]
    assert torch.isfinite(gx[keep_rows]).all() and torch.isfinite(gw[:, keep_cols]).all() and torch.isfinite(gb[keep_cols]).all()


@pytest.mark.parametrize("dtype,act", [(BF, "gelu"), (F32, "silu")])
def test_offsets_beyond_32_bits(dtype, act):
    """More than 2^31 elements in y, pre, dy and the residual: rows and columns at both ends against the formula."""
    n, K, cols = 65600, 64, 32800
    t = {"x": torch.empty(n, K, dtype=dtype, device="cuda").normal_(),
         "w": torch.empty(K, cols, dtype=dtype, device="cuda").normal_(std=K ** -0.5),
         "bias": torch.randn(cols, device="cuda")}
    t["dy"], t["residual"] = (torch.empty(n, cols, dtype=dtype, device="cuda").normal_() for _ in range(2))
    y, kept = L._forward(t, act, residual=True, pre=True)
    rows = torch.cat([torch.arange(0, 64), torch.arange(n - 200, n)]).cuda()
    u = {k: (v[rows] if v.shape[0] == n else v) for k, v in t.items()}
    L._check_forward(u, y[rows], kept[rows], act, residual=True)
    del y
    t["pre"] = kept
    gx, gw, gb = L._backward(t, act)
    u["pre"] = kept[rows]
    L._check_backward(u, act, gx[rows], None, None)
    at = torch.cat([torch.arange(0, 16), torch.arange(cols - 24, cols)]).cuda()
    v = {k: (t[k][:, at] if k in ("w", "dy", "pre") else t[k]) for k in ("x", "w", "dy", "pre")}
    L._check_backward(v, act, None, gw[:, at], gb[at])


@pytest.mark.parametrize("scale", [1e-30, 1e-33, 1e-36, 1e-38])
@pytest.mark.parametrize("n", [4, 64, 3000])
def test_fp32_operands_near_the_smallest_float(n, scale):
    """The three bf16 planes of an entry end at 2^-133: below 2^-110 that, and not 24 bits, bounds what is lost of it, half
    a step of 2^-133."""
    t = L._make(n, 512, 256, F32)
    t["x"] *= scale
    y, _ = L._forward(t, bias=False)
    x, w = t["x"].double(), t["w"].double()
    bound = L._steps(t, 512) * (x.abs() @ w.abs()) + 2.0 ** -134 * w.abs().sum(0) + 512 * 2.0 ** -149
    assert ((y.double() - x @ w).abs() <= bound).all()
