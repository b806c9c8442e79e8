"""Cross attention at the edges of its values: scores far below zero and numbers that are none among the keys in use.  Bounds in
decoder_reference, or beside the test."""
import math

import pytest
import torch

import decoder_reference as ref
import test_gpu_cross_attention as attn
from operator_reference import HALF, U32

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("first", [0, 5, 200])
@pytest.mark.parametrize("factor", [2.0, math.inf])
@pytest.mark.parametrize("Tq", [1, 140])
def test_scores_far_below_zero(Tq, factor, first, dtype):
    """q.k is -2^110 for the keys from `first` on and -2^111 or minus infinity for those before, the scale 2^-66: the former share a row's
    weight evenly, the latter have none.  Scores and weights are exact, so only the sum of the values (one fp32 rounding per 16 of them on the tensor cores, one per
    key elsewhere) and the output are rounded."""
    Tk, length, scale = 300, 290, 2.0 ** -66
    t = attn.make(1, Tq, Tk, 2, 1, 64, dtype, [length])
    t["q"].zero_()
    t["q"][..., 0] = 2.0 ** 60
    t["k"][:, :length].zero_()
    t["k"][:, :length, :, 0] = -2.0 ** 50
    t["k"][:, :first, :, 0] *= factor
    o, lse = attn.forward(t, scale=scale)
    v = t["v"][0, first:length, 0].double()
    want, size = v.mean(0), v.abs().mean(0)
    bound = (Tk + 16) * U32 * size + HALF[dtype] * (want.abs() + Tk * U32 * size)
    assert torch.isfinite(o).all() and ((o[0].double() - want).abs() <= bound).all()
    assert ((lse.double() + 2.0 ** 44).abs() <= 2.0 ** 22).all()          # four half steps of 2^44


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Tq", [1, 140])
@pytest.mark.parametrize("up", [True, False])
def test_scales_at_the_ends_of_their_range(up, Tq, dtype):
    """Queries of 2^64 on keys of 2^-126 with a scale of 2^66, and the other way round: the scores are -16 to -19 (or 2^-4 of that) though a query
    times the scale is beyond fp32 (or below its normal numbers)."""
    t = attn.make(1, Tq, 300, 2, 1, 64, dtype, [290])
    e = 1 if up else -1
    t["q"].zero_()
    t["q"][..., 0] = 2.0 ** (64 * e)
    t["k"][:, :290].zero_()
    t["k"][:, :290, 0, 0] = -(2.0 ** (-126 * e)) * (1 + torch.arange(290, device="cuda") % 4 / 16).to(dtype)
    scale = 2.0 ** (66 * e)
    o, lse = attn.forward(t, scale=scale)
    attn.check_forward(t, o, lse, scale)


def _finite_like(got, want, bound, what):
    """Finite where the formula is, there within bound of it, and nowhere else."""
    got, there = got.double(), torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), there), f"{what}: finite where the formula is not, or the other way round"
    assert ((got - want).abs()[there] <= bound[there]).all(), what


VALUE_SIZES = [(2, 1, 200, 4, 2, 64, [200, 70]), (2, 3, 150, 2, 2, 128, [150, 0]), (2, 150, 300, 4, 2, 128, [300, 130]), (2, 200, 260, 4, 2, 64, [260, 100]),
               (1, 40, 3000, 2, 1, 64, [2900]), (1, 1300, 200, 4, 1, 128, [190])]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("size", VALUE_SIZES)
@pytest.mark.parametrize("name,bad", [("q", math.nan), ("k", math.nan), ("v", math.nan), ("v", math.inf), ("v", -math.inf), ("dout", math.nan),
                                      ("dout", math.inf)])
def test_a_number_that_is_none(name, bad, size, dtype):
    """One NaN or infinity: what the formula keeps free of it stays as it was - other heads and sources, other columns of o, and dv, which
    depends neither on v nor, but for one column, on dO."""
    t = attn.make(*size[:6], dtype, size[6])
    scale = size[5] ** -0.5
    lengths = attn.lengths_of(t)
    clean = {n: x.clone() if torch.is_tensor(x) else x for n, x in t.items()}
    t[name][0, min(t[name].shape[1] - 1, 77), 0, 3] = bad
    o, lse = attn.forward(t)
    o_clean, lse_clean = attn.forward(clean)
    (want, _), (want_lse, _) = ref.attention(t["q"], t["k"], t["v"], lengths, scale)
    (_, bound), (_, lse_bound) = ref.attention(clean["q"], clean["k"], clean["v"], lengths, scale)
    _finite_like(o, want, bound, "o")
    _finite_like(lse, want_lse, lse_bound, "lse")
    grads = attn.backward(t, o, lse)
    wants = ref.attention_grad(t["q"], t["k"], t["v"], lengths, scale, o, lse, t["dout"])
    bounds = ref.attention_grad(clean["q"], clean["k"], clean["v"], lengths, scale, o_clean, lse_clean, clean["dout"])
    for got, (want, _), (_, bound), what in zip(grads, wants, bounds, ("dq", "dk", "dv")):
        if what != "dq":
            behind = (torch.arange(size[2], device="cuda") >= lengths[:, None])[:, :, None, None].expand_as(want)
            assert not got[behind].any()
            want = want.masked_fill(behind, 0.0)
        _finite_like(got, want, bound, what)
