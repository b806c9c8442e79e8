"""Routing of logits far from zero and far from one another, against the definition in 64 bits.

A softmax depends on differences of logits only, so its weights, means and gradients are held to a bound in the
largest difference of a row, whatever the row's offset.  The exponent of a score is a difference of logits times
log2(e), rounded once: its error, times ln 2, is the difference times U; some 24 U are left to exp2, the division and the
scale.  A sigmoid's exponent is the logit itself."""
import math

import pytest
import torch

import test_gpu_route as R
from paper_2006_16668_b200 import binding as B

pytestmark = pytest.mark.gpu

BF, F32 = R.BF, R.F32
OFFSETS = (0.0, 100.0, -100.0, 1e3, -1e3, 1e4, -1e4, 1e5, -1e5, 5e5, -5e5, 9e5)


@pytest.fixture
def bounds_in_differences(monkeypatch):
    def spread(l):
        there = torch.isfinite(l) & (l.abs() < 1e30)
        top = l.masked_fill(~there, -math.inf).amax(-1, keepdim=True)
        low = l.masked_fill(~there, math.inf).amin(-1, keepdim=True)
        return 24 + torch.where(top >= low, top - low, torch.zeros_like(top))
    monkeypatch.setattr(R, "_spread", spread)


def _offset_logits(G, S, E, dtype, std, seed, offsets=OFFSETS):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    l = torch.randn(G, S, E, generator=gen, device="cuda") * std
    at = torch.randint(0, len(offsets), (G, S, 1), generator=gen, device="cuda")
    return (l + torch.tensor(offsets, device="cuda")[at]).to(dtype)


def _both_ways(kw, logits, bias, k, m=True):
    G, S, E = logits.shape
    cfg = B.make_route(G=G, S=S, E=E, k=k, dtype="bf16" if logits.dtype == BF else "f32", **kw)
    out = R._route(cfg, logits, bias, m=m, load=m)
    R._check_forward(cfg, kw, logits, bias, out)
    gen = torch.Generator(device="cuda").manual_seed(E + k)
    dweight = torch.randn(G, S, k, generator=gen, device="cuda")
    dm = torch.randn(G, E, generator=gen, device="cuda")
    for d in (None, dm):
        R._check_backward(cfg, kw, logits, out[0], dweight, d, R._backward(cfg, logits, out[0], dweight, d))


# 8 or 32 lanes per token, single-element loads, and the kernel of every other shape
SHAPES = [(2, 70, 64, 4), (1, 2400, 64, 2), (1, 2400, 256, 8), (1, 70, 100, 3), (1, 40, 602, 2), (2, 30, 2048, 2), (1, 9, 3000, 4)]


@pytest.mark.parametrize("m", [False, True])
@pytest.mark.parametrize("std", [1.0, 8.0])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("G,S,E,k", SHAPES)
def test_raw_softmax_weights_ignore_a_common_offset(G, S, E, k, dtype, std, m, bounds_in_differences):
    logits = _offset_logits(G, S, E, dtype, std, seed=E + S)
    _both_ways(dict(renormalise=False), logits, None, k, m=m)


@pytest.mark.parametrize("kw", [{}, dict(renormalise=False, groups=4, groups_kept=2),
                                dict(renormalise=False, groups=4, groups_kept=2, group_top=2)])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("G,S,E,k", [(1, 2400, 64, 4), (2, 70, 256, 8), (1, 60, 100, 3)])
def test_offsets_with_groups_and_renormalised(G, S, E, k, dtype, kw, bounds_in_differences):
    # with sums of scores, offsets at which a step of either type leaves the scores far above 2^-53 of one another
    logits = _offset_logits(G, S, E, dtype, 2.0, seed=E + S + 1, offsets=OFFSETS[:3] if kw.get("group_top") == 2 else OFFSETS)
    _both_ways(kw, logits, None, k)


def test_barred_experts_beside_an_offset(bounds_in_differences):
    """NaN, infinities and empty rows among rows with offsets: the clean-up of one token leaves its neighbours alone."""
    for E in (64, 100, 2048):
        logits = _offset_logits(1, 300, E, F32, 1.0, seed=E)
        logits[0, ::5, 3], logits[0, 1::7, 9], logits[0, 2::11] = math.nan, -math.inf, -math.inf
        logits[0, 3::13, 5] = math.inf
        _both_ways(dict(renormalise=False), logits, None, 3)


@pytest.mark.parametrize("renormalise", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("G,S,E,k", SHAPES)
def test_sigmoid_of_wide_logits(G, S, E, k, dtype, renormalise):
    """Standard deviation 8: scores near 0 and 1, whose gradient s (1 - s) is small but not zero."""
    logits = R._logits(G, S, E, dtype, seed=3, std=8.0)
    _both_ways(dict(score="sigmoid", renormalise=renormalise), logits, None, k)


@pytest.mark.parametrize("E", [32, 100, 512, 3000])
def test_sigmoid_gradient_at_given_logits(E):
    """d m / d l = s (1 - s) / S from -90 to 90: relative error as at zero."""
    logits = torch.linspace(-90, 90, E, device="cuda").reshape(1, 1, E).contiguous()
    logits[0, 0, 0], logits[0, 0, 1] = -math.inf, math.nan
    cfg = B.make_route(G=1, S=1, E=E, k=2, score="sigmoid")
    idx = torch.full((1, 1, 2), -1, dtype=torch.int32, device="cuda")
    got = R._backward(cfg, logits, idx, torch.zeros(1, 1, 2, device="cuda"), torch.ones(1, E, device="cuda")).double()
    l = logits.double()
    want = torch.sigmoid(l) * torch.sigmoid(-l)
    assert (got[..., :2] == 0).all()
    err = (got - want).abs()[..., 2:]
    assert (err <= (24 + l[..., 2:].abs()) * 4 * R.U32 * want[..., 2:] + 1e-37).all(), float((err / want[..., 2:]).max())


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,groups,S", [(32, 8, 500), (64, 8, 2500), (96, 3, 90)])
@pytest.mark.parametrize("size", [1e3, 1e6])
def test_groups_whose_best_values_cancel(size, E, groups, S, score):
    """Each group's two best are a score plus a large bias and a score minus it: the sum is small, its error in fp32 is
    that of the large values."""
    logits = R._logits(1, S, E, F32, seed=11)
    bias = torch.full((groups, E // groups), -4 * size, device="cuda")
    bias[:, 1], bias[:, 2] = size, -size
    kw = dict(score=score, groups=groups, groups_kept=max(1, groups // 3), group_top=2)
    cfg = B.make_route(G=1, S=S, E=E, k=2, **kw)
    bias = bias.reshape(E).contiguous()
    R._check_forward(cfg, kw, logits, bias, R._route(cfg, logits, bias))


def test_group_with_one_expert_left():
    """The lowest float as a bias for experts that are switched off, all but one of some groups."""
    E, groups, S = 64, 8, 600
    for score in ("softmax", "sigmoid"):
        logits = R._logits(1, S, E, F32, seed=12)
        bias = torch.zeros(groups, E // groups, device="cuda")
        bias[2, 1:] = torch.finfo(torch.float32).min
        bias[5] = torch.finfo(torch.float32).min
        kw = dict(score=score, groups=groups, groups_kept=3, group_top=2)
        cfg = B.make_route(G=1, S=S, E=E, k=6, **kw)
        R._check_forward(cfg, kw, logits, bias.reshape(E), R._route(cfg, logits, bias.reshape(E)))
