"""Routing with general scores, bias, groups and k, and its gradient, against the definition in 64 bits.

Choices and counts must be equal: the reference compares in 64 bits, where inputs drawn from 2^24 values
leave no near ties, and equal values go to the lower index on both sides.  Weights are a few fp32 operations
on exp of a difference of logits: (24 + largest |difference|) U relative, plus E / 8 + 16 additions in a softmax sum."""
import math

import pytest
import torch

from operator_reference import HALF, U32, choose, log_scores, route_weights, scores, usable, within
from paper_2006_16668_b200 import binding as B

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def _logits(G, S, E, dtype, seed=0, masked=False, std=1.0):
    gen = torch.Generator(device="cuda").manual_seed(G * 7919 + S * 31 + E + seed)
    l = torch.randn(G, S, E, generator=gen, device="cuda") * std
    if masked:
        l[torch.rand(G, S, E, generator=gen, device="cuda") < 0.3] = -math.inf
        l[torch.rand(G, S, generator=gen, device="cuda") < 0.1] = -math.inf
        l[torch.rand(G, S, E, generator=gen, device="cuda") < 0.02] = math.nan
        l[torch.rand(G, S, E, generator=gen, device="cuda") < 0.002] = math.inf
    return l.to(dtype)


def _route(cfg, logits, bias=None, m=True, load=True):
    G, S, E, k = cfg.G, cfg.S, cfg.E, cfg.k
    idx = torch.full((G, S, k), -7, dtype=torch.int32, device="cuda")
    weight = torch.full((G, S, k), math.nan, device="cuda")
    m = torch.full((G, E), math.nan, device="cuda") if m else None
    load = torch.full((G, E), -7, dtype=torch.int32, device="cuda") if load else None
    ws = torch.empty(B.gshard_moe_route_workspace_bytes(cfg), dtype=torch.uint8, device="cuda") if m is not None else None
    B.gshard_moe_route(cfg, logits, idx, weight, bias=bias, m=m, load=load, workspace=ws)
    return idx, weight, m, load


def _spread(l):
    finite = torch.where(torch.isfinite(l) & (l.abs() < 1e30), l, torch.zeros_like(l))
    return 24 + 2 * finite.abs().amax(-1, keepdim=True)


def _check_forward(cfg, kw, logits, bias, out):
    idx, weight, m, load = out
    G, S, E, k = cfg.G, cfg.S, cfg.E, cfg.k
    score, renorm = kw.get("score", "softmax"), kw.get("renormalise", True)
    want = choose(logits.reshape(-1, E), bias, k=k, score=score, groups=kw.get("groups", 1),
                  groups_kept=kw.get("groups_kept", kw.get("groups", 1)), group_top=kw.get("group_top", 1)).cuda()
    assert torch.equal(idx.reshape(-1, k).long(), want)
    l = usable(logits).reshape(-1, E)
    w = route_weights(l, want, score, renorm, kw.get("scale", 1.0))
    rel = (_spread(l) + E / 8 + 16 + k) * 2 * U32
    within(weight.reshape(-1, k), w, rel * w.abs() + 1e-37, "weight")
    if m is not None:
        s = scores(l, score).reshape(G, S, E)
        bound = (rel.reshape(G, S, 1) * s).mean(1) + (S + 16) * U32 * s.mean(1) + 1e-37
        within(m, s.mean(1), bound, "m")
    if load is not None:
        flat = want.reshape(G, -1)
        count = torch.stack([torch.bincount(r[r >= 0], minlength=E) for r in flat])
        assert torch.equal(load.long(), count)


def _backward(cfg, logits, idx, dweight, dm):
    out = torch.full_like(logits, math.nan)
    B.gshard_moe_route_backward(cfg, logits, idx, dweight, out, dm=dm)
    return out


def _check_backward(cfg, kw, logits, idx, dweight, dm, got):
    """The formula's terms in 64 bits; every term's rounding counts with its absolute value."""
    G, S, E, k = cfg.G, cfg.S, cfg.E, cfg.k
    score, renorm, scale = kw.get("score", "softmax"), kw.get("renormalise", True), kw.get("scale", 1.0)
    l = usable(logits).reshape(-1, E)
    at = idx.reshape(-1, k).long()
    at = torch.where((at >= E) | (at < -1), torch.full_like(at, -1), at)
    gone = (at < 0) | (l.gather(-1, at.clamp(min=0)) == -math.inf)
    at = torch.where(gone, torch.full_like(at, -1), at)
    dw = dweight.reshape(-1, k).double().masked_fill(gone, 0.0)
    s = log_scores(l, score).exp()
    w = route_weights(l, at, score, renorm, scale)
    part = w * dw - (w * (w * dw).sum(-1, keepdim=True) / scale if renorm else 0)
    part_abs = (w * dw).abs() + (w.abs() * (w * dw).abs().sum(-1, keepdim=True) / abs(scale) if renorm else 0)
    dlog = torch.zeros_like(l).scatter_add_(-1, at.clamp(min=0), part.masked_fill(gone, 0.0))
    dlog_abs = torch.zeros_like(l).scatter_add_(-1, at.clamp(min=0), part_abs.masked_fill(gone, 0.0))
    if dm is not None:
        d = (dm.double() / S)[:, None, :].expand(G, S, E).reshape(-1, E)
        dlog, dlog_abs = dlog + s * d, dlog_abs + s * d.abs()
    if score == "softmax":
        want = dlog - s * dlog.sum(-1, keepdim=True)
        size = dlog_abs + s * dlog_abs.sum(-1, keepdim=True)
    else:
        want, size = dlog * torch.sigmoid(-l), dlog_abs * torch.sigmoid(-l)
    barred = l == -math.inf
    want, size = want.masked_fill(barred, 0.0), size.masked_fill(barred, 0.0)
    bound = (_spread(l) + E / 8 + 32 + k) * 4 * U32 * size + 1e-37
    half = HALF[logits.dtype]
    within(got.reshape(-1, E), want, bound + half * (want.abs() + bound), "dlogits")


CASES = [
    (1, 1, 2, 2, {}), (1, 1, 128, 2, {}), (1, 5, 1, 1, {}), (2, 33, 8, 2, dict(renormalise=False)),
    (3, 70, 17, 3, dict(scale=2.5)), (2, 129, 64, 8, dict(score="sigmoid")), (1, 200, 100, 10, dict(score="sigmoid", scale=0.5)),
    (2, 65, 256, 8, dict(score="sigmoid", groups=8, groups_kept=4, group_top=2, scale=2.5)),
    (1, 64, 96, 6, dict(groups=3, groups_kept=1)), (1, 90, 60, 4, dict(groups=5, groups_kept=2, group_top=2)),
    (2, 50, 160, 6, dict(groups=8, groups_kept=3, renormalise=False, scale=16.0)), (1, 40, 512, 2, dict(renormalise=False)),
    (2, 30, 513, 32, {}), (1, 40, 1024, 16, dict(score="sigmoid", groups=32, groups_kept=7, group_top=2)),
    (2, 40, 2048, 2, dict(renormalise=False)), (1, 12, 2046, 9, dict(groups=31, groups_kept=30)),
    (1, 9, 3000, 4, {}), (1, 5, 16384, 8, dict(score="sigmoid")), (1, 30, 32, 32, {}), (1, 30, 32, 32, dict(score="sigmoid")),
    (1, 20, 2046, 5, dict(groups=2, groups_kept=1)), (2, 9, 2044, 3, dict(groups=2, groups_kept=1, group_top=2)),
    (1, 30, 1022, 4, dict(score="sigmoid", groups=2, groups_kept=1)), (1, 33, 128, 6, dict(groups=16, groups_kept=5)),
    (1, 2400, 64, 4, dict(groups=8, groups_kept=3)), (1, 2400, 60, 3, dict(score="sigmoid", groups=4, groups_kept=2, group_top=2)),
    (1, 2500, 200, 7, dict(groups=2, groups_kept=1)), (1, 2370, 24, 5, dict(score="sigmoid")),
    (1, 700, 64, 1, {}), (4, 300, 32, 4, dict(groups=16, groups_kept=9, group_top=2)), (1, 50, 64, 5, dict(groups=32, groups_kept=16)),
]


@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("G,S,E,k,kw", CASES)
def test_against_the_definition(G, S, E, k, kw, dtype, with_bias, masked):
    cfg = B.make_route(G=G, S=S, E=E, k=k, dtype="bf16" if dtype == BF else "f32", **kw)
    logits = _logits(G, S, E, dtype, masked=masked)
    gen = torch.Generator(device="cuda").manual_seed(E + k)
    bias = 0.1 * torch.randn(E, generator=gen, device="cuda") if with_bias else None
    out = _route(cfg, logits, bias)
    _check_forward(cfg, kw, logits, bias, out)
    plain = _route(cfg, logits, bias, m=False, load=False)
    assert torch.equal(plain[0], out[0]) and torch.equal(plain[1], out[1])
    dweight = torch.randn(G, S, k, generator=gen, device="cuda")
    dm = torch.randn(G, E, generator=gen, device="cuda")
    for d in (None, dm):
        _check_backward(cfg, kw, logits, out[0], dweight, d, _backward(cfg, logits, out[0], dweight, d))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("kw", [{}, dict(score="sigmoid"), dict(score="sigmoid", groups=4, groups_kept=2, group_top=2)])
def test_equal_values_go_to_the_lowest_index(kw, dtype):
    """Few distinct logits, so that every boundary is a tie (also between +0 and -0)."""
    G, S, E, k = 1, 300, 64, 6
    gen = torch.Generator(device="cuda").manual_seed(2)
    logits = (torch.randint(-1, 2, (G, S, E), generator=gen, device="cuda").float() * 0.5)
    logits[..., ::3] *= -0.0
    logits = logits.to(dtype)
    for bias in (None, torch.zeros(E, device="cuda"), 0.25 * torch.randint(0, 2, (E,), generator=gen, device="cuda").float()):
        cfg = B.make_route(G=G, S=S, E=E, k=k, dtype="bf16" if dtype == BF else "f32", **kw)
        _check_forward(cfg, kw, logits, bias, _route(cfg, logits, bias))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_near_ties_are_decided_in_64_bits(score):
    """Scores plus bias that agree to fp32 rounding: adjacent logits (one step apart) under a bias far larger
    than the difference, so that fp32 sums are equal while the 64-bit ones are not."""
    G, S, E, k = 1, 257, 96, 8
    gen = torch.Generator(device="cuda").manual_seed(5)
    base = torch.randn(S, 1, generator=gen, device="cuda") * 0.3
    # steps 2^i - 1: no two pairs of them have the same sum, so that group sums have no 64-bit near ties
    steps = 2.0 ** torch.randint(0, 6, (S, E), generator=gen, device="cuda") - 1
    logits = (base + steps * 2.0 ** -23).reshape(G, S, E).contiguous()
    bias = torch.full((E,), 1.0, device="cuda")
    for kw in (dict(score=score), dict(score=score, groups=8, groups_kept=3, group_top=2)):
        cfg = B.make_route(G=G, S=S, E=E, k=k, **kw)
        _check_forward(cfg, kw, logits, bias, _route(cfg, logits, bias))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_scores_that_underflow_keep_their_weights(score):
    """Renormalised weights come from differences of logits, not from scores that have become 0."""
    logits = torch.randn(1, 64, 16, device="cuda") - 300.0
    logits[..., 0] = -299.0
    cfg = B.make_route(G=1, S=64, E=16, k=4, score=score)
    out = _route(cfg, logits)
    _check_forward(cfg, dict(score=score), logits, None, (*out[:2], None, out[3]))
    assert torch.allclose(out[1].sum(-1), torch.ones(1, 64, device="cuda"), atol=1e-6)
    # and with a wide spread, where the smaller ones are 0 in fp32
    wide = torch.arange(16, device="cuda").float().reshape(1, 1, 16) * 40 - 300
    cfg = B.make_route(G=1, S=1, E=16, k=4, score=score)
    _check_forward(cfg, dict(score=score), wide, None, (*_route(cfg, wide)[:2], None, None))


def test_bias_that_bars_and_bias_that_forces():
    logits = _logits(1, 100, 32, F32)
    bias = torch.zeros(32, device="cuda")
    bias[3], bias[7], bias[9] = -math.inf, math.nan, math.inf
    cfg = B.make_route(G=1, S=100, E=32, k=31)
    out = _route(cfg, logits, bias)
    assert (out[0][..., 0] == 9).all() and (out[0][..., -1] == -1).all()
    assert not ((out[0] == 3) | (out[0] == 7)).any()
    _check_forward(cfg, {}, logits, bias, out)


def test_no_tokens():
    for G, S in ((0, 5), (3, 0)):
        cfg = B.make_route(G=G, S=S, E=8, k=2)
        logits = torch.empty(G, S, 8, device="cuda")
        idx, weight, m, load = _route(cfg, logits)
        assert idx.numel() == 0 and (m == 0).all() and (load == 0).all()
        assert _backward(cfg, logits, idx, weight, m).numel() == 0


def test_foreign_indices_in_the_backward():
    """Out-of-range entries count as absent, a repeated expert gets both shares, barred experts none."""
    for kw in ({}, dict(renormalise=False), dict(score="sigmoid"), dict(score="sigmoid", renormalise=False)):
        cfg = B.make_route(G=2, S=40, E=24, k=5, **kw)
        logits = _logits(2, 40, 24, F32)
        logits[0, 0, 3] = -math.inf
        gen = torch.Generator(device="cuda").manual_seed(1)
        idx = torch.randint(-3, 27, (2, 40, 5), generator=gen, device="cuda", dtype=torch.int32)
        idx[0, 0] = torch.tensor([3, 3, 4, 4, 4], dtype=torch.int32)
        idx[1, 1] = torch.tensor([2 ** 31 - 1, -2 ** 31, 5, 5, -1], dtype=torch.int32)
        dweight = torch.randn(2, 40, 5, generator=gen, device="cuda")
        dm = torch.randn(2, 24, generator=gen, device="cuda")
        for d in (None, dm):
            _check_backward(cfg, kw, logits, idx, dweight, d, _backward(cfg, logits, idx, dweight, d))


@pytest.mark.parametrize("kw", [{}, dict(renormalise=False, scale=2.5), dict(score="sigmoid"),
                                dict(score="sigmoid", renormalise=False)])
def test_gradient_against_differences(kw):
    G, S, E, k = 2, 9, 20, 4
    cfg = B.make_route(G=G, S=S, E=E, k=k, **kw)
    logits = _logits(G, S, E, F32, seed=3)
    idx = _route(cfg, logits)[0]
    gen = torch.Generator(device="cuda").manual_seed(8)
    dweight = torch.randn(G, S, k, generator=gen, device="cuda")
    dm = torch.randn(G, E, generator=gen, device="cuda")
    grad = _backward(cfg, logits, idx, dweight, dm).double()
    at = idx.reshape(-1, k).long()
    for trial in range(4):
        d = torch.randn(G, S, E, generator=gen, device="cuda", dtype=torch.float64)

        def loss(h):
            l = (logits.double() + h * d).reshape(-1, E)
            w = route_weights(l, at, kw.get("score", "softmax"), kw.get("renormalise", True), kw.get("scale", 1.0))
            m = scores(l, kw.get("score", "softmax")).reshape(G, S, E).mean(1)
            return float((w * dweight.reshape(-1, k)).sum() + (m * dm).sum())

        want = (loss(1e-5) - loss(-1e-5)) / 2e-5
        assert float((grad * d).sum()) == pytest.approx(want, rel=1e-4, abs=1e-4)


def test_top2_agrees_with_the_gate_stage_and_feeds_capacity():
    """softmax, k = 2, raw weights: expert_idx, gate12 and m as gshard_moe_gate computes them."""
    G, S, M, E, C = 2, 256, 64, 32, 20
    shape = B.make_shape(G=G, S=S, M=M, H=64, E=E, C=C, dtype="f32")
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn(G, S, M, generator=gen, device="cuda")
    wg = torch.randn(M, E, generator=gen, device="cuda") * M ** -0.5
    ws = B.alloc_workspace(shape)
    e0 = torch.empty(G, S, 2, dtype=torch.int32, device="cuda")
    g0, m0 = torch.empty(G, S, 2, device="cuda"), torch.empty(G, E, device="cuda")
    B.gshard_moe_gate(shape, x, wg, e0, g0, m0, ws)
    logits = torch.empty(G * S, E, device="cuda")
    B.gshard_linear_forward(x.reshape(G * S, M), wg, logits,
                            workspace=torch.empty(B.gshard_linear_workspace_bytes(G * S, M, E, F32), dtype=torch.uint8, device="cuda"))
    cfg = B.make_route(G=G, S=S, E=E, k=2, renormalise=False)
    idx, g12, m, _ = _route(cfg, logits.reshape(G, S, E))
    assert torch.equal(idx, e0)
    torch.testing.assert_close(g12, g0, rtol=1e-5, atol=0)
    torch.testing.assert_close(m, m0, rtol=1e-5, atol=0)
    u = torch.rand(G, S, generator=gen, device="cuda")
    both = []
    for e, g, mm in ((e0, g0, m0), (idx, g12, m)):
        rt, rs = B.alloc_routing(shape)
        l_aux = torch.zeros(1, device="cuda")
        B.gshard_moe_capacity(shape, e, g, u, mm, rs, l_aux, ws)
        both.append((rt, l_aux))
    assert torch.equal(both[0][0]["slot"], both[1][0]["slot"])
    torch.testing.assert_close(both[0][1], both[1][1], rtol=1e-5, atol=0)


def test_same_bits_again_on_another_stream_and_in_a_graph():
    G, S, E, k = 4, 1000, 256, 8
    kw = dict(score="sigmoid", groups=8, groups_kept=4, group_top=2)
    cfg = B.make_route(G=G, S=S, E=E, k=k, **kw)
    logits, bias = _logits(G, S, E, F32), 0.1 * torch.randn(E, device="cuda")
    first = _route(cfg, logits, bias)
    dweight, dm = torch.randn(G, S, k, device="cuda"), torch.randn(G, E, device="cuda")
    grad = _backward(cfg, logits, first[0], dweight, dm)
    out = [torch.zeros_like(v) for v in (*first, grad)]
    ws = torch.empty(B.gshard_moe_route_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")

    def step():
        B.gshard_moe_route(cfg, logits, out[0], out[1], bias=bias, m=out[2], load=out[3], workspace=ws)
        B.gshard_moe_route_backward(cfg, logits, out[0], dweight, out[4], dm=dm)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    for got, want in zip(out, (*first, grad)):
        assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    logits.copy_(_logits(G, S, E, F32, seed=77))
    for _ in range(2):                                  # a second replay starts from the first one's counts
        graph.replay()
    _check_forward(cfg, kw, logits, bias, out[:4])
    _check_backward(cfg, kw, logits, out[0], dweight, dm, out[4])


def test_offsets_beyond_32_bits():
    """More than 2^31 logits: the last tokens are routed as they are alone."""
    E, S = 2048, 32768
    G = (1 << 31) // (E * S) + 1
    logits = torch.empty(G, S, E, dtype=BF, device="cuda")
    logits.normal_()
    cfg = B.make_route(G=G, S=S, E=E, k=2, dtype="bf16")
    idx, weight, m, load = _route(cfg, logits)
    tail = B.make_route(G=1, S=S, E=E, k=2, dtype="bf16")
    one = _route(tail, logits[-1:])
    assert torch.equal(idx[-1:], one[0]) and torch.equal(weight[-1:], one[1])
    assert torch.equal(m[-1:], one[2]) and torch.equal(load[-1:], one[3])
    out = torch.empty_like(logits)
    dw = torch.randn(G, S, 2, device="cuda")
    B.gshard_moe_route_backward(cfg, logits, idx, dw, out, dm=m)
    alone = torch.empty_like(logits[-1:])
    B.gshard_moe_route_backward(tail, logits[-1:], idx[-1:].contiguous(), dw[-1:].contiguous(), alone, dm=m[-1:].contiguous())
    assert torch.equal(out[-1:], alone)


def test_refusals():
    cfg = B.make_route(G=1, S=4, E=8, k=2)
    l = torch.zeros(1, 4, 8, device="cuda")
    idx, w = torch.zeros(1, 4, 2, dtype=torch.int32, device="cuda"), torch.zeros(1, 4, 2, device="cuda")
    for bad in (dict(logits=l.bfloat16()), dict(idx=idx.long()), dict(w=w[:, :2]), dict(bias=torch.zeros(7, device="cuda")),
                dict(logits=l.transpose(1, 2)), dict(m=torch.zeros(1, 8))):
        a = dict(logits=l, idx=idx, w=w, bias=None, m=None)
        a.update(bad)
        with pytest.raises(ValueError):
            B.gshard_moe_route(cfg, a["logits"], a["idx"], a["w"], bias=a["bias"], m=a["m"])
    with pytest.raises(B.GshardError) as e:                   # the mean scores need the workspace
        B.gshard_moe_route(cfg, l, idx, w, m=torch.zeros(1, 8, device="cuda"))
    assert e.value.code == B.GSHARD_ERR_INVALID_ARG
    with pytest.raises(B.GshardError):
        B.gshard_moe_route_backward(cfg, l, idx, w, l)


@pytest.mark.parametrize("kw", [{}, dict(groups=4, groups_kept=2), dict(score="sigmoid", groups=4, groups_kept=2, group_top=2)])
def test_infinity_and_the_largest_float_are_equal(kw):
    """+inf counts as the largest float, so the lower index wins between the two; NaN never does."""
    logits = _logits(1, 64, 32, F32, seed=21)
    logits[0, :, 5], logits[0, :, 9], logits[0, :, 2] = torch.finfo(torch.float32).max, math.inf, math.nan
    logits[0, ::2, 13] = math.inf
    for with_bias in (False, True):
        bias = torch.zeros(32, device="cuda") if with_bias else None
        cfg = B.make_route(G=1, S=64, E=32, k=3, **kw)
        out = _route(cfg, logits, bias)
        if kw.get("group_top", 1) == 1:                  # with sums a better pair may shut 5's group out
            assert (out[0][..., 0] == 5).all() and (out[0][..., 1] == 9).all()
        _check_forward(cfg, kw, logits, bias, out)
