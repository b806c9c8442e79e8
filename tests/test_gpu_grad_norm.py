"""The norm of many gradients and their clipping, against 64-bit sums.

Bounds.  16 bytes of squares are added in fp32 (at most 8 roundings of 2^-24 of their sum), everything else in fp64; the root halves
that, and its fp32 copy adds half a step.  A clipped gradient is one fp32 product with a factor rounded to fp32, rounded to
the tensor's type."""
import math

import pytest
import torch

from operator_reference import HALF, U32, within
from paper_2006_16668_b200 import binding as B

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def clip(grads, max_norm, outs=None):
    lst = B.make_grad_list(grads, outs)
    ws = torch.full((B.gshard_grad_norm_workspace_bytes(lst),), 255, dtype=torch.uint8, device="cuda")
    sumsq = torch.full((1,), math.nan, dtype=torch.float64, device="cuda")
    norm = torch.full((1,), math.nan, device="cuda")
    B.gshard_grad_norm(lst, sumsq, workspace=ws)
    B.gshard_grad_clip(lst, sumsq, max_norm, norm=norm)
    return float(sumsq), float(norm)


def check(grads, before, outs, max_norm, sumsq, norm):
    want = math.fsum(float(g.double().square().sum()) for g in before)
    assert abs(sumsq - want) <= 8 * U32 * want
    root = math.sqrt(want)
    assert abs(norm - root) <= 5 * U32 * root + 1e-45
    factor = max_norm / root if root > max_norm else 1.0
    for o, g in zip(outs, before):
        value = g.double() * factor
        bound = (8 * U32 * value.abs() + HALF[g.dtype] * value.abs()) if factor != 1.0 else torch.zeros_like(value)
        within(o, value, bound * 1.01 + (2.0 ** -133 if factor != 1.0 else 0), "clipped")


def tensors(counts, dtypes, seed=0, gap=0):
    """Parts of one buffer per type, one behind the other: at any alignment of their elements."""
    gen = torch.Generator(device="cuda").manual_seed(seed + sum(counts))
    out, buffers = [], {}
    for d in (BF, F32):
        total = sum(c + gap for c, t in zip(counts, dtypes) if t is d)
        buffers[d] = torch.randn(total + 1, generator=gen, device="cuda").to(d)
    at = {BF: 0, F32: 0}
    for c, d in zip(counts, dtypes):
        out.append(buffers[d][at[d]:at[d] + c])
        at[d] += c + gap
    return out, buffers


CASES = [([1], [F32]), ([7], [BF]), ([16384], [F32]), ([16385, 3], [BF, F32]), ([0, 5, 0, 40001], [F32, BF, BF, F32]),
         ([1000003, 17, 250000], [BF, BF, F32]), ([100] * 64, [F32] * 64), ([33] * 65, [BF, F32] * 32 + [BF]),
         ([5 + i % 90 for i in range(2100)], [BF, F32] * 1050), ([20000019], [BF])]


@pytest.mark.parametrize("max_norm", [0.25, 1e9])
@pytest.mark.parametrize("counts,dtypes", CASES)
def test_norm_and_clipping(counts, dtypes, max_norm):
    grads, buffers = tensors(counts, dtypes)
    before = [g.clone() for g in grads]
    outs = [torch.full_like(g, 7) for g in grads]
    first = clip(grads, max_norm, outs)
    check(grads, before, outs, max_norm, *first)
    assert all(torch.equal(g, b) for g, b in zip(grads, before))
    whole = {d: b.clone() for d, b in buffers.items()}
    assert clip(grads, max_norm) == first                       # in place, and the same bits
    assert all(torch.equal(g, o) for g, o in zip(grads, outs))
    # nothing around the tensors was touched
    assert all(torch.equal(buffers[d][-1:], whole[d][-1:]) for d in whole)


@pytest.mark.parametrize("shift_in", range(0, 5))
@pytest.mark.parametrize("shift_out", range(0, 9, 3))
def test_any_alignment_in_and_out(shift_in, shift_out):
    for dtype in (BF, F32):
        src = torch.randn(70000, device="cuda").to(dtype)
        dst = torch.full((70000,), 7.0, dtype=dtype, device="cuda")
        g, o = src[shift_in:shift_in + 50001], dst[shift_out:shift_out + 50001]
        check([g], [g.clone()], [o], 3.0, *clip([g], 3.0, [o]))
        assert (dst[:shift_out] == 7).all() and (dst[shift_out + 50001:] == 7).all()


@pytest.mark.parametrize("size", [1e-30, 1e-18, 1e18, 1e30])
def test_range_of_the_squares(size):
    g = [torch.randn(50000, device="cuda") * size, (torch.randn(3001, device="cuda") * size).to(BF)]
    before = [x.clone() for x in g]
    check(g, before, g, size, *clip(g, size))


def test_mixed_magnitudes_in_one_pack():
    g = torch.randn(4096, device="cuda")
    g[::4] *= 1e25
    g[1::4] *= 1e-25
    check([g], [g.clone()], [g], math.inf, *clip([g], math.inf))


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_norms_that_are_no_numbers_leave_the_gradients(bad):
    g = [torch.randn(5000, device="cuda"), torch.randn(70, device="cuda").to(BF)]
    g[1][33] = bad
    before = [x.clone() for x in g]
    outs = [torch.zeros_like(x) for x in g]
    sumsq, norm = clip(g, 1.0, outs)
    assert not math.isfinite(norm) and (math.isnan(norm) == math.isnan(bad))
    for o, b in zip(outs, before):
        assert torch.equal(o.view(torch.int16 if o.dtype is BF else torch.int32), b.view(torch.int16 if b.dtype is BF else torch.int32))


def test_zero_gradients_zero_bound_and_no_tensors():
    g = [torch.zeros(100, device="cuda")]
    assert clip(g, 1.0) == (0.0, 0.0)
    h = [torch.ones(100, device="cuda")]
    assert clip(h, 0.0)[1] == 10.0 and not h[0].any()
    assert clip([], 1.0) == (0.0, 0.0)


def test_capture():
    grads, _ = tensors([5000, 123, 70001], [BF, F32, F32])
    outs = [torch.empty_like(g) for g in grads]
    want = clip(grads, 1.0, outs)
    kept = [o.clone() for o in outs]
    lst = B.make_grad_list(grads, outs)
    ws = torch.empty(B.gshard_grad_norm_workspace_bytes(lst), dtype=torch.uint8, device="cuda")
    sumsq, norm = torch.empty(1, dtype=torch.float64, device="cuda"), torch.empty(1, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.gshard_grad_norm(lst, sumsq, workspace=ws)
        B.gshard_grad_clip(lst, sumsq, 1.0, norm=norm)
    for scale in (1.0, 2.0):
        for g in grads:
            g *= scale
        graph.replay()
        torch.cuda.synchronize()
        assert float(sumsq) == want[0] * scale ** 2 and float(norm) == want[1] * scale
        if scale == 1.0:
            assert all(torch.equal(o, k) for o, k in zip(outs, kept))
