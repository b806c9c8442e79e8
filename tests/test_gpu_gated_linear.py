"""The gated linear operator, forward and backward, against the formula in 64 bits; bounds in decoder_reference."""
import pytest
import torch

import decoder_reference as ref
from operator_reference import within
from paper_2006_16668_b200 import binding as B

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
NAN = float("nan")


def make(n, K, cols, dtype, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(n * 31 + K * 7 + cols + seed)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    return {"x": r(n, K).to(dtype), "w": (r(K, 2 * cols) * K ** -0.5).to(dtype), "pre": (1.5 * r(n, 2 * cols)).to(dtype),
            "dh": r(n, cols).to(dtype)}


def workspace(t, back):
    (n, K), cols = t["x"].shape, t["dh"].shape[1]
    need = B.gshard_gated_linear_workspace_bytes(n, K, cols, t["x"].dtype, for_backward=back)
    assert need > 0
    return torch.empty(need, dtype=torch.uint8, device="cuda")


def forward(t, act, pre=True):
    h = torch.full_like(t["dh"], NAN)
    kept = torch.full_like(t["pre"], NAN) if pre else None
    ws = workspace(t, False)
    B.gshard_gated_linear_forward(t["x"], t["w"], h, pre=kept, activation=act, workspace=ws)
    assert B.gshard_moe_last_device_status(ws) == B.GSHARD_OK
    return h, kept


def backward(t, act, dx=True, dw=True):
    gx, gw = torch.full_like(t["x"], NAN) if dx else None, torch.full_like(t["w"], NAN) if dw else None
    ws = workspace(t, True)
    B.gshard_gated_linear_backward(t["x"], t["w"], t["pre"], t["dh"], gx, gw, activation=act, workspace=ws)
    if t["x"].shape[0]:
        assert B.gshard_moe_last_device_status(ws) == B.GSHARD_OK
    return gx, gw


def check(t, act, h, kept, gx, gw):
    (want, bound), (want_pre, pre_bound) = ref.gated(t["x"], t["w"], act)
    within(h, want, bound, "h")
    if kept is not None:
        within(kept, want_pre, pre_bound, "pre")
    for got, (value, bound), name in zip((gx, gw), ref.gated_grad(t["x"], t["w"], t["pre"], t["dh"], act), ("dx", "dw")):
        if got is not None:
            within(got, value, bound, name)


SIZES = [(1, 8, 8), (1, 1024, 4096), (2, 136, 72), (3, 16, 24), (8, 2048, 96), (9, 72, 40), (33, 200, 264), (64, 1024, 512),
         (127, 136, 328), (128, 256, 128), (129, 264, 136), (200, 8, 1024), (257, 1032, 264), (300, 4096, 128), (1000, 520, 1000),
         (2050, 256, 768), (5000, 128, 1544)]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,K,cols", SIZES)
def test_against_the_formula(n, K, cols, dtype):
    t = make(n, K, cols, dtype)
    act = ACTS[(n + K // 8 + cols // 8) % 5]
    h, kept = forward(t, act)
    check(t, act, h, kept, *backward(t, act))
    alone, _ = forward(t, act, pre=False)
    assert torch.equal(alone, h)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("n", [1, 6, 300, 3000])
def test_every_activation_and_output(n, act, dtype):
    t = make(n, 136, 648, dtype)
    h, kept = forward(t, act)
    gx, gw = backward(t, act)
    check(t, act, h, kept, gx, gw)
    assert torch.equal(backward(t, act, dw=False)[0], gx) and torch.equal(backward(t, act, dx=False)[1], gw)


def test_no_rows():
    t = make(0, 64, 64, BF)
    B.gshard_gated_linear_forward(t["x"], t["w"], t["dh"], workspace=workspace(make(1, 64, 64, BF), False))
    assert not backward(t, "silu")[1].any()


@pytest.mark.parametrize("act", ACTS)
def test_far_projections(act):
    """Gates of some hundreds of either sign: no overflow on the way turns into NaN, the far left is zero."""
    t = make(300, 64, 64, BF)
    t["w"][:, :64] *= 200
    t["pre"][:, :64] *= 200
    h, kept = forward(t, act)
    gx, gw = backward(t, act)
    for x in (h, kept, gx, gw):
        assert torch.isfinite(x).all()
    check(t, act, h, kept, gx, gw)


@pytest.mark.parametrize("n", [1, 40, 3000])
def test_capture(n):
    t = make(n, 264, 520, BF)
    h, kept = forward(t, "silu")
    gx, gw = backward(t, "silu")
    out = [torch.empty_like(x) for x in (h, kept, gx, gw)]
    wf, wb = workspace(t, False), workspace(t, True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.gshard_gated_linear_forward(t["x"], t["w"], out[0], pre=out[1], activation="silu", workspace=wf)
        B.gshard_gated_linear_backward(t["x"], t["w"], t["pre"], t["dh"], out[2], out[3], activation="silu", workspace=wb)
    for _ in range(2):
        for x in out:
            x.fill_(NAN)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, (h, kept, gx, gw)))
