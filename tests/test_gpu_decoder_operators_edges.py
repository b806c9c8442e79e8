"""Calls of cross attention, gated linear and gradient clipping at the edges of what they take: queries within wider rows, very many
sources or heads, sizes beyond 31 bits, two streams at once, a captured call whose lengths change.  Bounds in decoder_reference."""
import math

import pytest
import torch

import decoder_reference as ref
import test_gpu_cross_attention as attn
from operator_reference import HALF, U32, within
from paper_2006_16668_b200 import binding as B

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
NAN = float("nan")


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("size", [(3, 1, 200, 8, 8, 128, [200, 0, 3]), (2, 70, 300, 4, 2, 64, [300, 31]), (1, 40, 3000, 2, 1, 128, [2900]),
                                  (2, 1300, 100, 4, 2, 64, [100, 60])])
def test_queries_within_wider_rows(size, dtype):
    Bn, Tq, Tk, H, Hkv, D, lengths = size
    t = attn.make(Bn, Tq, Tk, H, Hkv, D, dtype, lengths)
    wide = torch.stack((t["q"], t["q"], t["q"]), 2)
    t["q"] = wide[:, :, 1]
    o, lse = attn.forward(t)
    attn.check_forward(t, o, lse)
    whole = torch.full_like(wide, 7.0)
    dq, dk, dv = whole[:, :, 1], torch.full_like(t["k"], NAN), torch.full_like(t["v"], NAN)
    ws = attn.workspace(t, True)
    B.gshard_cross_attention_backward(t["q"], t["k"], t["v"], o, lse, t["dout"], dq, dk, dv, k_lengths=t["lengths"], workspace=ws)
    assert B.gshard_moe_last_device_status(ws) == B.GSHARD_OK
    assert (whole[:, :, 0] == 7).all() and (whole[:, :, 2] == 7).all()
    attn.check_backward(t, o, lse, (dq, dk, dv))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("size", [(70000, 1, 3, 2, 1, 8), (70000, 9, 2, 1, 1, 8), (1, 1, 70, 160, 1, 64), (1, 3, 70, 160, 160, 16), (2, 2, 9, 96, 2, 24)])
def test_very_many_sources_or_heads(size, dtype):
    Bn, Tk = size[0], size[2]
    t = attn.make(*size, dtype)
    t["given"], t["lengths"] = True, (torch.arange(Bn, device="cuda") % (Tk + 1)).to(torch.int32)
    for x in (t["k"], t["v"]):
        x.masked_fill_((torch.arange(Tk, device="cuda") >= t["lengths"][:, None])[:, :, None, None], NAN)
    o, lse = attn.forward(t)
    scale = size[5] ** -0.5
    (want, bound), (want_lse, lse_bound) = ref.attention(t["q"], t["k"], t["v"], t["lengths"], scale)
    within(o, want, bound, "o")
    empty = torch.isinf(want_lse)
    assert torch.equal(lse == -math.inf, empty)
    within(lse.masked_fill(empty, 0), want_lse.masked_fill(empty, 0), lse_bound, "lse")
    grads = attn.backward(t, o, lse)
    for got, (value, bound), name in zip(grads, ref.attention_grad(t["q"], t["k"], t["v"], t["lengths"], scale, o, lse, t["dout"]), ("dq", "dk", "dv")):
        within(got, value, bound, name)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("size", [(2, 40, 3000, 2, 1, 64), (2, 1300, 200, 4, 1, 128)])
def test_replay_with_other_lengths_and_parts(size, dtype):
    t = attn.make(*size, dtype, [size[2], size[2] // 2])
    for x in (t["k"], t["v"]):
        x.nan_to_num_(nan=0.5, posinf=0.5)               # every key may come to be used
    o, lse = torch.empty_like(t["q"]), torch.empty(size[0], size[3], size[1], device="cuda")
    grads = [torch.empty_like(t[n]) for n in "qkv"]
    wf, wb = attn.workspace(t, False), attn.workspace(t, True)

    def call():
        B.gshard_cross_attention_forward(t["q"], t["k"], t["v"], o, lse=lse, k_lengths=t["lengths"], workspace=wf)
        B.gshard_cross_attention_backward(t["q"], t["k"], t["v"], o, lse, t["dout"], *grads, k_lengths=t["lengths"], workspace=wb)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for lengths in ([1, size[2]], [size[2] - 1, 0], [130, 129]):
        t["lengths"].copy_(torch.tensor(lengths, dtype=torch.int32))
        for x in (o, lse, *grads):
            x.fill_(NAN)
        graph.replay()
        torch.cuda.synchronize()
        attn.check_forward(t, o, lse)
        attn.check_backward(t, o, lse, grads)


def test_two_streams_at_once():
    """Calls that have their own workspaces and outputs do not know of one another."""
    calls = [attn.make(2, 300, 700, 4, 2, 128, BF, [700, 333]), attn.make(2, 1300, 200, 4, 1, 64, BF, [200, 77])]
    alone = []
    for t in calls:
        o, lse = attn.forward(t)
        alone.append((o, lse, *attn.backward(t, o, lse)))
    streams = [torch.cuda.Stream() for _ in calls]
    torch.cuda.synchronize()
    got = []
    for t, s in zip(calls, streams):
        with torch.cuda.stream(s):
            outs = [torch.empty_like(x) for x in alone[len(got)]]
            got.append((outs, attn.workspace(t, False), attn.workspace(t, True)))
    torch.cuda.synchronize()
    for _ in range(5):
        for t, s, (x, wf, wb) in zip(calls, streams, got):
            B.gshard_cross_attention_forward(t["q"], t["k"], t["v"], x[0], lse=x[1], k_lengths=t["lengths"], workspace=wf, stream=s)
            B.gshard_cross_attention_backward(t["q"], t["k"], t["v"], x[0], x[1], t["dout"], *x[2:], k_lengths=t["lengths"], workspace=wb, stream=s)
    torch.cuda.synchronize()
    for (x, _, _), want in zip(got, alone):
        assert all(torch.equal(a, b) for a, b in zip(x, want))


def test_gated_rows_beyond_31_bits():
    n, K, cols = 140000, 64, 8192                         # pre: 2.3e9 elements
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(n, K, generator=gen, device="cuda").to(BF)
    w = (torch.randn(K, 2 * cols, generator=gen, device="cuda") / 8).to(BF)
    h, pre = torch.empty(n, cols, dtype=BF, device="cuda"), torch.empty(n, 2 * cols, dtype=BF, device="cuda")
    ws = torch.empty(B.gshard_gated_linear_workspace_bytes(n, K, cols, BF), dtype=torch.uint8, device="cuda")
    B.gshard_gated_linear_forward(x, w, h, pre=pre, activation="silu", workspace=ws)
    for rows in (slice(0, 40), slice(n - 40, n)):
        (want, bound), (want_pre, pre_bound) = ref.gated(x[rows], w, "silu")
        within(h[rows], want, bound, "h")
        within(pre[rows], want_pre, pre_bound, "pre")
    dx, dw = torch.full_like(x, NAN), torch.full_like(w, NAN)
    back = torch.empty(B.gshard_gated_linear_workspace_bytes(n, K, cols, BF, for_backward=True), dtype=torch.uint8, device="cuda")
    B.gshard_gated_linear_backward(x, w, pre, h, dx, dw, activation="silu", workspace=back)      # dh: anything of its shape
    assert B.gshard_moe_last_device_status(back) == B.GSHARD_OK and torch.isfinite(dw).all()
    rows = slice(n - 40, n)
    value, bound = ref.gated_grad(x[rows], w, pre[rows], h[rows], "silu")[0]
    within(dx[rows], value, bound, "dx")


def test_a_gradient_beyond_31_bits():
    count = 2 ** 31 + 11
    g = torch.zeros(count, dtype=BF, device="cuda")
    places = torch.tensor([0, 5, 2 ** 31 - 1, 2 ** 31, 2 ** 31 + 10], device="cuda")
    values = torch.tensor([3.0, -4.0, 12.0, 84.0, 13.0], device="cuda").to(BF)
    g[places] = values
    small = torch.full((3,), 2.0, device="cuda")
    grads = B.make_grad_list([small, g])
    ws = torch.empty(B.gshard_grad_norm_workspace_bytes(grads), dtype=torch.uint8, device="cuda")
    sumsq, norm = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(1, device="cuda")
    B.gshard_grad_norm(grads, sumsq, workspace=ws)
    want = 9 + 16 + 144 + 84 ** 2 + 169 + 12
    assert float(sumsq) == want                           # integers
    B.gshard_grad_clip(grads, sumsq, 1.0, norm=norm)
    assert abs(float(norm) - want ** 0.5) <= U32 * want ** 0.5
    scaled = values.double() / want ** 0.5
    within(g[places], scaled, (HALF[BF] + 4 * U32) * scaled.abs(), "clipped")
    assert int((g != 0).sum()) == len(places)
