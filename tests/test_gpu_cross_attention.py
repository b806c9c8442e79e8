"""Cross attention, forward and backward, against the formula in 64 bits; the bounds are derived in decoder_reference."""
import math

import pytest
import torch

import decoder_reference as ref
from operator_reference import within
from paper_2006_16668_b200 import binding as B

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
NAN = float("nan")


def make(Bn, Tq, Tk, H, Hkv, D, dtype, lengths=None, fused=False, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(Bn + 3 * Tq + 7 * Tk + 11 * H + 13 * D + seed)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(dtype)
    t = {"q": r(Bn, Tq, H, D), "dout": r(Bn, Tq, H, D)}
    if fused:
        kv = r(Bn, Tk, 2, Hkv, D)
        t["k"], t["v"] = kv[:, :, 0], kv[:, :, 1]
    else:
        t["k"], t["v"] = r(Bn, Tk, Hkv, D), r(Bn, Tk, Hkv, D)
    t["lengths"] = torch.full((Bn,), Tk, dtype=torch.int32, device="cuda") if lengths is None else \
        torch.tensor(lengths, dtype=torch.int32, device="cuda")
    t["given"] = lengths is not None
    # what lies behind a source's length is not to be looked at
    for b in range(Bn):
        n = max(0, min(int(t["lengths"][b]), Tk))
        t["k"][b, n:], t["v"][b, n:] = NAN, math.inf
    return t


def workspace(t, back):
    (Bn, Tq, H, D), (Tk, Hkv) = t["q"].shape, t["k"].shape[1:3]
    need = B.gshard_cross_attention_workspace_bytes(Bn, Tq, Tk, H, Hkv, D, t["q"].dtype, for_backward=back)
    assert need >= 256
    return torch.empty(need, dtype=torch.uint8, device="cuda")


def forward(t, lse=True, scale=None, stream=None):
    Bn, Tq, H, D = t["q"].shape
    o = torch.full((Bn, Tq, H, D), NAN, dtype=t["q"].dtype, device="cuda")
    kept = torch.full((Bn, H, Tq), NAN, device="cuda") if lse else None
    ws = workspace(t, False)
    B.gshard_cross_attention_forward(t["q"], t["k"], t["v"], o, lse=kept, k_lengths=t["lengths"] if t["given"] else None, scale=scale,
                                     workspace=ws, stream=stream)
    if o.numel():
        assert B.gshard_moe_last_device_status(ws) == B.GSHARD_OK
    return o, kept


def backward(t, o, lse, scale=None):
    grads = []
    for x in (t["q"], t["k"], t["v"]):
        whole = torch.full((x.untyped_storage().nbytes() // x.element_size(),), NAN, dtype=x.dtype, device="cuda")
        grads.append(whole.as_strided(x.shape, x.stride(), x.storage_offset()))
    ws = workspace(t, True)
    B.gshard_cross_attention_backward(t["q"], t["k"], t["v"], o, lse, t["dout"], *grads, k_lengths=t["lengths"] if t["given"] else None,
                                      scale=scale, workspace=ws)
    assert B.gshard_moe_last_device_status(ws) == B.GSHARD_OK
    return grads


def lengths_of(t):
    return t["lengths"].clamp(0, t["k"].shape[1])


def check_forward(t, o, lse, scale=None):
    scale = t["q"].shape[-1] ** -0.5 if scale is None else scale
    (want, bound), (want_lse, lse_bound) = ref.attention(t["q"], t["k"], t["v"], lengths_of(t), scale)
    within(o, want, bound, "o")
    if lse is not None:
        empty = torch.isinf(want_lse)
        assert torch.equal(lse == -math.inf, empty)
        within(lse.masked_fill(empty, 0), want_lse.masked_fill(empty, 0), lse_bound, "lse")


def check_backward(t, o, lse, grads, scale=None):
    scale = t["q"].shape[-1] ** -0.5 if scale is None else scale
    want = ref.attention_grad(t["q"], t["k"], t["v"], lengths_of(t), scale, o, lse, t["dout"])
    for got, (value, bound), name in zip(grads, want, ("dq", "dk", "dv")):
        within(got, value, bound, name)
    for b, n in enumerate(lengths_of(t).tolist()):
        assert not grads[1][b, n:].any() and not grads[2][b, n:].any()


SIZES = [  # B, Tq, Tk, H, Hkv, D, lengths, k and v in one buffer
    (1, 1, 1, 1, 1, 64, None, False),
    (1, 1, 200, 16, 16, 128, None, False),
    (3, 1, 77, 8, 2, 128, [77, 1, 0], True),
    (2, 5, 130, 4, 4, 64, [129, 128], False),
    (2, 16, 500, 4, 1, 128, [500, 3], True),
    (1, 17, 129, 2, 2, 40, None, False),
    (2, 64, 64, 2, 1, 8, [64, 63], False),
    (2, 100, 127, 4, 2, 96, [65, 127], True),
    (1, 127, 256, 2, 2, 120, [255], False),
    (3, 128, 128, 4, 4, 128, [128, 0, 127], False),
    (2, 129, 300, 4, 1, 128, [300, 257], True),
    (1, 256, 384, 2, 2, 64, [383], False),
    (2, 300, 513, 6, 3, 128, [513, 400], False),
    (2, 257, 1, 2, 2, 128, [1, 0], True),
    (1, 520, 1025, 2, 2, 72, None, True),
    (2, 700, 650, 4, 2, 64, [-5, 9000], False),
    # groups of heads that share a tile, and some that do not fit one
    (2, 37, 300, 32, 1, 64, [300, 17], True),
    (2, 70, 260, 8, 1, 128, [259, 128], False),
    (1, 50, 200, 12, 2, 72, [131], False),
    (1, 3, 400, 64, 1, 64, None, False),
    # few rows and a long source: parts of it, some of them empty
    (1, 9, 1024, 1, 1, 128, None, False),
    (2, 20, 5000, 2, 1, 64, [4999, 700], True),
    (3, 13, 2500, 4, 2, 128, [2500, 0, 513], True),
    (1, 300, 4100, 1, 1, 40, [3000], False),
    # few keys and many rows: parts of the queries
    (1, 1500, 100, 8, 1, 128, [99], False),
    (2, 1300, 300, 4, 2, 64, [300, 100], True),
    (3, 900, 260, 6, 1, 40, [0, 130, 257], False),
]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("size", SIZES)
def test_against_the_formula(size, dtype):
    Bn, Tq, Tk, H, Hkv, D, lengths, fused = size
    t = make(Bn, Tq, Tk, H, Hkv, D, dtype, lengths, fused)
    o, lse = forward(t)
    check_forward(t, o, lse)
    only, none = forward(t, lse=False)
    assert torch.equal(only, o)
    check_backward(t, o, lse, backward(t, o, lse))


@pytest.mark.parametrize("Tq", [9, 100, 130, 300])
def test_many_short_ragged_sources(Tq):
    """More sources than multiprocessors, each of one block or two that end inside 16 keys: whatever a kernel does for the last keys of
    a source it does many times in a row."""
    lengths = [(37 * i) % 200 for i in range(160)]
    t = make(160, Tq, 200, 4, 2, 64, BF, lengths)
    o, lse = forward(t)
    check_forward(t, o, lse)
    check_backward(t, o, lse, backward(t, o, lse))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Tq", [150, 1300])
def test_nothing_between_or_behind_the_rows_is_written(Tq, dtype):
    t = make(2, Tq, 140, 4, 2, 64, dtype, [100, 140], fused=True)
    o, lse = forward(t)
    whole = torch.full((2, 140, 3, 2, 64), 7.0, dtype=dtype, device="cuda")
    wide = lambda x: torch.stack((x, x, x), 2)
    k, v = wide(t["k"])[:, :, 1], wide(t["v"])[:, :, 1]
    dq = torch.empty_like(t["q"])
    rest = torch.full((2, 140, 3, 2, 64), 7.0, dtype=dtype, device="cuda")
    B.gshard_cross_attention_backward(t["q"], k, v, o, lse, t["dout"], dq, whole[:, :, 1], rest[:, :, 2], k_lengths=t["lengths"],
                                      workspace=workspace(t, True))
    assert (whole[:, :, 0] == 7).all() and (whole[:, :, 2] == 7).all() and (rest[:, :, :2] == 7).all()
    check_backward(t, o, lse, (dq, whole[:, :, 1], rest[:, :, 2]))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Tq", [1, 200])
def test_large_scores_and_scales(Tq, dtype):
    """Rows that attend to a single key, scores of some hundreds of either sign, and a scale of one."""
    t = make(2, Tq, 333, 4, 2, 64, dtype, [333, 200])
    t["q"] *= 8
    for scale in (1.0, 0.02):
        o, lse = forward(t, scale=scale)
        check_forward(t, o, lse, scale)
        check_backward(t, o, lse, backward(t, o, lse, scale), scale)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Tq", [1, 140])
def test_rising_and_falling_maxima(Tq, dtype):
    """The running maximum grows in every tile of keys, or is reached by the first."""
    for sign in (1.0, -1.0):
        t = make(1, Tq, 900, 2, 2, 64, dtype)
        t["q"][:] = 0.5
        t["k"] *= 0.25
        t["k"] += (sign * torch.linspace(-1.5, 1.5, 900, device="cuda")[None, :, None, None]).to(dtype)
        o, lse = forward(t)
        check_forward(t, o, lse)
        check_backward(t, o, lse, backward(t, o, lse))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("Tq,Tk", [(0, 5), (5, 0), (0, 0)])
def test_no_queries_or_no_keys(Tq, Tk, dtype):
    t = make(2, Tq, Tk, 4, 2, 64, dtype)
    o, lse = forward(t)
    assert not o.any() and (lse == -math.inf).all()
    if Tq or Tk:
        assert not any(g.any() for g in backward(t, o, lse))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_gradient_against_differences(dtype):
    """d<dout, o> along a direction of q, k and v together, by central differences of the 64-bit forward."""
    t = make(2, 9, 33, 4, 2, 64, dtype, [33, 20])
    for x in (t["k"], t["v"]):
        x[1, 20:] = 0
    o, lse = forward(t)
    grads = backward(t, o, lse)
    gen = torch.Generator(device="cuda").manual_seed(5)
    step = [torch.randn(x.shape, generator=gen, device="cuda", dtype=torch.float64) for x in (t["q"], t["k"], t["v"])]
    value = lambda e: (ref.attention(*[x.double() + e * s for x, s in zip((t["q"], t["k"], t["v"]), step)], t["lengths"], 0.125)[0][0]
                       * t["dout"].double()).sum()
    want = (value(1e-5) - value(-1e-5)) / 2e-5
    got = sum((g.double() * s).sum() for g, s in zip(grads, step))
    size = sum((g.double() * s).square().sum() for g, s in zip(grads, step)).sqrt()
    # the terms' roundings are independent: the sum is off by some of them times the root of the sum of squares; bf16 rounds
    # P or dS, o (through delta) and the gradient itself
    assert abs(got - want) < (6 * 2.0 ** -8 if dtype == BF else 2.0 ** -16) * size


def test_capture_and_a_second_stream():
    t = make(2, 200, 300, 4, 2, 128, BF, [300, 111])
    few = make(4, 1, 300, 4, 2, 128, BF, [300, 111, 0, 7])
    want, want_lse = forward(t)
    want_few, _ = forward(few)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o, lse = forward(t, stream=side)
    side.synchronize()
    assert torch.equal(o, want) and torch.equal(lse, want_lse)
    grads = backward(t, want, want_lse)
    ws, wf, wb = workspace(t, False), workspace(few, False), workspace(t, True)
    o, lse, of = torch.empty_like(want), torch.empty_like(want_lse), torch.empty_like(want_few)
    again = [torch.empty_like(g) for g in grads]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.gshard_cross_attention_forward(t["q"], t["k"], t["v"], o, lse=lse, k_lengths=t["lengths"], workspace=ws)
        B.gshard_cross_attention_forward(few["q"], few["k"], few["v"], of, k_lengths=few["lengths"], workspace=wf)
        B.gshard_cross_attention_backward(t["q"], t["k"], t["v"], o, lse, t["dout"], *again, k_lengths=t["lengths"], workspace=wb)
    for _ in range(2):
        o.fill_(NAN); lse.fill_(NAN); of.fill_(NAN)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want) and torch.equal(lse, want_lse) and torch.equal(of, want_few)
        assert all(torch.equal(a, g) for a, g in zip(again, grads))
    t["lengths"][0] = 40                              # a replay reads the lengths of its time
    graph.replay()
    torch.cuda.synchronize()
    t["k"][0, 40:], t["v"][0, 40:] = NAN, NAN
    check_forward(t, o, lse)


def test_keys_beyond_31_bits():
    """A cache whose last source starts beyond 2^31 elements."""
    Bn, Tk, H, D = 3, 8192, 2, 128
    stride = 100 * 1024                               # of a token: 3 x 8192 x 102400 = 2.5e9 elements, 5 GB
    buf = torch.empty(Bn * Tk * stride, dtype=BF, device="cuda")
    kv = buf.as_strided((Bn, Tk, 2, H, D), (Tk * stride, stride, H * D, D, 1))
    gen = torch.Generator(device="cuda").manual_seed(1)
    kv.copy_(torch.randn(Bn, Tk, 2, H, D, generator=gen, device="cuda"))
    for Tq in (1, 40):
        t = {"q": torch.randn(Bn, Tq, H, D, generator=gen, device="cuda").to(BF), "k": kv[:, :, 0], "v": kv[:, :, 1], "given": True,
             "lengths": torch.tensor([Tk, 5000, Tk - 1], dtype=torch.int32, device="cuda")}
        o, lse = forward(t)
        check_forward(t, o, lse)
