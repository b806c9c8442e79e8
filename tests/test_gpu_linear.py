"""The linear operator, forward and backward, against the formula in 64 bits.

Bounds.  The tensor core adds 16 products per step to an fp32 accumulator, so a product over K carries K/16
roundings (plus a few of the joins and the epilogue) of at most 2^-23 of the absolute sum S = |x| |w|; the
CUDA-core path K roundings of 2^-24.  An activation is a handful of fp32 operations on a value that is off
by that much, times its slope (at most 1.13).  Outputs add half a step of their type.  In bf16 dpre is rounded
once, half a step (2^-8) of each of its entries, before both gradient products."""
import itertools

import pytest
import torch

from operator_reference import HALF, U32, activation, slope, within
from paper_2006_16668_b200 import binding as B

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def _make(n, K, cols, dtype, out_dtype=None, seed=0):
    out_dtype = out_dtype or dtype
    gen = torch.Generator(device="cuda").manual_seed(n * 31 + K * 7 + cols + seed)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    return {"x": r(n, K).to(dtype), "w": (r(K, cols) * K ** -0.5).to(dtype), "bias": 0.3 * r(cols),
            "residual": r(n, cols).to(out_dtype), "pre": (1.5 * r(n, cols)).to(out_dtype), "dy": r(n, cols).to(out_dtype)}


def _ws(t, back):
    n, K = t["x"].shape
    need = B.gshard_linear_workspace_bytes(n, K, t["w"].shape[1], t["x"].dtype, t["dy"].dtype, for_backward=back)
    assert need > 0
    return torch.empty(need, dtype=torch.uint8, device="cuda")


def _forward(t, act="none", bias=True, residual=False, pre=False, y=None):
    y = torch.full_like(t["dy"], float("nan")) if y is None else y
    kept = torch.full_like(t["dy"], float("nan")) if pre else None
    ws = _ws(t, False)
    B.gshard_linear_forward(t["x"], t["w"], y, bias=t["bias"] if bias else None, residual=t["residual"] if residual else None,
                            pre=kept, activation=act, workspace=ws)
    assert B.gshard_moe_last_device_status(ws) == B.GSHARD_OK
    return y, kept


def _steps(t, K):
    return (K / 16 + 16) * 2 * U32 if t["x"].dtype == BF else (K + 16) * U32


def _check_forward(t, y, kept, act, bias=True, residual=False):
    x, w = t["x"].double(), t["w"].double()
    want_pre = x @ w + (t["bias"].double() if bias else 0)
    bound = _steps(t, x.shape[1]) * (x.abs() @ w.abs() + (t["bias"].double().abs() if bias else 0)) + 1e-30
    half = HALF[t["dy"].dtype]
    if kept is not None:
        within(kept, want_pre, bound + half * (want_pre.abs() + bound), "pre")
    want = activation(want_pre, act)
    bound = 1.2 * bound + (0 if act in ("none", "relu") else 24 * U32 * (want_pre.abs() + 1))
    if residual:
        want = want + t["residual"].double()
        bound = bound + 2 * U32 * t["residual"].double().abs()
    within(y, want, bound + half * (want.abs() + bound), "y")


def _backward(t, act="none", dx=True, dw=True, db=True):
    n, K = t["x"].shape
    cols = t["w"].shape[1]
    nan = float("nan")
    gx = torch.full_like(t["x"], nan) if dx else None
    gw = torch.full_like(t["w"], nan) if dw else None
    gb = torch.full((cols,), nan, device="cuda") if db else None
    ws = _ws(t, True)
    B.gshard_linear_backward(t["x"], t["w"], t["dy"], gx, gw, gb, pre=None if act == "none" else t["pre"], activation=act,
                             workspace=ws)
    if n:
        assert B.gshard_moe_last_device_status(ws) == B.GSHARD_OK
    return gx, gw, gb


def _check_backward(t, act, gx, gw, gb):
    x, w, dy = t["x"].double(), t["w"].double(), t["dy"].double()
    n, K = x.shape
    cols = w.shape[1]
    s = slope(t["pre"].double(), act)
    dpre = dy * s
    off = dy.abs() * 24 * U32 * (0 if act in ("none", "relu") else (1 + t["pre"].double().abs()))    # of the slope
    rounded = t["x"].dtype == BF and (act != "none" or t["dy"].dtype == F32)
    slack = off + (HALF[BF] * (dpre.abs() + off) if rounded else 0)
    half = HALF[t["x"].dtype]
    for got, want, terms, slack_terms, depth, name in (
            (gx, dpre @ w.t(), dpre.abs() @ w.abs().t(), slack @ w.abs().t(), cols, "dx"),
            (gw, x.t() @ dpre, x.abs().t() @ dpre.abs(), x.abs().t() @ slack, n, "dw")):
        if got is None:
            continue
        bound = _steps(t, depth) * (terms + slack_terms) + slack_terms + 1e-30
        within(got, want, bound + half * (want.abs() + bound), name)
        # the roundings are independent: over the whole matrix they stay below one half step (rms of a rounding is
        # at most 0.58 of its half step; two of them, of dpre and of the output, 0.82)
        if want.numel() > 4096:
            assert float((got.double() - want).norm() / want.norm()) < max(half, _steps(t, depth)), name
    if gb is not None:
        within(gb, dpre.sum(0), ((n / 8 + 64) * U32) * dpre.abs().sum(0) + off.sum(0) + 1e-30, "dbias")


SIZES = [(1, 64, 64), (1, 8, 8), (1, 1024, 8192), (3, 16, 24), (7, 72, 40), (16, 1024, 512), (33, 200, 264), (64, 2048, 96),
         (127, 136, 648), (128, 256, 256), (129, 264, 136), (200, 8, 1024), (257, 1032, 520), (300, 4096, 256), (1000, 520, 1000),
         (2050, 256, 768)]


@pytest.mark.parametrize("dtype,out", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("n,K,cols", SIZES)
def test_against_the_formula(n, K, cols, dtype, out):
    t = _make(n, K, cols, dtype, out)
    act = ACTS[(n + K + cols) % 5]
    y, kept = _forward(t, act, residual=True, pre=True)
    _check_forward(t, y, kept, act, residual=True)
    _check_backward(t, act, *_backward(t, act))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("n", [5, 300])
def test_every_activation_and_option(n, act, dtype):
    t = _make(n, 136, 328, dtype)
    for bias, residual, pre in itertools.product((False, True), repeat=3):
        y, kept = _forward(t, act, bias=bias, residual=residual, pre=pre)
        _check_forward(t, y, kept, act, bias=bias, residual=residual)
    full = _backward(t, act)
    _check_backward(t, act, *full)
    for dx, dw, db in ((True, False, False), (False, True, False), (False, False, True), (True, True, False)):
        part = _backward(t, act, dx=dx, dw=dw, db=db)
        for a, b in zip(part, full):
            assert a is None or torch.equal(a, b)


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu", "relu"])
def test_far_pre_activations(act):
    """Large values of either sign: no overflow turns into NaN, the far left is zero."""
    t = _make(64, 64, 64, BF)
    t["x"] = (t["x"].float() * 300).to(BF)
    y, kept = _forward(t, act, pre=True)
    _check_forward(t, y, kept, act)
    t["pre"] = (t["pre"].float() * 100).to(BF)
    _check_backward(t, act, *_backward(t, act))


@pytest.mark.parametrize("n", [9, 400])
def test_residual_in_place_and_guard_rows(n):
    for dtype in (BF, F32):
        t = _make(n, 256, 512, dtype)
        want, _ = _forward(t, "silu", residual=True)
        big = torch.full((n + 2, 512), 7.0, dtype=dtype, device="cuda")
        big[1:n + 1] = t["residual"]
        t["residual"] = big[1:n + 1]
        got, _ = _forward(t, "silu", residual=True, y=big[1:n + 1])
        assert torch.equal(got, want)
        assert (big[0] == 7).all() and (big[-1] == 7).all()


def test_no_rows():
    t = _make(0, 64, 128, BF)
    B.gshard_linear_forward(t["x"], t["w"], torch.empty_like(t["dy"]), bias=t["bias"], workspace=_ws(t, False))
    gx, gw, gb = _backward(t, "relu")
    assert gx.numel() == 0 and (gw == 0).all() and (gb == 0).all()


def test_infinity_and_nan_reach_their_row_only():
    t = _make(300, 256, 256, BF)
    y0, _ = _forward(t)
    t["x"][17, 5] = float("nan")
    y, _ = _forward(t)
    assert torch.isnan(y[17]).all()
    keep = torch.arange(300, device="cuda") != 17
    assert torch.equal(y[keep], y0[keep])


@pytest.mark.parametrize("n,K,cols", [(1, 1024, 2048), (40, 512, 256), (3000, 256, 512)])
def test_same_bits_again_on_another_stream_and_in_a_graph(n, K, cols):
    t = _make(n, K, cols, BF)
    y, kept = _forward(t, "gelu", residual=True, pre=True)
    grads = _backward(t, "gelu")
    out = [torch.zeros_like(v) for v in (y, kept, *grads)]
    wf, wb = _ws(t, False), _ws(t, True)

    def step():
        B.gshard_linear_forward(t["x"], t["w"], out[0], bias=t["bias"], residual=t["residual"], pre=out[1], activation="gelu",
                                workspace=wf)
        B.gshard_linear_backward(t["x"], t["w"], t["dy"], out[2], out[3], out[4], pre=t["pre"], activation="gelu", workspace=wb)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    for got, want in zip(out, (y, kept, *grads)):
        assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    fresh = _make(n, K, cols, BF, seed=4)
    for k in t:
        t[k].copy_(fresh[k])
    graph.replay()
    _check_forward(t, out[0], out[1], "gelu", residual=True)
    _check_backward(t, "gelu", *out[2:])


def test_gradients_against_differences():
    """fp32, pre from the forward itself: directional derivatives of the 64-bit loss."""
    for act in ACTS:
        t = _make(24, 40, 56, F32)
        _, t["pre"] = _forward(t, act, pre=True)
        gx, gw, gb = _backward(t, act)
        gen = torch.Generator(device="cuda").manual_seed(3)
        for name, grad in (("x", gx), ("w", gw), ("bias", gb)):
            d = torch.randn(t[name].shape, generator=gen, device="cuda", dtype=torch.float64)

            def loss(h):
                u = {k: v.double() for k, v in t.items()}
                u[name] = u[name] + h * d
                return (activation(u["x"] @ u["w"] + u["bias"], act) * u["dy"]).sum()

            want = float((loss(1e-6) - loss(-1e-6)) / 2e-6)
            got = float((grad.double() * d).sum())
            # a relu kink within the step of some pre-activation would show up as at most |d pre| 1e-6 each
            assert abs(got - want) < 1e-4 * (1 + float((grad.double().abs() * d.abs()).sum()) * 0.01), (act, name)


def test_large_ragged_batch_sampled_rows():
    """The feed-forward projections over a ragged batch; rows at tile edges and a sample of the others."""
    for K, cols, act in ((1024, 8192, "relu"), (8192, 1024, "none")):
        n = 20011
        t = _make(n, K, cols, BF)
        y, _ = _forward(t, act, residual=True)
        rows = torch.cat([torch.arange(0, 300), torch.arange(n - 300, n), torch.randint(0, n, (200,))]).unique().cuda()
        u = {k: (v[rows] if v.shape[0] == n else v) for k, v in t.items()}
        _check_forward(u, y[rows], None, act, residual=True)


def test_refusals():
    t = _make(4, 64, 128, BF)
    y = torch.empty_like(t["dy"])
    for kw in (dict(w=t["w"].t()), dict(w=t["w"].float()), dict(bias=t["bias"].bfloat16()), dict(residual=t["residual"][:2]),
               dict(y=y.cpu()), dict(x=t["x"].half()), dict(workspace=torch.empty(256, dtype=torch.uint8))):
        a = dict(x=t["x"], w=t["w"], y=y, bias=None, residual=None, workspace=_ws(t, False))
        a.update(kw)
        with pytest.raises(ValueError):
            B.gshard_linear_forward(a["x"], a["w"], a["y"], bias=a["bias"], residual=a["residual"], workspace=a["workspace"])
    with pytest.raises(B.GshardError) as e:
        B.gshard_linear_forward(t["x"], t["w"], y)
    assert e.value.code == B.GSHARD_ERR_INVALID_ARG
    odd = _make(4, 60, 128, BF)
    with pytest.raises(B.GshardError) as e:
        B.gshard_linear_forward(odd["x"], odd["w"], y, workspace=_ws(t, False))
    assert e.value.code == B.GSHARD_ERR_UNSUPPORTED_SHAPE
    for act in (7, -1):
        with pytest.raises(B.GshardError) as e:
            B.gshard_linear_forward(t["x"], t["w"], y, activation=act, workspace=_ws(t, False))
        assert e.value.code == B.GSHARD_ERR_INVALID_ARG
    with pytest.raises(B.GshardError):                       # relu's gradient needs the pre-activations
        B.gshard_linear_backward(t["x"], t["w"], t["dy"], torch.empty_like(t["x"]), activation="relu", workspace=_ws(t, True))
    square = _make(64, 64, 64, BF)
    with pytest.raises(B.GshardError):                       # an output over an operand
        B.gshard_linear_forward(square["x"], square["w"], square["x"], workspace=_ws(square, False))


# Products whose tiles of 128 x 64 or 128 x 128 run at once take one launch: one CTA, or 2 or 4 sharing the contraction.
ONE_LAUNCH = [(3, 1024, 72), (9, 8, 8), (17, 128, 64), (40, 136, 9472), (65, 256, 8), (100, 512, 1000), (127, 1160, 200),
              (128, 2048, 264), (129, 3840, 72), (130, 1024, 4744), (255, 640, 136), (513, 1096, 520), (1025, 776, 1160),
              (2049, 264, 640), (64, 8200, 1024), (31, 16392, 40)]


@pytest.mark.parametrize("n,K,cols", ONE_LAUNCH)
def test_products_of_one_launch(n, K, cols):
    t = _make(n, K, cols, BF)
    act = ACTS[(n + cols) % 5]
    guard = torch.full((n + 2, cols), 7.0, dtype=BF, device="cuda")
    y, kept = _forward(t, act, residual=True, pre=True, y=guard[1:n + 1])
    _check_forward(t, y, kept, act, residual=True)
    assert (guard[0] == 7).all() and (guard[-1] == 7).all()
    again, _ = _forward(t, act, residual=True)
    assert torch.equal(again, y)
    plain, _ = _forward(t, bias=False)
    _check_forward(t, plain, None, "none", bias=False)
    _check_backward(t, act, *_backward(t, act))


@pytest.mark.parametrize("out", [BF, F32])
@pytest.mark.parametrize("n", [1, 8, 9, 200, 3000])
def test_status_word_is_cleared(n, out):
    """A workspace full of ones, as another call may have left it, reads as success afterwards."""
    t = _make(n, 256, 512, BF, out)
    y = torch.empty_like(t["dy"])
    ws = _ws(t, False).fill_(255)
    B.gshard_linear_forward(t["x"], t["w"], y, workspace=ws)
    assert B.gshard_moe_last_device_status(ws) == B.GSHARD_OK
    for act in ("none", "gelu"):
        for wanted in ((1, 1, 1), (1, 0, 0), (0, 1, 0), (0, 0, 1), (0, 0, 0)):
            g = [torch.empty_like(v) if on else None for on, v in zip(wanted, (t["x"], t["w"], t["bias"]))]
            ws = _ws(t, True).fill_(255)
            B.gshard_linear_backward(t["x"], t["w"], t["dy"], *g, pre=None if act == "none" else t["pre"], activation=act,
                                     workspace=ws)
            assert B.gshard_moe_last_device_status(ws) == B.GSHARD_OK


def test_rows_of_one_launch_do_not_touch_each_other():
    """Infinities and NaN in a row of x stay in its row of y, whatever the rows that a tile does not have."""
    for n in (5, 60, 130):
        t = _make(n, 1024, 256, BF)
        y0, _ = _forward(t)
        t["x"][n - 1, 7] = float("nan")
        t["x"][0, 9] = float("inf")
        y, _ = _forward(t)
        assert torch.isnan(y[n - 1]).all() and not torch.isfinite(y[0]).any()
        assert torch.equal(y[1:n - 1], y0[1:n - 1])


@pytest.mark.parametrize("dtype,n,K,cols", [
    (BF, 9, 8, 8), (BF, 33, 264, 200), (BF, 100, 2048, 9000), (BF, 130, 8192, 40), (BF, 64, 2056, 4000), (BF, 1000, 1408, 712),
    (F32, 9, 8, 8), (F32, 33, 264, 200), (F32, 100, 2048, 1000), (F32, 60, 512, 9000), (F32, 130, 1024, 1032), (F32, 1025, 392, 648)])
def test_fp32_products_of_one_launch(dtype, n, K, cols):
    """fp32 results are accumulated in runs of 256, so their error does not grow with the depth."""
    t = _make(n, K, cols, dtype, F32)
    act = ACTS[(n + cols) % 5]
    guard = torch.full((n + 2, cols), 7.0, device="cuda")
    y, kept = _forward(t, act, residual=True, pre=True, y=guard[1:n + 1])
    _check_forward(t, y, kept, act, residual=True)
    assert (guard[0] == 7).all() and (guard[-1] == 7).all()
    again, _ = _forward(t, act, residual=True)
    assert torch.equal(again, y)
    # a run is 16 truncated steps of at most 2^-23 of the absolute sum; the small products, up to 240 steps at 2^-8 of it,
    # count as one, the sums of at most 64 runs and of the cluster, 2^-24 of a partial sum each, as fewer than 8, and the
    # three products left out as one: 32 covers them
    plain, _ = _forward(t, bias=False)
    want = t["x"].double() @ t["w"].double()
    total = t["x"].double().abs() @ t["w"].double().abs()
    within(plain, want, 32 * 2 * U32 * total + 1e-30, "product")
    _check_backward(t, act, *_backward(t, act))


def test_two_threads_at_once():
    """Calls of different sizes from two threads, each with its own stream and workspace, do not disturb each other."""
    import threading
    sizes = ([(3, 1024, 72), (128, 2048, 264)], [(100, 512, 1000), (700, 1096, 520)])
    cases = [[(t, _forward(t, "gelu", residual=True)[0], torch.empty_like(t["dy"]), _ws(t, False))
              for t in (_make(*s, BF) for s in group)] for group in sizes]
    torch.cuda.synchronize()
    failed = []

    def work(group):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for i in range(200):
                    t, want, y, ws = group[i % 2]
                    B.gshard_linear_forward(t["x"], t["w"], y, bias=t["bias"], residual=t["residual"], activation="gelu",
                                            workspace=ws)
                stream.synchronize()
        except Exception as e:                               # noqa: BLE001 - reported by the main thread
            failed.append(e)

    threads = [threading.Thread(target=work, args=(g,)) for g in cases]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert not failed, failed
    for group in cases:
        for _, want, y, ws in group:
            assert torch.equal(y, want) and B.gshard_moe_last_device_status(ws) == B.GSHARD_OK
