"""Layer norm, forward and backward, against the formula in 64 bits.

Bounds (U = 2^-24).  A thread adds at most 32 values in a row before at most 10 levels of pairwise sums, so
a sum over a row carries at most 48 roundings of its absolute sum: the mean is off by 48 U mean|x|, the
relative error of rstd is at most 48 U plus twice the mean's error over the spread plus a few U, and each
stored value adds half a step of its type.  Sums over rows add one rounding per row of a team's walk
(at most n / 148 + 1 rows) and 40 for the joins."""
import pytest
import torch

from operator_reference import HALF, U32, layer_norm, layer_norm_grad, within
from paper_2006_16668_b200 import binding as B

pytestmark = pytest.mark.gpu

EPS = 1e-5


def _make(n, M, dtype, seed=0, offset=0.3):
    gen = torch.Generator(device="cuda").manual_seed(1000 * n + M + seed)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    return {"x": (1.5 * r(n, M) + offset).to(dtype), "gamma": 1 + 0.1 * r(M), "beta": 0.1 * r(M),
            "dy": r(n, M).to(dtype), "dskip": r(n, M).to(dtype)}


def _forward(t, beta=True, stats=True, y=None):
    n, M = t["x"].shape
    y = torch.full_like(t["x"], float("nan")) if y is None else y
    mean, rstd = (torch.full((n,), float("nan"), device="cuda") for _ in range(2)) if stats else (None, None)
    B.gshard_layer_norm_forward(t["x"], t["gamma"], t["beta"] if beta else None, y, mean, rstd, eps=EPS)
    return y, mean, rstd


def _backward(t, mean, rstd, skip=True, dx=None, weights=True):
    n, M = t["x"].shape
    dx = torch.full_like(t["x"], float("nan")) if dx is None else dx
    dg, db = (torch.full((M,), float("nan"), device="cuda") for _ in range(2)) if weights else (None, None)
    ws = torch.empty(max(256, B.gshard_layer_norm_workspace_bytes(n, M)), dtype=torch.uint8, device="cuda") if weights else None
    B.gshard_layer_norm_backward(t["x"], t["gamma"], mean, rstd, t["dy"], dx, dg, db, dskip=t["dskip"] if skip else None,
                                 workspace=ws)
    return dx, dg, db


def _check_forward(t, y, mean, rstd, beta=True):
    want_y, want_mean, want_rstd = layer_norm(t["x"], t["gamma"], t["beta"] if beta else None, EPS)
    x, half = t["x"].double(), HALF[t["x"].dtype]
    mean_abs = x.abs().mean(1)
    mean_bound = 50 * U32 * mean_abs + 1e-38
    spread = (mean_bound * want_rstd) * 2 + 60 * U32
    if mean is not None:
        within(mean, want_mean, mean_bound, "mean")
        within(rstd, want_rstd, want_rstd * spread, "rstd")
    z = ((x - want_mean[:, None]) * want_rstd[:, None]).abs()
    b = 0 if not beta else t["beta"].double().abs()
    bound = t["gamma"].double().abs() * (z * spread[:, None] + (mean_bound * want_rstd)[:, None] + 6 * U32 * z) \
        + 4 * U32 * (want_y.abs() + b)
    within(y, want_y, bound + half * (want_y.abs() + bound), "y")


def _check_backward(t, mean, rstd, dx, dg, db, skip=True):
    want_dx, want_dg, want_db = layer_norm_grad(t["x"], t["gamma"], mean, rstd, t["dy"], t["dskip"] if skip else None)
    half = HALF[t["x"].dtype]
    r = rstd.double()[:, None]
    z = (t["x"].double().abs() + mean.double().abs()[:, None]) * r          # |z| before any cancellation
    dy = t["dy"].double().abs()
    g = dy * t["gamma"].double().abs()
    terms = r * (g + g.mean(1, keepdim=True) + z * (g * z).mean(1, keepdim=True))
    bound = 60 * U32 * terms + 4 * U32 * (t["dskip"].double().abs() if skip else 0)
    within(dx, want_dx, bound + half * (want_dx.abs() + bound) + 1e-38, "dx")
    if dg is not None:
        rows = t["x"].shape[0] / 148 + 50
        within(dg, want_dg, rows * U32 * (dy * z).sum(0) + 1e-38, "dgamma")
        within(db, want_db, rows * U32 * dy.sum(0) + 1e-38, "dbeta")


SIZES = [(1, 1024), (1, 1), (3, 7), (5, 8), (2, 32), (40, 255), (33, 256), (70, 264), (129, 513), (1300, 1024), (1184, 1000),
         (1190, 1022), (1201, 341), (2, 1025), (300, 2050), (37, 4096), (9, 8191), (5, 8192), (4, 8200), (3, 12345),
         (2, 16384), (1, 16383), (2500, 96)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,M", SIZES)
def test_forward_and_backward_against_the_formula(n, M, dtype):
    t = _make(n, M, dtype)
    y, mean, rstd = _forward(t)
    _check_forward(t, y, mean, rstd)
    dx, dg, db = _backward(t, mean, rstd)
    _check_backward(t, mean, rstd, dx, dg, db)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,M", [(7, 96), (1500, 1024), (6, 9000)])
def test_optional_tensors_and_in_place(n, M, dtype):
    t = _make(n, M, dtype, seed=1)
    full, mean, rstd = _forward(t)
    y, _, _ = _forward(t, beta=False, stats=False)
    _check_forward(t, y, None, None, beta=False)
    same = t["x"].clone()
    B.gshard_layer_norm_forward(same, t["gamma"], t["beta"], same, eps=EPS)
    assert torch.equal(same, full)
    dx, dg, db = _backward(t, mean, rstd, skip=False)
    _check_backward(t, mean, rstd, dx, dg, db, skip=False)
    only, _, _ = _backward(t, mean, rstd, skip=False, weights=False)
    assert torch.equal(only, dx)
    with_skip, _, _ = _backward(t, mean, rstd)
    for name in ("dy", "dskip"):                       # dx may overwrite either
        u = {k: v.clone() for k, v in t.items()}
        got, dg2, db2 = _backward(u, mean, rstd, dx=u[name])
        assert torch.equal(got, with_skip) and torch.equal(dg2, dg) and torch.equal(db2, db)


def test_rows_without_spread_and_large_offsets():
    """Constant rows (variance 0) give beta; rows far from zero keep their spread."""
    x = torch.full((4, 1024), 3.0, device="cuda")
    x[1] = 0.0
    t = _make(4, 1024, torch.float32)
    t["x"] = x
    y, mean, rstd = _forward(t)
    assert torch.equal(y, t["beta"].expand(4, -1))
    assert torch.allclose(rstd, torch.full_like(rstd, EPS ** -0.5), rtol=1e-6)
    far = _make(64, 1024, torch.float32, offset=1000.0)
    y, mean, rstd = _forward(far)
    _check_forward(far, y, mean, rstd)


def test_a_row_with_nan_or_infinity_stays_alone():
    t = _make(1400, 512, torch.bfloat16)
    y0, _, _ = _forward(t)
    t["x"][3, 100] = float("nan")
    t["x"][1000, 7] = float("inf")
    y, mean, rstd = _forward(t)
    assert torch.isnan(y[3]).all() and torch.isnan(y[1000]).all()
    rest = torch.ones(1400, dtype=torch.bool, device="cuda")
    rest[[3, 1000]] = False
    assert torch.equal(y[rest], y0[rest])


def test_no_rows():
    t = _make(0, 512, torch.bfloat16)
    y, mean, rstd = _forward(t)
    dx, dg, db = _backward(t, mean, rstd)
    assert y.numel() == 0 and dx.numel() == 0
    assert (dg == 0).all() and (db == 0).all()


def test_rows_behind_the_batch_are_left_alone():
    t = _make(50, 1024, torch.bfloat16)
    big = torch.full((52, 1024), 7.0, dtype=torch.bfloat16, device="cuda")
    y, mean, rstd = _forward(t, y=big[1:51])
    dx, _, _ = _backward(t, mean, rstd)
    assert (big[0] == 7).all() and (big[51] == 7).all()
    _check_forward(t, big[1:51], mean, rstd)


@pytest.mark.parametrize("n,M", [(1, 64), (5000, 1024), (700, 4096)])
def test_same_bits_again_on_another_stream_and_in_a_graph(n, M):
    t = _make(n, M, torch.bfloat16)
    y, mean, rstd = _forward(t)
    first = (y, *_backward(t, mean, rstd))
    out = {"y": torch.zeros_like(y), "mean": torch.zeros_like(mean), "rstd": torch.zeros_like(rstd),
           "dx": torch.zeros_like(y), "dg": torch.zeros(M, device="cuda"), "db": torch.zeros(M, device="cuda")}
    ws = torch.empty(B.gshard_layer_norm_workspace_bytes(n, M), dtype=torch.uint8, device="cuda")

    def step():
        B.gshard_layer_norm_forward(t["x"], t["gamma"], t["beta"], out["y"], out["mean"], out["rstd"], eps=EPS)
        B.gshard_layer_norm_backward(t["x"], t["gamma"], out["mean"], out["rstd"], t["dy"], out["dx"], out["dg"], out["db"],
                                     dskip=t["dskip"], workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    for got, want in zip((out["y"], out["dx"], out["dg"], out["db"]), first):
        assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    fresh = _make(n, M, torch.bfloat16, seed=5)
    for k in t:
        t[k].copy_(fresh[k])
    graph.replay()
    _check_forward(t, out["y"], out["mean"], out["rstd"])
    _check_backward(t, out["mean"], out["rstd"], out["dx"], out["dg"], out["db"])


@pytest.mark.parametrize("n,M", [(6, 40), (4, 1100)])
def test_gradients_against_differences(n, M):
    """Directional derivatives of the 64-bit forward: central differences with step 1e-5 are exact to about
    1e-9 relative, the fp32 gradients to about 60 U of the absolute terms, so 1e-4 is ample."""
    t = _make(n, M, torch.float32, seed=9)
    _, mean, rstd = _forward(t)
    dx, dg, db = _backward(t, mean, rstd, skip=False)
    gen = torch.Generator(device="cuda").manual_seed(3)
    for name, grad in (("x", dx), ("gamma", dg), ("beta", db)):
        d = torch.randn(t[name].shape, generator=gen, device="cuda", dtype=torch.float64)

        def loss(h):
            u = {k: v.double() for k, v in t.items()}
            u[name] = u[name] + h * d
            return (layer_norm(u["x"], u["gamma"], u["beta"], EPS)[0] * u["dy"]).sum()

        want = (loss(1e-5) - loss(-1e-5)) / 2e-5
        got = (grad.double() * d).sum()
        assert abs(float(got - want)) < 1e-4 * max(1.0, abs(float(want))) + 1e-4 * float((grad.double().abs() * d.abs()).sum()) * 0.01


def test_offsets_beyond_32_bits():
    """2^31 + elements: the last rows are the same as computed alone."""
    M, n = 16384, (1 << 31) // 16384 + 3
    x = torch.empty(n, M, dtype=torch.bfloat16, device="cuda")
    x.normal_()
    gamma, beta = torch.ones(M, device="cuda"), torch.zeros(M, device="cuda")
    y = torch.empty_like(x)
    B.gshard_layer_norm_forward(x, gamma, beta, y, eps=EPS)
    tail = torch.empty(3, M, dtype=torch.bfloat16, device="cuda")
    B.gshard_layer_norm_forward(x[-3:], gamma, beta, tail, eps=EPS)
    assert torch.equal(y[-3:], tail)


def test_refusals():
    t = _make(4, 64, torch.float32)
    y = torch.empty_like(t["x"])
    for bad in (dict(x=t["x"].t()), dict(gamma=t["gamma"][:32]), dict(y=y.bfloat16()), dict(gamma=t["gamma"].double()),
                dict(beta=t["beta"].cpu()), dict(x=t["x"].half())):
        a = {"x": t["x"], "gamma": t["gamma"], "beta": t["beta"], "y": y, **bad}
        with pytest.raises(ValueError):
            B.gshard_layer_norm_forward(a["x"], a["gamma"], a["beta"], a["y"])
    with pytest.raises(B.GshardError) as e:
        B.gshard_layer_norm_forward(t["x"], t["gamma"], t["beta"], y, eps=-1.0)
    assert e.value.code == B.GSHARD_ERR_INVALID_ARG
    big = torch.zeros(1, 16385, device="cuda")
    with pytest.raises(B.GshardError) as e:
        B.gshard_layer_norm_forward(big, big[0], None, big.clone())
    assert e.value.code == B.GSHARD_ERR_UNSUPPORTED_SHAPE
    _, mean, rstd = _forward(t)
    with pytest.raises(B.GshardError) as e:                   # weight gradients need the workspace
        B.gshard_layer_norm_backward(t["x"], t["gamma"], mean, rstd, t["dy"], y, torch.empty(64, device="cuda"))
    assert e.value.code == B.GSHARD_ERR_INVALID_ARG
    small = torch.empty(B.gshard_layer_norm_workspace_bytes(4, 64) - 256, dtype=torch.uint8, device="cuda")
    with pytest.raises(B.GshardError) as e:
        B.gshard_layer_norm_backward(t["x"], t["gamma"], mean, rstd, t["dy"], y, torch.empty(64, device="cuda"), workspace=small)
    assert e.value.code in (B.GSHARD_ERR_WORKSPACE_TOO_SMALL, B.GSHARD_ERR_INVALID_ARG)


def test_long_rows_from_two_threads_at_once():
    """Backward passes over rows of two lengths, whose blocks share different amounts of memory, from two threads."""
    import threading
    cases = []
    for M in (9000, 16384):
        t = _make(40, M, torch.float32)
        _, mean, rstd = _forward(t)
        cases.append((t, mean, rstd, _backward(t, mean, rstd)))
    torch.cuda.synchronize()
    failed = []

    def work(t, mean, rstd, want):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(100):
                    got = _backward(t, mean, rstd)
                torch.cuda.current_stream().synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want))
        except Exception as e:                               # noqa: BLE001 - reported by the main thread
            failed.append(e)

    threads = [threading.Thread(target=work, args=c) for c in cases]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert not failed, failed
