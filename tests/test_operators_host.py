"""Host-side checks of the layer norm, linear and routing entry points that need no GPU: sizes of
workspaces, refused arguments, and that valid ones fail only at the device check."""
import ctypes

import pytest
import torch

from paper_2006_16668_b200 import binding as B
from paper_2006_16668_b200.build import build_library

FAKE = 0x10000
INVALID, SHAPE, SMALL = B.GSHARD_ERR_INVALID_ARG, B.GSHARD_ERR_UNSUPPORTED_SHAPE, B.GSHARD_ERR_WORKSPACE_TOO_SMALL
NO_GPU = (B.GSHARD_ERR_CUDA, B.GSHARD_ERR_ARCH)


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_library()


def _ln_fwd(n=4, M=64, dtype=0, eps=1e-5, x=FAKE, gamma=FAKE, beta=FAKE, y=FAKE, mean=FAKE, rstd=FAKE):
    return B.load().gshard_layer_norm_forward(n, M, dtype, eps, x, gamma, beta, y, mean, rstd, None)


def _ln_bwd(n=4, M=64, dtype=0, x=FAKE, gamma=FAKE, mean=FAKE, rstd=FAKE, dy=FAKE, dskip=None, dx=FAKE, dgamma=FAKE, dbeta=FAKE,
            ws=FAKE, size=1 << 30):
    return B.load().gshard_layer_norm_backward(n, M, dtype, x, gamma, mean, rstd, dy, dskip, dx, dgamma, dbeta, ws, size, None)


def test_layer_norm_arguments():
    for kw, rc in ((dict(n=-1), INVALID), (dict(M=0), INVALID), (dict(M=16385), SHAPE), (dict(dtype=2), INVALID),
                   (dict(eps=-1e-3), INVALID), (dict(eps=float("nan")), INVALID), (dict(x=None), INVALID), (dict(y=None), INVALID),
                   (dict(gamma=None), INVALID), (dict(x=FAKE + 2), INVALID), (dict(mean=FAKE + 4), INVALID), (dict(n=1 << 40), SHAPE),
                   (dict(n=0, x=None, y=None), B.GSHARD_OK)):
        assert _ln_fwd(**kw) == rc, kw
    for kw, rc in ((dict(n=-1), INVALID), (dict(dy=None), INVALID), (dict(dx=None), INVALID), (dict(mean=None), INVALID),
                   (dict(rstd=None), INVALID), (dict(dskip=FAKE + 8), INVALID), (dict(ws=None), INVALID), (dict(ws=FAKE + 16), INVALID),
                   (dict(size=256), SMALL), (dict(M=20000), SHAPE),
                   (dict(n=0, dgamma=None, dbeta=None), B.GSHARD_OK)):
        assert _ln_bwd(**kw) == rc, kw
    assert B.gshard_layer_norm_workspace_bytes(10, 64) >= 2 * 64 * 4
    assert B.gshard_layer_norm_workspace_bytes(10, 0) == 0 and B.gshard_layer_norm_workspace_bytes(-1, 64) == 0
    if not torch.cuda.is_available():
        assert _ln_fwd() in NO_GPU and _ln_fwd(beta=None, mean=None, rstd=None) in NO_GPU
        assert _ln_bwd() in NO_GPU and _ln_bwd(dgamma=None, dbeta=None, ws=None, size=0) in NO_GPU


def _lin_fwd(n=4, K=64, cols=128, dtype=1, out=1, act=0, x=FAKE, w=FAKE + 4096, bias=None, res=None, y=FAKE + 8192, pre=None, ws=FAKE,
             size=1 << 30):
    return B.load().gshard_linear_forward(n, K, cols, dtype, out, act, x, w, bias, res, y, pre, ws, size, None)


def _lin_bwd(n=4, K=64, cols=128, dtype=1, out=1, act=0, x=FAKE, w=FAKE + 4096, pre=None, dy=FAKE + 8192, dx=FAKE + 12288,
             dw=FAKE + 16384, db=FAKE, ws=FAKE, size=1 << 30):
    return B.load().gshard_linear_backward(n, K, cols, dtype, out, act, x, w, pre, dy, dx, dw, db, ws, size, None)


def test_linear_arguments():
    for kw, rc in ((dict(n=-1), INVALID), (dict(K=0), INVALID), (dict(cols=-8), INVALID), (dict(K=60), SHAPE), (dict(cols=100), SHAPE),
                   (dict(dtype=0, out=1), INVALID), (dict(dtype=3), INVALID), (dict(act=5), INVALID), (dict(act=-1), INVALID),
                   (dict(n=(1 << 30) + 1), SHAPE), (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(y=None), INVALID),
                   (dict(bias=FAKE + 4), INVALID), (dict(res=FAKE + 2), INVALID), (dict(pre=FAKE + 8), INVALID), (dict(ws=None), INVALID),
                   (dict(ws=FAKE + 128), INVALID), (dict(size=16), SMALL), (dict(y=FAKE), INVALID), (dict(pre=FAKE + 8192), INVALID),
                   (dict(n=0, x=None, w=None, y=None, ws=None, size=0), B.GSHARD_OK)):
        assert _lin_fwd(**kw) == rc, kw
    for kw, rc in ((dict(n=-1), INVALID), (dict(K=60), SHAPE), (dict(act=1), INVALID), (dict(dy=None), INVALID), (dict(w=None), INVALID),
                   (dict(x=None), INVALID), (dict(size=300), SMALL), (dict(dx=FAKE), INVALID), (dict(dw=FAKE + 8192), INVALID),
                   (dict(n=0, dw=None, db=None), B.GSHARD_OK)):
        assert _lin_bwd(**kw) == rc, kw
    bf, f32 = torch.bfloat16, torch.float32
    assert B.gshard_linear_workspace_bytes(4, 60, 64, bf) == 0
    assert B.gshard_linear_workspace_bytes(4, 64, 64, f32, bf) == 0
    assert B.gshard_linear_workspace_bytes(4, 64, 64, bf, f32) >= 256
    assert B.gshard_linear_workspace_bytes(1000, 64, 64, bf, for_backward=True) >= 1000 * 64 * 2
    if not torch.cuda.is_available():
        assert _lin_fwd() in NO_GPU and _lin_fwd(res=FAKE + 8192, act=2) in NO_GPU and _lin_fwd(dtype=1, out=0) in NO_GPU
        assert _lin_bwd() in NO_GPU and _lin_bwd(dw=None, x=None) in NO_GPU and _lin_bwd(dx=None, w=None, act=1, pre=FAKE) in NO_GPU


def _route(cfg, logits=FAKE, bias=None, idx=FAKE, weight=FAKE, m=None, load=None, ws=None, size=0):
    return B.load().gshard_moe_route(ctypes.byref(cfg), logits, bias, idx, weight, m, load, ws, size, None)


def test_route_arguments():
    base = dict(G=2, S=8, E=16, k=2)
    for kw, rc in ((dict(E=0), INVALID), (dict(k=0), INVALID), (dict(k=17), INVALID), (dict(G=-1), INVALID), (dict(groups=3), INVALID),
                   (dict(groups=0), INVALID), (dict(groups=4, groups_kept=5), INVALID), (dict(groups=4, groups_kept=0), INVALID),
                   (dict(groups=8, groups_kept=1, k=3), INVALID), (dict(group_top=3), INVALID), (dict(group_top=0), INVALID),
                   (dict(scale=float("inf")), INVALID), (dict(scale=float("nan")), INVALID), (dict(E=20000), SHAPE),
                   (dict(E=64, k=33), SHAPE), (dict(E=66, groups=33), SHAPE), (dict(G=70000), SHAPE), (dict(G=60000, S=60000), SHAPE)):
        cfg = B.make_route(**{**base, **kw})
        assert _route(cfg) == rc, kw
        assert B.gshard_moe_route_workspace_bytes(cfg) == 0
        assert B.load().gshard_moe_route_backward(ctypes.byref(cfg), FAKE, FAKE, FAKE, None, FAKE + 4096, None) == rc
    cfg = B.make_route(**base)
    need = B.gshard_moe_route_workspace_bytes(cfg)
    assert need >= 2 * 16 * 4
    for kw in (dict(logits=None), dict(idx=None), dict(weight=None), dict(logits=FAKE + 8), dict(bias=FAKE + 4), dict(m=FAKE),
               dict(m=FAKE, ws=FAKE + 16, size=need), dict(load=FAKE + 4)):
        assert _route(cfg, **kw) == INVALID, kw
    assert _route(cfg, m=FAKE, ws=FAKE, size=need - 1) == SMALL
    assert B.load().gshard_moe_route(None, FAKE, None, FAKE, FAKE, None, None, None, 0, None) == INVALID
    bad = B.make_route(**base)
    bad.score = 2
    assert _route(bad) == INVALID
    bwd = B.load().gshard_moe_route_backward
    assert bwd(ctypes.byref(cfg), FAKE, FAKE, FAKE, None, FAKE, None) == INVALID       # over the logits
    assert bwd(ctypes.byref(cfg), FAKE, FAKE, None, None, FAKE + 4096, None) == INVALID
    empty = B.make_route(G=0, S=8, E=16, k=2)
    assert _route(empty, logits=None, idx=None, weight=None) == B.GSHARD_OK
    if not torch.cuda.is_available():
        assert _route(cfg) in NO_GPU and _route(cfg, m=FAKE, ws=FAKE, size=need) in NO_GPU
        assert bwd(ctypes.byref(cfg), FAKE, FAKE, FAKE, None, FAKE + 4096, None) in NO_GPU


def test_binding_refuses_host_tensors_and_mismatches():
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError, match="CUDA"):
        B.gshard_layer_norm_forward(x, torch.zeros(64), None, torch.zeros(4, 64))
    with pytest.raises(ValueError, match="gamma"):
        B.gshard_layer_norm_forward(x, torch.zeros(63), None, torch.zeros(4, 64))
    with pytest.raises(ValueError, match="dtype"):
        B.gshard_layer_norm_forward(x.half(), torch.zeros(64), None, torch.zeros(4, 64))
    with pytest.raises(ValueError, match="w:"):
        B.gshard_linear_forward(x, torch.zeros(32, 8), torch.zeros(4, 8))
    with pytest.raises(ValueError, match="residual"):
        B.gshard_linear_forward(x, torch.zeros(64, 8), torch.zeros(4, 8), residual=torch.zeros(8, 8).t()[:4])
    for act in ("gelu_fast", None, 1.5):
        with pytest.raises(ValueError, match="activation"):
            B.gshard_linear_forward(x, torch.zeros(64, 8), torch.zeros(4, 8), activation=act)
    cfg = B.make_route(G=1, S=4, E=8, k=2)
    with pytest.raises(ValueError, match="expert_idx"):
        B.gshard_moe_route(cfg, torch.zeros(1, 4, 8), torch.zeros(1, 4, 2, dtype=torch.int64), torch.zeros(1, 4, 2))
