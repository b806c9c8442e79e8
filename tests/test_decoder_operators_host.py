"""Host-side checks of cross attention, gated linear and gradient norm that need no GPU: sizes of workspaces, refused
arguments, and that valid ones fail only at the device check."""
import ctypes
import math

import pytest
import torch

from paper_2006_16668_b200 import binding as B
from paper_2006_16668_b200.build import build_library

P = [0x10000 * (i + 1) for i in range(12)]
INVALID, SHAPE, SMALL, OK = B.GSHARD_ERR_INVALID_ARG, B.GSHARD_ERR_UNSUPPORTED_SHAPE, B.GSHARD_ERR_WORKSPACE_TOO_SMALL, B.GSHARD_OK
NO_GPU = (B.GSHARD_ERR_CUDA, B.GSHARD_ERR_ARCH)


@pytest.fixture(scope="module", autouse=True)
def _built():
    build_library()


def _config(batch=2, q_len=5, k_len=7, heads=4, kv_heads=2, head_dim=64, dtype=1, scale=0.125, q_stride=None, k_stride=None, v_stride=None):
    q = heads * head_dim if q_stride is None else q_stride
    kv = kv_heads * head_dim
    return B.gshard_attention_config(batch, q_len, k_len, heads, kv_heads, head_dim, dtype, scale, q, kv if k_stride is None else k_stride,
                                     kv if v_stride is None else v_stride)


def _att_fwd(q=P[0], k=P[1], v=P[2], lengths=P[3], o=P[4], lse=P[5], ws=P[6], size=1 << 30, **cfg):
    return B.load().gshard_cross_attention_forward(ctypes.byref(_config(**cfg)), q, k, v, lengths, o, lse, ws, size, None)


def _att_bwd(q=P[0], k=P[1], v=P[2], lengths=P[3], o=P[4], lse=P[5], dout=P[7], dq=P[8], dk=P[9], dv=P[10], ws=P[6], size=1 << 30, **cfg):
    return B.load().gshard_cross_attention_backward(ctypes.byref(_config(**cfg)), q, k, v, lengths, o, lse, dout, dq, dk, dv, ws, size, None)


CONFIGS = [(dict(batch=-1), INVALID), (dict(q_len=-1), INVALID), (dict(k_len=-3), INVALID), (dict(heads=0), INVALID), (dict(kv_heads=0), INVALID),
           (dict(kv_heads=3), INVALID), (dict(kv_heads=8), INVALID), (dict(head_dim=60), SHAPE), (dict(head_dim=136), SHAPE),
           (dict(head_dim=0), INVALID), (dict(dtype=2), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
           (dict(scale=math.nan), INVALID), (dict(scale=math.inf), INVALID), (dict(scale=1e-21), INVALID), (dict(scale=2e20), INVALID), (dict(q_stride=255), INVALID), (dict(q_stride=260), INVALID),
           (dict(k_stride=120), INVALID), (dict(v_stride=132), INVALID), (dict(k_stride=1 << 36), SHAPE),
           (dict(heads=65536, kv_heads=2), SHAPE), (dict(batch=1 << 30, k_len=1 << 20), SHAPE), (dict(k_len=(1 << 30) + 1), SHAPE)]


@pytest.mark.parametrize("cfg,rc", CONFIGS)
def test_attention_sizes(cfg, rc):
    assert _att_fwd(**cfg) == rc and _att_bwd(**cfg) == rc
    c = _config(**cfg)
    assert B.load().gshard_cross_attention_workspace_bytes(ctypes.byref(c), 0) == 0
    assert B.load().gshard_cross_attention_workspace_bytes(ctypes.byref(c), 1) == 0


def test_attention_arguments():
    for kw, rc in ((dict(q=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(o=None), INVALID), (dict(q=P[0] + 8), INVALID),
                   (dict(lse=P[5] + 4), INVALID), (dict(lengths=P[3] + 2), INVALID), (dict(ws=None), INVALID), (dict(ws=P[6] + 128), INVALID),
                   (dict(size=0), SMALL), (dict(o=P[0]), INVALID), (dict(o=P[2]), INVALID), (dict(lse=P[4]), INVALID),
                   (dict(batch=0, q=None), OK), (dict(q_len=0, q=None, o=None), OK)):
        assert _att_fwd(**kw) == rc, kw
    for kw, rc in ((dict(dout=None), INVALID), (dict(lse=None), INVALID), (dict(o=None), INVALID), (dict(dq=None), INVALID), (dict(dk=None), INVALID),
                   (dict(dv=P[10] + 2), INVALID), (dict(dq=P[0]), INVALID), (dict(dk=P[9], dv=P[9]), INVALID), (dict(dq=P[7]), INVALID),
                   (dict(size=256), SMALL), (dict(batch=0), OK), (dict(q_len=0, k_len=0), OK)):
        assert _att_bwd(**kw) == rc, kw
    bytes_of = B.gshard_cross_attention_workspace_bytes
    assert bytes_of(2, 5, 7, 4, 2, 64, torch.bfloat16) >= 256
    assert bytes_of(2, 500, 7, 4, 2, 64, torch.bfloat16, for_backward=True) >= 2 * 500 * 4 * 4
    with pytest.raises(ValueError):
        bytes_of(2, 5, 1 << 31, 4, 2, 64, torch.bfloat16)
    with pytest.raises(ValueError):
        bytes_of(2, 5, 7, 4, 2, 64, torch.float16)
    if not torch.cuda.is_available():
        assert _att_fwd() in NO_GPU and _att_fwd(lse=None, lengths=None) in NO_GPU and _att_fwd(k_len=0, k=None, v=None) in NO_GPU
        assert _att_bwd() in NO_GPU and _att_bwd(q_len=0, q=None, o=None, lse=None, dout=None, dq=None) in NO_GPU


def test_attention_binding_checks_its_tensors():
    bf = torch.bfloat16
    q, o, lse = torch.zeros(2, 5, 4, 64, dtype=bf), torch.zeros(2, 5, 4, 64, dtype=bf), torch.zeros(2, 4, 5)
    kv = torch.zeros(2, 7, 2, 2, 64, dtype=bf)
    k, v = kv[:, :, 0], kv[:, :, 1]
    ws = torch.zeros(4096, dtype=torch.uint8)
    ok = dict(q=q, k=k, v=v, o=o, lse=lse, k_lengths=torch.zeros(2, dtype=torch.int32), workspace=ws)
    for change in (dict(k=k.float()), dict(v=v[:, :6]), dict(k=k.transpose(1, 2)), dict(v=kv[:, :, 1, :, ::2]), dict(q=q[:, ::2]), dict(q=q[:1]),
                   dict(o=o[:, :, :2]), dict(o=o.float()), dict(lse=lse.double()), dict(lse=lse.transpose(1, 2)),
                   dict(k_lengths=torch.zeros(2, dtype=torch.int64)), dict(k_lengths=torch.zeros(3, dtype=torch.int32)),
                   dict(q=q.half(), k=k.half(), v=v.half()), dict(k=k.flip(1)[:, :, :, :32]),
                   dict()):                              # the last: everything right, but not on a GPU
        with pytest.raises(ValueError):
            B.gshard_cross_attention_forward(**{**ok, **change})
    grads = dict(dout=o, dq=torch.zeros_like(q), dk=torch.zeros(2, 7, 2, 64, dtype=bf), dv=torch.zeros(2, 7, 2, 64, dtype=bf))
    with pytest.raises(ValueError, match="dk"):          # laid out unlike k
        B.gshard_cross_attention_backward(**ok, **grads)


def _gated_fwd(n=4, K=64, cols=128, dtype=1, act=4, x=P[0], w=P[1], h=P[2], pre=P[3], ws=P[4], size=1 << 30):
    return B.load().gshard_gated_linear_forward(n, K, cols, dtype, act, x, w, h, pre, ws, size, None)


def _gated_bwd(n=4, K=64, cols=128, dtype=1, act=4, x=P[0], w=P[1], pre=P[2], dh=P[3], dx=P[4], dw=P[5], ws=P[6], size=1 << 30):
    return B.load().gshard_gated_linear_backward(n, K, cols, dtype, act, x, w, pre, dh, dx, dw, ws, size, None)


def test_gated_linear_arguments():
    sizes = ((dict(n=-1), INVALID), (dict(K=0), INVALID), (dict(cols=0), INVALID), (dict(K=60), SHAPE), (dict(cols=100), SHAPE),
             (dict(cols=(1 << 30)), SHAPE), (dict(cols=(1 << 31) - 8), SHAPE), (dict(dtype=2), INVALID), (dict(act=5), INVALID), (dict(act=-1), INVALID),
             (dict(n=(1 << 30) + 1), SHAPE))
    for kw, rc in sizes + ((dict(x=None), INVALID), (dict(w=None), INVALID), (dict(h=None), INVALID), (dict(pre=P[3] + 8), INVALID),
                           (dict(h=P[0]), INVALID), (dict(h=P[1]), INVALID), (dict(pre=P[2]), INVALID), (dict(ws=None), INVALID),
                           (dict(ws=P[4] + 16), INVALID), (dict(size=16), SMALL), (dict(n=0, x=None, w=None, h=None, ws=None), OK)):
        assert _gated_fwd(**kw) == rc, kw
    for kw, rc in sizes + ((dict(dh=None), INVALID), (dict(pre=None), INVALID), (dict(x=None), INVALID), (dict(w=None), INVALID),
                           (dict(dx=P[3]), INVALID), (dict(dw=P[2]), INVALID), (dict(dx=P[5]), INVALID), (dict(size=300), SMALL),
                           (dict(n=0, dw=None), OK)):
        assert _gated_bwd(**kw) == rc, kw
    assert B.gshard_gated_linear_workspace_bytes(4, 60, 64, torch.bfloat16) == 0
    assert B.gshard_gated_linear_workspace_bytes(4, 64, 64, torch.bfloat16) >= 256
    assert B.gshard_gated_linear_workspace_bytes(1000, 64, 64, torch.bfloat16, for_backward=True) >= 1000 * 128 * 2
    if not torch.cuda.is_available():
        assert _gated_fwd() in NO_GPU and _gated_fwd(pre=None, dtype=0) in NO_GPU
        assert _gated_bwd() in NO_GPU and _gated_bwd(dx=None, w=None) in NO_GPU and _gated_bwd(dw=None, x=None, dtype=0) in NO_GPU


def _list(grads, outs, counts, dtypes, n=None):
    n = len(counts) if n is None else n
    arrays = ((ctypes.c_void_p * len(counts))(*grads), (ctypes.c_void_p * len(counts))(*outs), (ctypes.c_int64 * len(counts))(*counts),
              (ctypes.c_int32 * len(counts))(*dtypes))
    types = (ctypes.POINTER(ctypes.c_void_p), ctypes.POINTER(ctypes.c_void_p), ctypes.POINTER(ctypes.c_int64), ctypes.POINTER(ctypes.c_int32))
    lst = B.gshard_grad_list(n, *[ctypes.cast(a, t) for a, t in zip(arrays, types)])
    lst.keep = arrays
    return lst


def test_grad_norm_arguments():
    lib = B.load()
    norm = lambda lst, sumsq=P[0], ws=P[1], size=1 << 30: lib.gshard_grad_norm(ctypes.byref(lst), sumsq, ws, size, None)
    clip = lambda lst, sumsq=P[0], bound=1.0, out=P[1]: lib.gshard_grad_clip(ctypes.byref(lst), sumsq, bound, out, None)
    good = _list([P[2], P[3] + 2], [P[2], P[4] + 2], [100, 7], [0, 1])
    bad = [_list([P[2]], [P[2]], [100], [2]), _list([P[2] + 2], [P[2]], [100], [0]), _list([P[2] + 1], [P[2]], [100], [1]), _list([None], [P[2]], [1], [0]),
           _list([P[2]], [P[2]], [-1], [0]), _list([P[2]], [P[2]], [1], [0], n=-1)]
    for lst in bad:
        assert norm(lst) == INVALID and clip(lst) == INVALID
        assert lib.gshard_grad_norm_workspace_bytes(ctypes.byref(lst)) == 0
    assert norm(_list([P[2]], [P[2]], [1 << 39], [0])) == SHAPE
    assert clip(_list([P[2]], [None], [1], [0])) == INVALID and clip(_list([P[2]], [P[3] + 2], [1], [0])) == INVALID
    assert norm(good, sumsq=None) == INVALID and norm(good, sumsq=P[0] + 4) == INVALID and norm(good, ws=None) == INVALID
    assert norm(good, ws=P[1] + 64) == INVALID and norm(good, size=8) == SMALL
    assert clip(good, sumsq=None) == INVALID and clip(good, out=P[1] + 2) == INVALID
    assert clip(good, bound=-1.0) == INVALID and clip(good, bound=math.nan) == INVALID
    assert lib.gshard_grad_norm_workspace_bytes(ctypes.byref(good)) >= 16
    if not torch.cuda.is_available():
        assert norm(good) in NO_GPU and clip(good) in NO_GPU and clip(good, out=None) in NO_GPU


def test_grad_list_checks_its_tensors():
    g = [torch.zeros(10), torch.zeros(4, 4, dtype=torch.bfloat16)]
    for grads, outs in ((g, g[:1]), (g, [g[0], g[1].float()]), (g, [g[0], torch.zeros(16, dtype=torch.bfloat16)]), ([g[0].double()], [g[0].double()]),
                        ([torch.zeros(4, 8)[:, ::2]], [torch.zeros(4, 4)])):
        with pytest.raises(ValueError):
            B.make_grad_list(grads, outs)
    flat = torch.zeros(100)
    a, b = flat[:60], flat[60:]
    for grads, outs in (([a, a], [a, a]), ([a, flat[59:]], [a, flat[59:]]), ([a, b], [b.new_zeros(60), a[:40]]), ([a, b], [b.new_zeros(60), a[20:]]),
                        ([a[:40], b], [b, a[:40]]), ([a, b], [flat.new_zeros(60), flat[59:99]])):
        with pytest.raises(ValueError, match="another tensor"):
            B.make_grad_list(grads, outs)
    for grads, outs in (([a, b], [a, b]), ([a, a], [flat.new_zeros(60), flat.new_zeros(60)]), ([a, b], [a, flat.new_zeros(40)]), ([b, a], [b, a]),
                        ([flat[:0], a], [flat[:0], a])):
        B.make_grad_list(grads, outs)
    lst = B.make_grad_list(g)
    assert lst.struct.n == 2 and lst.struct.counts[1] == 16 and lst.struct.grads[0] == lst.struct.outs[0] == g[0].data_ptr()
    with pytest.raises(ValueError, match="CUDA"):
        B.gshard_grad_norm(lst, torch.zeros(1, dtype=torch.float64), workspace=torch.zeros(512, dtype=torch.uint8))
