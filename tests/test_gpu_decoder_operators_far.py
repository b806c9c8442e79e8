"""Gradients whose operands lie beyond 2^31 elements: every address of the backward passes, against the formula in 64 bits."""
import pytest
import torch

import decoder_reference as ref
import test_gpu_cross_attention as attn
from operator_reference import within
from paper_2006_16668_b200 import binding as B

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
NAN = float("nan")


@pytest.mark.parametrize("dtype,Tq", [(BF, 40), (BF, 700), (F32, 5), (F32, 40)])
def test_attention_gradients_beyond_31_bits(dtype, Tq):
    Bn, Tk, H, D = 3, 8192, 2, 64
    stride = 90 * 1024                                # of a token: 3 x 8192 x 92160 = 2.26e9 elements
    gen = torch.Generator(device="cuda").manual_seed(1)
    rows = lambda: torch.empty(Bn * Tk * stride, dtype=dtype, device="cuda").as_strided((Bn, Tk, 2, H, D), (Tk * stride, stride, H * D, D, 1))
    kv, grads = rows(), rows()
    kv.copy_(torch.randn(Bn, Tk, 2, H, D, generator=gen, device="cuda"))
    grads.fill_(NAN)
    r = lambda: torch.randn(Bn, Tq, H, D, generator=gen, device="cuda").to(dtype)
    t = {"q": r(), "dout": r(), "k": kv[:, :, 0], "v": kv[:, :, 1], "given": True,
         "lengths": torch.tensor([Tk, 5000, Tk - 1], dtype=torch.int32, device="cuda")}
    o, lse = attn.forward(t)
    attn.check_forward(t, o, lse)
    dq = torch.full_like(t["q"], NAN)
    ws = attn.workspace(t, True)
    B.gshard_cross_attention_backward(t["q"], t["k"], t["v"], o, lse, t["dout"], dq, grads[:, :, 0], grads[:, :, 1], k_lengths=t["lengths"], workspace=ws)
    assert B.gshard_moe_last_device_status(ws) == B.GSHARD_OK
    attn.check_backward(t, o, lse, (dq, grads[:, :, 0], grads[:, :, 1]))


def test_gated_weight_gradient_beyond_31_bits():
    n, K, cols = 140000, 64, 8192                         # pre: 2.3e9 elements
    gen = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda", dtype=BF)
    x, w, pre, dh = r(n, K), r(K, 2 * cols) / 8, r(n, 2 * cols), r(n, cols)
    dx, dw = torch.full_like(x, NAN), torch.full_like(w, NAN)
    ws = torch.empty(B.gshard_gated_linear_workspace_bytes(n, K, cols, BF, for_backward=True), dtype=torch.uint8, device="cuda")
    B.gshard_gated_linear_backward(x, w, pre, dh, dx, dw, activation="silu", workspace=ws)
    assert B.gshard_moe_last_device_status(ws) == B.GSHARD_OK
    some = torch.tensor([0, 1, 127, 128, 4095, 5001, 8191], device="cuda")
    both = torch.cat((some, cols + some))
    value, bound = ref.gated_grad(x, w[:, both], pre[:, both], dh[:, some], "silu")[1]
    within(dw[:, both], value, bound, "dw")
    assert torch.isfinite(dw).all()
    rows = torch.tensor([0, 70000, 131072, n - 1], device="cuda")
    value, bound = ref.gated_grad(x[rows], w, pre[rows], dh[rows], "silu")[0]
    within(dx[rows], value, bound, "dx")
