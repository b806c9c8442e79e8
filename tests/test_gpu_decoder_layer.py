"""The operators of a decoder layer as it uses them, in one piece and compared with automatic differentiation in 64 bits:

    a = LN(x),  q = a Wq,  [k, v] = e Wkv (encoder states e, padded),  x1 = x + attention(q, k, v) Wo,
    b = LN(x1),  h = act(b Wg) * (b Wu),  x2 = x1 + h Wd

forward, backward, the norm of all weight gradients and their clipping.  fp32 bounds: every operator is within a few 1e-6 of its
formula relative to the absolute terms (their own tests), a chain of eight of them within 5e-5 relative Frobenius; bf16 rounds about
ten tensors on the way (activations, P, dS, dpre, outputs), each at most 2^-9 rms of its values, so 2^-9 sqrt(10) = 6e-3 where
errors add independently; twice that and more is left for gradients in which large terms cancel: 2.5e-2."""
import pytest
import torch

from operator_reference import activation, layer_norm
from paper_2006_16668_b200 import binding as B

pytestmark = pytest.mark.gpu

EPS = 1e-5


def _fro(got, want):
    return float((got.double() - want).norm() / want.norm())


def _new(*shape, dtype=torch.float32):
    return torch.full(shape, float("nan"), device="cuda").to(dtype)


def _bytes(n):
    return torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")


class Layer:
    """The layer's calls on flat activations [batch * tokens, M]."""

    def __init__(self, M, H, Hkv, D, F, act, w):
        self.M, self.H, self.Hkv, self.D, self.F, self.act, self.w = M, H, Hkv, D, F, act, w

    def linear(self, x, w, residual=None):
        n, K = x.shape
        y = _new(n, w.shape[1], dtype=x.dtype)
        B.gshard_linear_forward(x, w, y, residual=residual, workspace=_bytes(B.gshard_linear_workspace_bytes(n, K, w.shape[1], x.dtype)))
        return y

    def linear_back(self, x, w, dy):
        dx, dw = torch.empty_like(x), torch.empty_like(w)
        B.gshard_linear_backward(x, w, dy, dx, dw, workspace=_bytes(B.gshard_linear_workspace_bytes(*x.shape, w.shape[1], x.dtype, for_backward=True)))
        return dx, dw

    def norm(self, x, gamma, beta):
        y, mean, rstd = torch.empty_like(x), _new(x.shape[0]), _new(x.shape[0])
        B.gshard_layer_norm_forward(x, gamma, beta, y, mean, rstd, eps=EPS)
        return y, mean, rstd

    def norm_back(self, x, gamma, mean, rstd, dy, dskip):
        dx, dg, db = torch.empty_like(x), _new(self.M), _new(self.M)
        B.gshard_layer_norm_backward(x, gamma, mean, rstd, dy, dx, dg, db, dskip=dskip, workspace=_bytes(B.gshard_layer_norm_workspace_bytes(*x.shape)))
        return dx, dg, db

    def attention_args(self, q, kv, batch):
        Tq, Tk = q.shape[0] // batch, kv.shape[0] // batch
        kv = kv.reshape(batch, Tk, 2, self.Hkv, self.D)
        return q.reshape(batch, Tq, self.H, self.D), kv[:, :, 0], kv[:, :, 1]

    def attention(self, q, kv, lengths):
        q, k, v = self.attention_args(q, kv, len(lengths))
        o, lse = torch.empty_like(q), _new(q.shape[0], self.H, q.shape[1])
        ws = _bytes(B.gshard_cross_attention_workspace_bytes(*q.shape[:2], k.shape[1], self.H, self.Hkv, self.D, q.dtype))
        B.gshard_cross_attention_forward(q, k, v, o, lse=lse, k_lengths=lengths, workspace=ws)
        return o.reshape(-1, self.H * self.D), lse

    def attention_back(self, q, kv, lengths, o, lse, do):
        q4, k, v = self.attention_args(q, kv, len(lengths))
        dq, dkv = torch.empty_like(q), torch.empty_like(kv)
        dq4, dk, dv = self.attention_args(dq, dkv, len(lengths))
        ws = _bytes(B.gshard_cross_attention_workspace_bytes(*q4.shape[:2], k.shape[1], self.H, self.Hkv, self.D, q.dtype, for_backward=True))
        B.gshard_cross_attention_backward(q4, k, v, o.reshape(q4.shape), lse, do.reshape(q4.shape), dq4, dk, dv, k_lengths=lengths, workspace=ws)
        return dq, dkv

    def forward(self, x, e, lengths):
        w, s = self.w, {}
        s["a"], s["mean1"], s["rstd1"] = self.norm(x, w["g1"], w["b1"])
        s["q"], s["kv"] = self.linear(s["a"], w["wq"]), self.linear(e, w["wkv"])
        s["o"], s["lse"] = self.attention(s["q"], s["kv"], lengths)
        s["x1"] = self.linear(s["o"], w["wo"], residual=x)
        s["b"], s["mean2"], s["rstd2"] = self.norm(s["x1"], w["g2"], w["b2"])
        n = x.shape[0]
        s["h"], s["pre"] = _new(n, self.F, dtype=x.dtype), _new(n, 2 * self.F, dtype=x.dtype)
        B.gshard_gated_linear_forward(s["b"], w["wgu"], s["h"], pre=s["pre"], activation=self.act,
                                      workspace=_bytes(B.gshard_gated_linear_workspace_bytes(n, self.M, self.F, x.dtype)))
        return self.linear(s["h"], w["wd"], residual=s["x1"]), s

    def backward(self, x, e, lengths, s, dy):
        w, g = self.w, {}
        dh, g["wd"] = self.linear_back(s["h"], w["wd"], dy)
        db, g["wgu"] = torch.empty_like(s["b"]), torch.empty_like(w["wgu"])
        B.gshard_gated_linear_backward(s["b"], w["wgu"], s["pre"], dh, db, g["wgu"], activation=self.act,
                                       workspace=_bytes(B.gshard_gated_linear_workspace_bytes(x.shape[0], self.M, self.F, x.dtype, for_backward=True)))
        dx1, g["g2"], g["b2"] = self.norm_back(s["x1"], w["g2"], s["mean2"], s["rstd2"], db, dy)
        do, g["wo"] = self.linear_back(s["o"], w["wo"], dx1)
        dq, dkv = self.attention_back(s["q"], s["kv"], lengths, s["o"], s["lse"], do)
        de, g["wkv"] = self.linear_back(e, w["wkv"], dkv)
        da, g["wq"] = self.linear_back(s["a"], w["wq"], dq)
        dx, g["g1"], g["b1"] = self.norm_back(x, w["g1"], s["mean1"], s["rstd1"], da, dx1)
        return dx, de, g


def _make(batch, Tq, Tk, M, H, Hkv, D, F, act, dtype):
    gen = torch.Generator(device="cuda").manual_seed(batch * Tq + Tk + F)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    w = {"g1": 1 + 0.1 * r(M), "b1": 0.1 * r(M), "g2": 1 + 0.1 * r(M), "b2": 0.1 * r(M)}
    for name, K, cols in (("wq", M, H * D), ("wkv", M, 2 * Hkv * D), ("wo", H * D, M), ("wgu", M, 2 * F), ("wd", F, M)):
        w[name] = (r(K, cols) * K ** -0.5).to(dtype)
    return Layer(M, H, Hkv, D, F, act, w), r(batch * Tq, M).to(dtype), r(batch * Tk, M).to(dtype), r(batch * Tq, M).to(dtype)


def _exact(layer, p, x, e, lengths, batch):
    H, Hkv, D = layer.H, layer.Hkv, layer.D
    a = layer_norm(x, p["g1"], p["b1"], EPS)[0]
    q = (a @ p["wq"]).reshape(batch, -1, H, D).transpose(1, 2)
    kv = (e @ p["wkv"]).reshape(batch, -1, 2, Hkv, D)
    k, v = (kv[:, :, i].transpose(1, 2).repeat_interleave(H // Hkv, 1) for i in (0, 1))
    out = []
    for b, n in enumerate(lengths):                     # a source without tokens adds nothing
        s = torch.softmax(q[b] @ k[b, :, :n].transpose(-1, -2) * D ** -0.5, -1) @ v[b, :, :n] if n else torch.zeros_like(q[b])
        out.append(s.transpose(0, 1).reshape(-1, H * D))
    x1 = x + torch.cat(out) @ p["wo"]
    pre = layer_norm(x1, p["g2"], p["b2"], EPS)[0] @ p["wgu"]
    return x1 + (activation(pre[:, :layer.F], layer.act) * pre[:, layer.F:]) @ p["wd"]


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 5e-5), (torch.bfloat16, 2.5e-2)])
@pytest.mark.parametrize("batch,Tq,Tk,M,H,Hkv,D,F,act,lengths", [(3, 70, 90, 256, 4, 2, 64, 344, "silu", [90, 0, 33]),
                                                                 (2, 300, 257, 512, 4, 4, 128, 1024, "gelu", [200, 257])])
def test_training_step_of_a_decoder_layer(batch, Tq, Tk, M, H, Hkv, D, F, act, lengths, dtype, tol):
    layer, x, e, dy = _make(batch, Tq, Tk, M, H, Hkv, D, F, act, dtype)
    n_keys = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    y, saved = layer.forward(x, e, n_keys)
    dx, de, grads = layer.backward(x, e, n_keys, saved, dy)
    p = {k: t.double().detach().requires_grad_() for k, t in {**layer.w, "x": x, "e": e}.items()}
    want = _exact(layer, p, p["x"], p["e"], lengths, batch)
    (want * dy.double()).sum().backward()
    assert _fro(y, want.detach()) < tol
    for name, got in {**grads, "x": dx, "e": de}.items():
        assert _fro(got, p[name].grad) < tol, "d" + name
    # all weight gradients together, scaled to a tenth of their norm
    names = sorted(grads)
    before = [grads[k].clone() for k in names]
    lst = B.make_grad_list([grads[k] for k in names])
    sumsq, norm = torch.empty(1, dtype=torch.float64, device="cuda"), torch.empty(1, device="cuda")
    exact = sum(float(g.double().square().sum()) for g in before) ** 0.5
    B.gshard_grad_norm(lst, sumsq, workspace=_bytes(B.gshard_grad_norm_workspace_bytes(lst)))
    B.gshard_grad_clip(lst, sumsq, 0.1 * exact, norm=norm)
    assert abs(float(norm) - exact) < 1e-6 * exact
    for k, b in zip(names, before):
        assert _fro(grads[k], 0.1 * b.double()) < (1e-6 if grads[k].dtype == torch.float32 else 2.0 ** -8), k


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 2e-5), (torch.bfloat16, 2e-2)])
def test_a_decoding_step_agrees_with_the_training_forward(dtype, tol):
    """One token per sentence through the same layer, the encoder's keys and values projected once."""
    batch, Tq, Tk, lengths = 4, 12, 150, [150, 1, 77, 128]
    layer, x, e, _ = _make(batch, Tq, Tk, 256, 8, 2, 64, 512, "gelu", dtype)
    n_keys = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    y, saved = layer.forward(x, e, n_keys)
    w, kv = layer.w, saved["kv"]
    for t in (0, Tq - 1):
        xt = x.reshape(batch, Tq, -1)[:, t].contiguous()
        a, _, _ = layer.norm(xt, w["g1"], w["b1"])
        o, _ = layer.attention(layer.linear(a, w["wq"]), kv, n_keys)
        x1 = layer.linear(o, w["wo"], residual=xt)
        b, _, _ = layer.norm(x1, w["g2"], w["b2"])
        h = _new(batch, layer.F, dtype=dtype)
        B.gshard_gated_linear_forward(b, w["wgu"], h, activation="gelu",
                                      workspace=_bytes(B.gshard_gated_linear_workspace_bytes(batch, layer.M, layer.F, dtype)))
        yt = layer.linear(h, w["wd"], residual=x1)
        assert _fro(yt, y.reshape(batch, Tq, -1)[:, t].double()) < tol
