"""Layer norm, linear and routing as a Transformer layer uses them, next to the stages of the MoE layer.

The sub-layer  o = x + W2 gelu(W1 LN(x) + b1) + b2  with a router on LN(x) beside it is run forward and backward in one
piece and compared with automatic differentiation in 64 bits; then the router's choice feeds the MoE
stages.  fp32 bounds: every operator is within a few 1e-6 of its formula relative to the absolute terms
(their own tests), a chain of five of them with sums over at most 512 terms within 2e-5 relative Frobenius; bf16
rounds about six tensors on the way (activations, dpre, outputs), each at most 2^-9 rms of its values: 2e-2."""
import pytest
import torch

from operator_reference import choose, layer_norm, log_scores, route_weights, scores
from paper_2006_16668_b200 import binding as B

pytestmark = pytest.mark.gpu

EPS = 1e-5


def _fro(got, want):
    return float((got.double() - want).norm() / want.norm())


def _empty(*shape, dtype=torch.float32):
    return torch.full(shape, float("nan"), device="cuda").to(dtype)


def _workspace(n, K, cols, dtype, out=None, back=False):
    return torch.empty(B.gshard_linear_workspace_bytes(n, K, cols, dtype, out, for_backward=back), dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 2e-5), (torch.bfloat16, 2e-2)])
@pytest.mark.parametrize("G,S,M,H,E,k,score", [(2, 100, 128, 512, 32, 2, "softmax"), (4, 257, 256, 512, 48, 4, "sigmoid")])
def test_sublayer_and_router_forward_and_backward(G, S, M, H, E, k, score, dtype, tol):
    n = G * S
    gen = torch.Generator(device="cuda").manual_seed(n + E)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    x, gamma, beta = r(n, M).to(dtype), 1 + 0.1 * r(M), 0.1 * r(M)
    w1, b1 = (r(M, H) * M ** -0.5).to(dtype), 0.1 * r(H)
    w2, b2 = (r(H, M) * H ** -0.5).to(dtype), 0.1 * r(M)
    wg, balance = (r(M, E) * M ** -0.5).to(dtype), 0.02 * r(E)
    do, dweight, dm = r(n, M).to(dtype), r(G, S, k), r(G, E)

    # forward
    a, mean, rstd = _empty(n, M, dtype=dtype), _empty(n), _empty(n)
    B.gshard_layer_norm_forward(x, gamma, beta, a, mean, rstd, eps=EPS)
    f, pre, o = _empty(n, H, dtype=dtype), _empty(n, H, dtype=dtype), _empty(n, M, dtype=dtype)
    B.gshard_linear_forward(a, w1, f, bias=b1, pre=pre, activation="gelu", workspace=_workspace(n, M, H, dtype))
    B.gshard_linear_forward(f, w2, o, bias=b2, residual=x, workspace=_workspace(n, H, M, dtype))
    logits = _empty(n, E)
    B.gshard_linear_forward(a, wg, logits, workspace=_workspace(n, M, E, dtype, torch.float32))
    cfg = B.make_route(G=G, S=S, E=E, k=k, score=score)
    idx, weight, m = torch.empty(G, S, k, dtype=torch.int32, device="cuda"), _empty(G, S, k), _empty(G, E)
    load = torch.empty(G, E, dtype=torch.int32, device="cuda")
    B.gshard_moe_route(cfg, logits.reshape(G, S, E), idx, weight, bias=balance, m=m, load=load,
                       workspace=torch.empty(B.gshard_moe_route_workspace_bytes(cfg), dtype=torch.uint8, device="cuda"))
    # backward
    dlogits = _empty(G, S, E)
    B.gshard_moe_route_backward(cfg, logits.reshape(G, S, E), idx, dweight, dlogits, dm=dm)
    da_router, dwg = _empty(n, M, dtype=dtype), _empty(M, E, dtype=dtype)
    B.gshard_linear_backward(a, wg, dlogits.reshape(n, E), da_router, dwg, workspace=_workspace(n, M, E, dtype, torch.float32, True))
    df, dw2, db2 = _empty(n, H, dtype=dtype), _empty(H, M, dtype=dtype), _empty(M)
    B.gshard_linear_backward(f, w2, do, df, dw2, db2, workspace=_workspace(n, H, M, dtype, back=True))
    da, dw1, db1 = _empty(n, M, dtype=dtype), _empty(M, H, dtype=dtype), _empty(H)
    B.gshard_linear_backward(a, w1, df, da, dw1, db1, pre=pre, activation="gelu", workspace=_workspace(n, M, H, dtype, back=True))
    da = (da.float() + da_router.float()).to(dtype)
    dx, dgamma, dbeta = _empty(n, M, dtype=dtype), _empty(M), _empty(M)
    B.gshard_layer_norm_backward(x, gamma, mean, rstd, da, dx, dgamma, dbeta, dskip=do,
                                 workspace=torch.empty(B.gshard_layer_norm_workspace_bytes(n, M), dtype=torch.uint8, device="cuda"))

    # the same in 64 bits, on the experts that were chosen
    p = {name: t.double().detach().requires_grad_() for name, t in
         dict(x=x, gamma=gamma, beta=beta, w1=w1, b1=b1, w2=w2, b2=b2, wg=wg).items()}
    ra = layer_norm(p["x"], p["gamma"], p["beta"], EPS)[0]
    rf = torch.nn.functional.gelu(ra @ p["w1"] + p["b1"])
    ro = p["x"] + rf @ p["w2"] + p["b2"]
    rl = ra @ p["wg"]
    chosen = idx.reshape(n, k).long()
    rw = route_weights(rl, chosen, score, True, 1.0)
    rm = scores(rl, score).reshape(G, S, E).mean(1)
    loss = (ro * do.double()).sum() + (rw * dweight.reshape(n, k).double()).sum() + (rm * dm.double()).sum()
    loss.backward()
    # the choice itself, on the logits as the router saw them
    assert torch.equal(chosen.cpu(), choose(logits, balance, k=k, score=score))
    assert torch.equal(load.long(), torch.stack([torch.bincount(row, minlength=E) for row in chosen.reshape(G, -1)]))
    for name, got, want in (("o", o, ro), ("logits", logits, rl), ("weight", weight.reshape(n, k), rw), ("m", m, rm)):
        assert _fro(got, want.detach()) < tol, name
    for name, got in (("x", dx), ("gamma", dgamma), ("beta", dbeta), ("w1", dw1), ("b1", db1), ("w2", dw2), ("b2", db2),
                      ("wg", dwg)):
        assert _fro(got, p[name].grad) < tol, "d" + name


def test_sigmoid_router_with_bias_feeds_the_moe_stages():
    """Sigmoid scores with a balancing bias and groups choose two experts per token; capacity, dispatch, expert FFN
    and combine then run on that choice, and a layer norm closes the sub-layer."""
    G, S, M, H, E = 2, 192, 64, 256, 16
    C = S                                                  # room for every token: nothing is dropped
    shape = B.make_shape(G=G, S=S, M=M, H=H, E=E, C=C, dtype="f32")
    gen = torch.Generator(device="cuda").manual_seed(6)
    r = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    x, wg, balance = r(G, S, M), r(M, E) * M ** -0.5, 0.1 * r(E)
    wi, wo = r(E, M, H) * M ** -0.5, r(E, H, M) * H ** -0.5
    n = G * S
    logits = _empty(n, E)
    B.gshard_linear_forward(x.reshape(n, M), wg, logits, workspace=_workspace(n, M, E, torch.float32))
    kw = dict(score="sigmoid", groups=4, groups_kept=2, group_top=2, renormalise=False)
    cfg = B.make_route(G=G, S=S, E=E, k=2, **kw)
    idx, g12, m = torch.empty(G, S, 2, dtype=torch.int32, device="cuda"), _empty(G, S, 2), _empty(G, E)
    B.gshard_moe_route(cfg, logits.reshape(G, S, E), idx, g12, bias=balance, m=m,
                       workspace=torch.empty(B.gshard_moe_route_workspace_bytes(cfg), dtype=torch.uint8, device="cuda"))
    ws = B.alloc_workspace(shape)
    rt, rs = B.alloc_routing(shape)
    l_aux = torch.zeros(1, device="cuda")
    u = torch.zeros(G, S, device="cuda")                   # every second choice passes the random test
    B.gshard_moe_capacity(shape, idx, g12, u, m, rs, l_aux, ws)
    buf, out, y = _empty(E, G * C, M), _empty(E, G * C, M), _empty(G, S, M)
    B.gshard_moe_dispatch(shape, x, rt["slot_token"], buf)
    B.gshard_moe_expert_ffn(shape, buf, wi, wo, out, ws)
    B.gshard_moe_combine(shape, out, idx, rt["slot"], rt["weight"], y)
    h, z = (x + y).reshape(n, M), _empty(n, M)
    B.gshard_layer_norm_forward(h, torch.ones(M, device="cuda"), None, z, eps=EPS)

    want_idx = choose(logits, balance, k=2, score="sigmoid", groups=4, groups_kept=2, group_top=2).cuda()
    assert torch.equal(idx.reshape(n, 2).long(), want_idx)
    g = log_scores(logits.double(), "sigmoid").exp().gather(-1, want_idx)
    w = g / g.sum(-1, keepdim=True)
    xd, yd = x.reshape(n, M).double(), torch.zeros(n, M, dtype=torch.float64, device="cuda")
    for e in range(E):
        f = torch.relu(xd @ wi[e].double()) @ wo[e].double()
        yd += (w * (want_idx == e)).sum(-1, keepdim=True) * f
    assert _fro(y.reshape(n, M), yd) < 1e-5
    assert _fro(z, layer_norm(xd + yd, torch.ones(M, device="cuda"), None, EPS)[0]) < 1e-5
