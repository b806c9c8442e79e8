"""Cases that time and check the operators around the MoE layer, next to their plain forms.

Three operators, each with its backward pass:

    layer norm   y = gamma (x - mean) / sqrt(var + eps) + beta over the last dimension, after the
                 residual connection of a sub-layer
    linear       y = act(x w + bias) + residual, the projections of a Transformer layer
    route        scores of the experts (softmax or sigmoid), the best k of them by score plus a
                 balancing bias, optionally inside the best groups of experts, and their weights

``run`` computes a case in plain torch operations, in 32 bits (the choice of experts in 64, where
near ties decide), or, with ``own`` true, through the library's binding.  ``exact`` is the same
definition in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTIVATIONS = ("none", "relu", "gelu", "gelu_tanh", "silu")
BIGGEST = torch.finfo(torch.float32).max


# ---- cases ------------------------------------------------------------------------------------

def _ln(name, direction, n, M, dtype, skip=False):
    return {"name": name, "op": "layer_norm", "direction": direction, "n": n, "M": M, "dtype": dtype, "skip": skip}


def _linear(name, direction, n, K, cols, dtype, act, bias=True, residual=False, pre=False, out="same"):
    return {"name": name, "op": "linear", "direction": direction, "n": n, "K": K, "cols": cols, "dtype": dtype,
            "act": act, "bias": bias, "residual": residual, "pre": pre, "out": out}


def _route(name, direction, G, S, E, k, dtype, score="softmax", bias=False, groups=1, kept=1, group_top=1,
           renorm=True, scale=1.0, mean=False, load=False, masked=False):
    return {"name": name, "op": "route", "direction": direction, "G": G, "S": S, "E": E, "k": k, "dtype": dtype,
            "score": score, "bias": bias, "groups": groups, "kept": kept, "group_top": group_top, "renorm": renorm,
            "scale": scale, "mean": mean, "load": load, "masked": masked}


def listed():
    return [
        # one token of a decoding step, model dimension of the paper's layers
        _ln("ln_fwd_token", "forward", 1, 1024, "bf16"),
        # the batch of the MoE(2048E) layer: 32 groups of 4096 tokens
        _ln("ln_fwd_batch", "forward", 131072, 1024, "bf16"),
        # training step of the MoE(512E) layer, the gradient of the skip connection added in
        _ln("ln_bwd_train", "backward", 65536, 1024, "bf16", skip=True),
        # float32 training with a row length that is no multiple of 16 bytes, ragged batch
        _ln("ln_bwd_odd", "backward", 9001, 2050, "f32"),
        # one token of a decoding step through the first projection of the feed-forward sub-layer
        _linear("linear_fwd_token", "forward", 1, 1024, 8192, "bf16", "gelu"),
        # second projection of the feed-forward sub-layer over 16 groups of 4096 tokens, with its skip connection
        _linear("linear_fwd_ffn_out", "forward", 65536, 8192, 1024, "bf16", "none", residual=True),
        # first projection's gradients, ragged batch (padding removed)
        _linear("linear_bwd_ffn_in", "backward", 30011, 1024, 8192, "bf16", "gelu"),
        # float32 training (the paper's precision), forward that keeps its pre-activations
        _linear("linear_fwd_f32", "forward", 4100, 1024, 4096, "f32", "relu", pre=True),
        # one token of a decoding step, 128 experts
        _route("route_fwd_token", "forward", 1, 1, 128, 2, "f32"),
        # the MoE(2048E) layer's batch: top-2 raw gates and the mean gates of the auxiliary loss
        _route("route_fwd_2048e", "forward", 32, 4096, 2048, 2, "f32", renorm=False, mean=True),
        # sigmoid scores, balancing bias, 4 of 8 groups, 8 experts a token, the load that moves the bias
        _route("route_fwd_grouped", "forward", 16, 4096, 512, 8, "bf16", "sigmoid", bias=True, groups=8, kept=4,
               group_top=2, scale=2.5, load=True, masked=True),
        # training step of the MoE(512E) layer: gradient of the weights and of the mean gates
        _route("route_bwd_512e", "backward", 16, 4096, 512, 2, "f32", mean=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("layer_norm", "linear", "route"))
    direction = rng.choice(("forward", "backward"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if op == "layer_norm":
        M = _log_int(rng, 16, 16384)
        if rng.random() < 0.5:
            M = max(16, M // 8 * 8)
        n = _log_int(rng, 1, max(1, min(131072, (1 << 27) // M // (2 if dtype == "f32" else 1))))
        return {k: v for k, v in _ln("", direction, n, M, dtype, direction == "backward" and rng.random() < 0.5).items()
                if k != "name"}
    if op == "linear":
        K = 8 * _log_int(rng, 2, 1024)
        cols = 8 * _log_int(rng, 2, 1024)
        room = (1 << 37 if dtype == "bf16" else 1 << 34) // (K * cols)
        n = _log_int(rng, 1, max(1, min(65536, room)))
        act = rng.choice(ACTIVATIONS)
        case = _linear("", direction, n, K, cols, dtype, act, bias=rng.random() < 0.7,
                       residual=direction == "forward" and rng.random() < 0.4,
                       pre=direction == "forward" and act != "none" and rng.random() < 0.5,
                       out="f32" if rng.random() < 0.25 else "same")
        return {k: v for k, v in case.items() if k != "name"}
    E = 2 * _log_int(rng, 4, 1024)
    divisors = [g for g in (2, 4, 8, 16, 32) if E % g == 0 and E // g >= 2]
    groups = rng.choice(divisors) if divisors and rng.random() < 0.5 else 1
    kept = rng.randint(1, groups)
    k = rng.randint(1, min(16, kept * (E // groups)))
    n = _log_int(rng, 1, min(131072, (1 << 28) // E))
    G = rng.choice((1, 1, 4, 16))
    case = _route("", direction, G, max(1, n // G), E, k, dtype, rng.choice(("softmax", "sigmoid")),
                  bias=rng.random() < 0.5, groups=groups, kept=kept, group_top=rng.choice((1, 2)),
                  renorm=rng.random() < 0.7, scale=rng.choice((1.0, 2.5)), mean=rng.random() < 0.5,
                  load=rng.random() < 0.5, masked=rng.random() < 0.4)
    return {k: v for k, v in case.items() if k != "name"}


# ---- inputs -----------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(gen, shape, dtype, std=1.0, mean=0.0):
    return (torch.randn(shape, generator=gen, device="cuda") * std + mean).to(dtype)


def _inputs(case, seed):
    gen = _gen(seed)
    dt = DTYPES[case["dtype"]]
    t = {}
    if case["op"] == "layer_norm":
        n, M = case["n"], case["M"]
        # a residual stream: a few features are far larger than the rest and off centre
        feature = torch.randn(M, generator=gen, device="cuda")
        spread = torch.where(feature.abs() > 2.5, 8.0, 1.0)
        t["x"] = (torch.randn(n, M, generator=gen, device="cuda") * spread + 0.3 * feature).to(dt)
        t["gamma"] = _randn(gen, M, torch.float32, 0.1, 1.0)
        t["beta"] = _randn(gen, M, torch.float32, 0.1)
        if case["direction"] == "backward":
            t["dy"] = _randn(gen, (n, M), dt)
            t["skip"] = _randn(gen, (n, M), dt) if case["skip"] else None
            x = t["x"].double()
            mean = x.mean(1)
            t["mean"] = mean.float()
            t["rstd"] = ((x - mean[:, None]).square().mean(1) + EPS).rsqrt().float()
    elif case["op"] == "linear":
        n, K, cols = case["n"], case["K"], case["cols"]
        odt = torch.float32 if case["out"] == "f32" else dt
        t["x"] = _randn(gen, (n, K), dt)
        t["w"] = _randn(gen, (K, cols), dt, K ** -0.5)
        t["bias"] = _randn(gen, cols, torch.float32, 0.1) if case["bias"] else None
        if case["direction"] == "forward":
            t["residual"] = _randn(gen, (n, cols), odt) if case["residual"] else None
        else:
            t["dy"] = _randn(gen, (n, cols), odt)
            # what the forward kept: unit-variance pre-activations
            t["pre"] = _randn(gen, (n, cols), odt) if case["act"] != "none" else None
    else:
        G, S, E, k = case["G"], case["S"], case["E"], case["k"]
        popular = 0.5 * torch.randn(E, generator=gen, device="cuda")
        logits = torch.randn(G, S, E, generator=gen, device="cuda") + popular
        if case["masked"]:      # padding tokens (no expert at all) and experts that a token may not use
            padding = torch.rand(G, S, 1, generator=gen, device="cuda") < 0.03
            barred = torch.rand(G, S, E, generator=gen, device="cuda") < 0.02
            logits = logits.masked_fill(padding | barred, -math.inf)
        t["logits"] = logits.to(dt)
        t["bias"] = _randn(gen, E, torch.float32, 0.05) if case["bias"] else None
        if case["direction"] == "backward":
            t["dweight"] = _randn(gen, (G, S, k), torch.float32)
            t["dmean"] = _randn(gen, (G, E), torch.float32) if case["mean"] else None
            t["expert_idx"] = _choose(case, t["logits"], t["bias"])
    return t


def prepare(case, seed):
    t = _inputs(case, seed)
    if not own:
        return {"case": case, "t": t}
    from paper_2006_16668_b200 import binding as B
    dt = DTYPES[case["dtype"]]
    out, handle = {}, None
    empty = lambda shape, dtype: torch.empty(shape, dtype=dtype, device="cuda")
    ws_bytes = 0
    if case["op"] == "layer_norm":
        n, M = case["n"], case["M"]
        if case["direction"] == "forward":
            out = {"y": empty((n, M), dt), "mean": empty(n, torch.float32), "rstd": empty(n, torch.float32)}
        else:
            out = {"dx": empty((n, M), dt), "dgamma": empty(M, torch.float32), "dbeta": empty(M, torch.float32)}
            ws_bytes = B.gshard_layer_norm_workspace_bytes(n, M)
    elif case["op"] == "linear":
        n, K, cols = case["n"], case["K"], case["cols"]
        odt = torch.float32 if case["out"] == "f32" else dt
        back = case["direction"] == "backward"
        if back:
            out = {"dx": empty((n, K), dt), "dw": empty((K, cols), dt),
                   "dbias": empty(cols, torch.float32) if case["bias"] else None}
        else:
            out = {"y": empty((n, cols), odt), "pre": empty((n, cols), odt) if case["pre"] else None}
        ws_bytes = B.gshard_linear_workspace_bytes(n, K, cols, dt, odt, for_backward=back)
    else:
        G, S, E, k = case["G"], case["S"], case["E"], case["k"]
        handle = B.make_route(G=G, S=S, E=E, k=k, dtype=case["dtype"], score=case["score"], groups=case["groups"],
                              groups_kept=case["kept"], group_top=case["group_top"], renormalise=case["renorm"],
                              scale=case["scale"])
        if case["direction"] == "forward":
            out = {"expert_idx": empty((G, S, k), torch.int32), "weight": empty((G, S, k), torch.float32),
                   "mean": empty((G, E), torch.float32) if case["mean"] else None,
                   "load": empty((G, E), torch.int32) if case["load"] else None}
            ws_bytes = B.gshard_moe_route_workspace_bytes(handle)
        else:
            out = {"dlogits": empty((G, S, E), dt)}
    return {"case": case, "t": t, "out": out, "handle": handle,
            "workspace": empty(ws_bytes, torch.uint8) if ws_bytes else None}


# ---- the operators through the library ----------------------------------------------------------

def _run_own(state):
    from paper_2006_16668_b200 import binding as B
    case, t, o, ws = state["case"], state["t"], state["out"], state["workspace"]
    forward = case["direction"] == "forward"
    if case["op"] == "layer_norm":
        if forward:
            B.gshard_layer_norm_forward(t["x"], t["gamma"], t["beta"], o["y"], o["mean"], o["rstd"], eps=EPS)
            return o["y"], o["mean"], o["rstd"]
        B.gshard_layer_norm_backward(t["x"], t["gamma"], t["mean"], t["rstd"], t["dy"], o["dx"], o["dgamma"],
                                     o["dbeta"], dskip=t["skip"], workspace=ws)
        return o["dx"], o["dgamma"], o["dbeta"]
    if case["op"] == "linear":
        if forward:
            B.gshard_linear_forward(t["x"], t["w"], o["y"], bias=t["bias"], residual=t["residual"], pre=o["pre"],
                                    activation=case["act"], workspace=ws)
            return _present(o["y"], o["pre"])
        B.gshard_linear_backward(t["x"], t["w"], t["dy"], o["dx"], o["dw"], o["dbias"], pre=t["pre"],
                                 activation=case["act"], workspace=ws)
        return _present(o["dx"], o["dw"], o["dbias"])
    if forward:
        B.gshard_moe_route(state["handle"], t["logits"], o["expert_idx"], o["weight"], bias=t["bias"], m=o["mean"],
                           load=o["load"], workspace=ws)
        return _present(o["expert_idx"], o["weight"], o["mean"], o["load"])
    B.gshard_moe_route_backward(state["handle"], t["logits"], t["expert_idx"], t["dweight"], o["dlogits"],
                                dm=t["dmean"])
    return (o["dlogits"],)


def _present(*tensors):
    return tuple(x for x in tensors if x is not None)


# ---- plain forms --------------------------------------------------------------------------------

def _act(v, act):
    if act == "relu":
        return torch.where(v > 0, v, torch.zeros_like(v))
    if act == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * (0.5 ** 0.5)))
    if act == "gelu_tanh":
        return 0.5 * v * (1.0 + torch.tanh((2.0 / math.pi) ** 0.5 * (v + 0.044715 * v * v * v)))
    if act == "silu":
        return v / (1.0 + torch.exp(-v))
    return v


def _act_grad(v, act):
    if act == "relu":
        return (v > 0).to(v.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(v * (0.5 ** 0.5))) + v * torch.exp(-0.5 * v * v) * (2.0 * math.pi) ** -0.5
    if act == "gelu_tanh":
        c = (2.0 / math.pi) ** 0.5
        u = torch.tanh(c * (v + 0.044715 * v * v * v))
        return 0.5 * (1.0 + u) + 0.5 * v * (1.0 - u * u) * c * (1.0 + 3 * 0.044715 * v * v)
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-v))
        return s * (1.0 + v * (1.0 - s))
    return torch.ones_like(v)


def _usable(logits):
    """A logit of -inf or NaN bars its expert for the token; +inf counts as the largest float."""
    l = logits.float()
    l = torch.where(torch.isnan(l), torch.full_like(l, -math.inf), l)
    return torch.where(l > BIGGEST, torch.full_like(l, BIGGEST), l)


def _scores(l, score):
    """Scores in l's precision: 0 for a barred expert, all 0 for a token with none left."""
    if score == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-l))
    top = l.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    e = torch.exp(l - top)
    total = e.sum(-1, keepdim=True)
    return e / torch.where(total > 0, total, torch.ones_like(total))


def _choose(case, logits, bias):
    """The k experts of each token, best first, ties to the lowest index; -1 where none is left.

    Without a bias a larger logit is a larger score, so that the logits themselves are compared;
    scores plus bias are compared in 64 bits."""
    l = _usable(logits)
    need_scores = bias is not None or (case["groups"] > 1 and case["group_top"] == 2)
    s = _scores(l.double(), case["score"]) if need_scores else None
    key = l if bias is None else torch.where(l == -math.inf, torch.full_like(s, -math.inf), s + bias.double())
    if case["groups"] > 1:
        g = case["groups"]
        value = key if s is None or bias is not None else torch.where(l == -math.inf, torch.full_like(s, -math.inf), s)
        value = value.reshape(*l.shape[:-1], g, -1)
        best = value.amax(-1)
        if case["group_top"] == 2 and value.shape[-1] > 1:
            rest = value.scatter(-1, value.argmax(-1, keepdim=True), -math.inf).amax(-1)
            best = torch.where(rest == -math.inf, best, best + rest)
        keep = torch.zeros_like(best, dtype=torch.bool)
        for _ in range(case["kept"]):
            at = best.argmax(-1, keepdim=True)
            keep.scatter_(-1, at, True)
            best = best.scatter(-1, at, -math.inf)
        keep = keep[..., None].expand_as(value).reshape(l.shape)
        key = torch.where(keep, key, torch.full_like(key, -math.inf))
    chosen = []
    for _ in range(case["k"]):
        at = key.argmax(-1, keepdim=True)
        value = key.gather(-1, at)
        chosen.append(torch.where(value == -math.inf, torch.full_like(at, -1), at))
        key = key.scatter(-1, at, -math.inf)
    return torch.cat(chosen, -1).to(torch.int32)


def _relative(l, idx, score):
    """Scores of the chosen experts over the largest of them, 0 where there is none (also where the
    scores themselves are too small for the type)."""
    there = idx >= 0
    pick = torch.where(there, l.gather(-1, idx.clamp(min=0).long()), torch.full_like(l[..., :1], -math.inf))
    top = pick.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    r = torch.exp(pick - top)
    if score == "sigmoid":
        r = torch.where(top < 0, r * (1.0 + torch.exp(top.clamp(max=0))) / (1.0 + torch.exp(pick.clamp(max=0))),
                        (1.0 + torch.exp(-top.clamp(min=0))) / (1.0 + torch.exp(-pick)))
    return torch.where(there, r, torch.zeros_like(r))


def _route_forward(case, t):
    l = _usable(t["logits"])
    idx = _choose(case, t["logits"], t["bias"])
    s = _scores(l, case["score"]) if case["mean"] or not case["renorm"] else None
    if case["renorm"]:
        r = _relative(l, idx, case["score"])
        total = r.sum(-1, keepdim=True)
        weight = case["scale"] * r / torch.where(total > 0, total, torch.ones_like(total))
    else:
        weight = case["scale"] * torch.where(idx >= 0, s.gather(-1, idx.clamp(min=0).long()), torch.zeros_like(s[..., :1]))
    mean = s.double().mean(1).float() if case["mean"] else None
    load = None
    if case["load"]:
        one = torch.zeros(case["G"], case["E"] + 1, dtype=torch.int32, device=l.device)
        at = torch.where(idx >= 0, idx, torch.full_like(idx, case["E"])).long().reshape(case["G"], -1)
        load = one.scatter_add_(1, at, torch.ones_like(at, dtype=torch.int32))[:, :-1].contiguous()
    return _present(idx, weight, mean, load)


def _route_backward(case, t):
    """Gradient of sum(dweight * weight) + sum(dmean * mean) with the choice held constant."""
    l = _usable(t["logits"])
    idx = t["expert_idx"]
    there, at = idx >= 0, idx.clamp(min=0).long()
    s = _scores(l, case["score"])
    dw = torch.where(there, t["dweight"], torch.zeros_like(t["dweight"]))
    dl = torch.zeros_like(l)
    if case["renorm"]:
        r = _relative(l, idx, case["score"])
        total = r.sum(-1, keepdim=True)
        w = r / torch.where(total > 0, total, torch.ones_like(total))
        # d weight_i / d log(score_j) = scale w_i (1[i = j] - w_j)
        g = case["scale"] * w * (dw - (dw * w).sum(-1, keepdim=True))
        if case["score"] == "sigmoid":
            g = g / (1.0 + torch.exp(l.gather(-1, at)))           # d log(sigmoid) = 1 - sigmoid
        dl.scatter_add_(-1, at, torch.where(there, g, torch.zeros_like(g)))
    ds = torch.zeros_like(l)
    if not case["renorm"]:
        ds.scatter_add_(-1, at, case["scale"] * dw)
    if case["mean"]:
        ds = ds + t["dmean"][:, None, :] / case["S"]
    if case["score"] == "softmax":
        dl = dl + s * (ds - (ds * s).sum(-1, keepdim=True))
    else:
        dl = dl + ds * s * (1.0 / (1.0 + torch.exp(l)))
    dl = torch.where(l == -math.inf, torch.zeros_like(dl), dl)
    return (dl.to(t["logits"].dtype),)


def _run_plain(state):
    case, t = state["case"], state["t"]
    forward = case["direction"] == "forward"
    if case["op"] == "layer_norm":
        x = t["x"].float()
        if forward:
            mean = x.mean(1)
            centred = x - mean[:, None]
            rstd = (centred.square().mean(1) + EPS).rsqrt()
            y = centred * rstd[:, None] * t["gamma"] + t["beta"]
            return y.to(t["x"].dtype), mean, rstd
        xhat = (x - t["mean"][:, None]) * t["rstd"][:, None]
        dy = t["dy"].float()
        g = dy * t["gamma"]
        dx = t["rstd"][:, None] * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
        if t["skip"] is not None:
            dx = dx + t["skip"].float()
        return dx.to(t["x"].dtype), (dy * xhat).sum(0), dy.sum(0)
    if case["op"] == "linear":
        x, w = t["x"].float(), t["w"].float()
        if forward:
            odt = torch.float32 if case["out"] == "f32" else t["x"].dtype
            pre = x @ w
            if t["bias"] is not None:
                pre = pre + t["bias"]
            y = _act(pre, case["act"])
            if t["residual"] is not None:
                y = y + t["residual"].float()
            return _present(y.to(odt), pre.to(odt) if case["pre"] else None)
        dpre = t["dy"].float()
        if case["act"] != "none":
            dpre = dpre * _act_grad(t["pre"].float(), case["act"])
        dx, dw = dpre @ w.T, x.T @ dpre
        return _present(dx.to(t["x"].dtype), dw.to(t["x"].dtype), dpre.sum(0) if case["bias"] else None)
    return _route_forward(case, t) if forward else _route_backward(case, t)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without ----------------------------------------------------------------

def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    forward = case["direction"] == "forward"
    if case["op"] == "layer_norm":
        n, M = case["n"], case["M"]
        if forward:
            return {"bytes": 2 * n * M * es + 8 * M + 8 * n, "flops": 8 * n * M}
        return {"bytes": (4 if case["skip"] else 3) * n * M * es + 12 * M + 8 * n, "flops": 14 * n * M}
    if case["op"] == "linear":
        n, K, cols = case["n"], case["K"], case["cols"]
        ys = 4 if case["out"] == "f32" else es
        if forward:
            rows = 1 + (1 if case["residual"] else 0) + (1 if case["pre"] else 0)
            return {"bytes": (n * K + K * cols) * es + rows * n * cols * ys + (4 * cols if case["bias"] else 0),
                    "flops": 2 * n * K * cols}
        rows = 1 + (1 if case["act"] != "none" else 0)
        return {"bytes": 2 * (n * K + K * cols) * es + rows * n * cols * ys + (4 * cols if case["bias"] else 0),
                "flops": 4 * n * K * cols}
    G, S, E, k = case["G"], case["S"], case["E"], case["k"]
    n = G * S
    if forward:
        extra = (4 * G * E if case["mean"] else 0) + (4 * G * E if case["load"] else 0) + (4 * E if case["bias"] else 0)
        return {"bytes": n * E * es + 8 * n * k + extra, "flops": 6 * n * E}
    return {"bytes": 2 * n * E * es + 8 * n * k + (4 * G * E if case["mean"] else 0), "flops": 8 * n * E}


# ---- the definitions in 64 bits -------------------------------------------------------------------

def _exact_route_choice(case, l, bias):
    """Order of preference by a stable sort of (score + bias), whole groups struck out first."""
    E = case["E"]
    barred = l == -math.inf
    plain = torch.sigmoid(l) if case["score"] == "sigmoid" else torch.softmax(l.masked_fill(barred.all(-1, keepdim=True), 0.0), -1)
    merit = l.clone() if bias is None else (plain + bias.double()).masked_fill(barred, -math.inf)
    if case["groups"] > 1:
        by_sum = case["group_top"] == 2
        value = (plain if bias is None else plain + bias.double()) if by_sum else merit
        value = value.masked_fill(barred, -math.inf).unflatten(-1, (case["groups"], E // case["groups"]))
        ranked = value.sort(dim=-1, descending=True).values[..., :2 if by_sum else 1]
        total = ranked.masked_fill(ranked == -math.inf, 0.0).sum(-1).masked_fill(ranked[..., 0] == -math.inf, -math.inf)
        order = total.sort(dim=-1, descending=True, stable=True).indices
        rank = torch.empty_like(order).scatter_(-1, order, torch.arange(case["groups"], device=l.device).expand_as(order))
        merit = merit.unflatten(-1, (case["groups"], -1)).masked_fill((rank >= case["kept"])[..., None], -math.inf).flatten(-2)
    ranked = merit.sort(dim=-1, descending=True, stable=True)
    idx = ranked.indices[..., :case["k"]]
    return idx.masked_fill(ranked.values[..., :case["k"]] == -math.inf, -1)


def _exact_route(case, t):
    raw = t["logits"].double()
    l = raw.nan_to_num(nan=-math.inf, posinf=BIGGEST, neginf=-math.inf)
    nothing = (l == -math.inf).all(-1, keepdim=True)
    logscore = torch.nn.functional.logsigmoid(l) if case["score"] == "sigmoid" else \
        torch.log_softmax(l.masked_fill(nothing, 0.0), -1).masked_fill(nothing, -math.inf)
    if case["direction"] == "forward":
        idx = _exact_route_choice(case, l, t["bias"])
        gone = idx < 0
        pick = logscore.gather(-1, idx.clamp(min=0)).masked_fill(gone, -math.inf)
        if case["renorm"]:
            pick = pick - torch.logsumexp(pick.masked_fill(gone.all(-1, keepdim=True), 0.0), -1, keepdim=True)
        weight = case["scale"] * pick.exp().masked_fill(gone, 0.0)
        mean = logscore.exp().mean(1) if case["mean"] else None
        load = None
        if case["load"]:
            load = torch.stack([torch.bincount(row[row >= 0], minlength=case["E"]) for row in idx.flatten(1)]).int()
        return _present(idx.int(), weight, mean, load)
    idx = t["expert_idx"].long()
    gone = idx < 0
    dw = t["dweight"].double().masked_fill(gone, 0.0)
    pick = logscore.gather(-1, idx.clamp(min=0)).masked_fill(gone, -math.inf)
    # gradient with respect to the log scores first, then through log softmax or log sigmoid
    if case["renorm"]:
        w = (pick - torch.logsumexp(pick.masked_fill(gone.all(-1, keepdim=True), 0.0), -1, keepdim=True)).exp()
        w = w.masked_fill(gone, 0.0)
        at_chosen = case["scale"] * (w * dw - w * (w * dw).sum(-1, keepdim=True))
    else:
        at_chosen = case["scale"] * dw * pick.exp()
    dlog = torch.zeros_like(l).scatter_add_(-1, idx.clamp(min=0), at_chosen)
    if case["mean"]:
        dlog = dlog + logscore.exp() * (t["dmean"].double() / case["S"])[:, None, :]
    if case["score"] == "softmax":
        dl = dlog - logscore.exp() * dlog.sum(-1, keepdim=True)
    else:
        dl = dlog * torch.sigmoid(-l)
    return (dl.masked_fill(l == -math.inf, 0.0),)


def exact(case, seed):
    t = _inputs(case, seed)
    forward = case["direction"] == "forward"
    if case["op"] == "route":
        return _exact_route(case, t)
    if case["op"] == "layer_norm":
        x = t["x"].double()
        gamma = t["gamma"].double()
        if forward:
            var, mean = torch.var_mean(x, dim=1, correction=0)
            rstd = 1.0 / torch.sqrt(var + EPS)
            return torch.addcmul(t["beta"].double(), (x - mean[:, None]) * rstd[:, None], gamma), mean, rstd
        # the mean and rstd that the forward kept are inputs of the backward
        z = (x - t["mean"].double()[:, None]) * t["rstd"].double()[:, None]
        dy = t["dy"].double()
        gy = dy * gamma
        dx = (gy - (gy.sum(1) / case["M"])[:, None] - z * ((gy * z).sum(1) / case["M"])[:, None]) * t["rstd"].double()[:, None]
        if t["skip"] is not None:
            dx += t["skip"].double()
        return dx, torch.einsum("nm,nm->m", dy, z), dy.sum(0)
    x, w = t["x"].double(), t["w"].double()
    act = case["act"]
    if forward:
        pre = torch.matmul(x, w)
        if t["bias"] is not None:
            pre += t["bias"].double()
        f = torch.nn.functional
        y = {"none": lambda v: v.clone(), "relu": f.relu, "gelu": f.gelu,
             "gelu_tanh": lambda v: f.gelu(v, approximate="tanh"), "silu": f.silu}[act](pre)
        if t["residual"] is not None:
            y += t["residual"].double()
        return _present(y, pre if case["pre"] else None)
    dpre = t["dy"].double()
    if act == "relu":
        dpre = dpre.masked_fill(t["pre"].double() <= 0, 0.0)
    elif act != "none":
        v = t["pre"].double().requires_grad_()
        f = torch.nn.functional
        a = {"gelu": f.gelu, "gelu_tanh": lambda u: f.gelu(u, approximate="tanh"), "silu": f.silu}[act](v)
        dpre = torch.autograd.grad(a, v, dpre)[0]
    return _present(torch.matmul(dpre, w.t()), torch.matmul(x.t(), dpre), dpre.sum(0) if case["bias"] else None)
