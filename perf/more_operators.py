"""Cases that time and check the operators of a decoder layer and its training step, next to their plain forms.

    cross attention   o = softmax(scale q k^T) v over the states of an encoder, padded to a common length
    gated linear      h = act(x w_gate) * (x w_up), the first half of a gated feed-forward block
    gradient norm     the norm of all gradients together, and their clipping to a bound

Cross attention and gated linear have their backward passes.  ``run`` computes a case in plain torch
operations, in 32 bits (long sums of squares in 64), or, with ``own`` true, through the library's binding.
``exact`` is the same definition in 64 bits.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTIVATIONS = ("none", "relu", "gelu", "gelu_tanh", "silu")


# ---- cases ------------------------------------------------------------------------------------

def _attention(name, direction, B, Tq, Tk, H, Hkv, D, dtype, lse=False, empty=False, fused=True):
    """fused: k and v are the two halves of one projection's output; empty: a source may have no token."""
    return {"name": name, "op": "attention", "direction": direction, "B": B, "Tq": Tq, "Tk": Tk, "H": H, "Hkv": Hkv, "D": D,
            "dtype": dtype, "lse": lse, "empty": empty, "fused": fused}


def _gated(name, direction, n, K, cols, dtype, act, pre=False):
    return {"name": name, "op": "gated", "direction": direction, "n": n, "K": K, "cols": cols, "dtype": dtype, "act": act,
            "pre": pre}


def _norm(name, tensors, elements, dtype, ratio, in_place):
    """ratio: norm over bound; above 1 the gradients are scaled down."""
    return {"name": name, "op": "grad_norm", "tensors": tensors, "elements": elements, "dtype": dtype, "ratio": ratio,
            "in_place": in_place}


def listed():
    return [
        # one decoding step of one sentence: 16 heads of 128 as in the paper's layers, a source of 200 tokens
        _attention("attn_fwd_token", "forward", 1, 1, 200, 16, 16, 128, "bf16"),
        # a decoding step of 96 sentences over ragged sources, some slots of the batch empty
        _attention("attn_fwd_decode", "forward", 96, 1, 1024, 16, 16, 128, "bf16", empty=True),
        # training batch of 64 pairs of 1024 tokens, ragged sources
        _attention("attn_fwd_train", "forward", 64, 1024, 1024, 16, 16, 128, "bf16", lse=True),
        # its gradients, at lengths off every tile, queries sharing keys four to one
        _attention("attn_bwd_train", "backward", 32, 1000, 1111, 16, 4, 128, "bf16"),
        # float32 training (the paper's precision), heads of 64
        _attention("attn_bwd_f32", "backward", 8, 517, 333, 16, 16, 64, "f32"),
        # one token of a decoding step through the first half of a gated feed-forward block
        _gated("gated_fwd_token", "forward", 1, 1024, 4096, "bf16", "silu"),
        # 16 groups of 4096 tokens, the forward of a training step
        _gated("gated_fwd_train", "forward", 65536, 1024, 8192, "bf16", "gelu", pre=True),
        # its gradients, ragged batch (padding removed)
        _gated("gated_bwd_train", "backward", 30011, 1024, 8192, "bf16", "gelu"),
        # float32 training, an inner width of two thirds of 4 x 1024, rounded to a multiple of 8
        _gated("gated_fwd_f32", "forward", 4100, 1024, 2736, "f32", "silu", pre=True),
        # the small parameters of a decoder layer (norms, biases), under the bound: nothing to scale
        _norm("norm_small", 18, 60011, "f32", 0.5, True),
        # every gradient of a 12-layer decoder, weights in bf16 and norms in float32, over the bound
        _norm("norm_decoder", 160, 400000003, "mixed", 3.0, False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("attention", "attention", "gated", "gated", "grad_norm"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if op == "attention":
        H = rng.choice((1, 4, 8, 16))
        Hkv = H // rng.choice([g for g in (1, 1, 2, 4, 8) if H % g == 0])
        D = rng.choice((64, 128, 128, 8 * rng.randint(1, 16)))
        form = rng.choice(("decode", "forward", "backward"))
        room = (1 << 30) if dtype == "bf16" else (1 << 25)      # scores
        if form == "decode":
            Tq, Tk = rng.choice((1, 1, rng.randint(1, 8))), _log_int(rng, 1, 32768)
            B = _log_int(rng, 1, max(1, min(256, (1 << 28) // (Tk * Hkv * D))))
        else:
            Tk = _log_int(rng, 1, 4096)
            Tq = _log_int(rng, 1, 4096)
            B = _log_int(rng, 1, max(1, min(64, room // (2 if form == "backward" else 1) // (H * Tq * Tk))))
        back = form == "backward"
        case = _attention("", "backward" if back else "forward", B, Tq, Tk, H, Hkv, D, dtype,
                          lse=form == "forward" and rng.random() < 0.5, empty=form == "decode" and rng.random() < 0.5,
                          fused=rng.random() < 0.5)
    elif op == "gated":
        direction = rng.choice(("forward", "backward"))
        K = 8 * _log_int(rng, 2, 1024)
        cols = 8 * _log_int(rng, 2, 1024)
        room = (1 << 38 if dtype == "bf16" else 1 << 34) // (K * cols)
        n = _log_int(rng, 1, max(1, min(65536, room)))
        case = _gated("", direction, n, K, cols, dtype, rng.choice(ACTIVATIONS),
                      pre=direction == "forward" and rng.random() < 0.5)
    else:
        tensors = _log_int(rng, 1, 700)
        case = _norm("", tensors, tensors + _log_int(rng, 1, 390000000), rng.choice(("bf16", "f32", "mixed")),
                     rng.choice((0.3, 0.9, 1.5, 40.0)), False)
        case["in_place"] = case["ratio"] < 1 and rng.random() < 0.5
    return {k: v for k, v in case.items() if k != "name"}


# ---- inputs -----------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(gen, shape, dtype, std=1.0, mean=0.0):
    return (torch.randn(shape, generator=gen, device="cuda") * std + mean).to(dtype)


def _tensor_sizes(case):
    """Elements and types of the gradients, spread over three orders of magnitude."""
    rng = random.Random(case["tensors"] * 1000003 + case["elements"])
    share = [10 ** rng.uniform(-3, 0) for _ in range(case["tensors"])]
    left = case["elements"] - case["tensors"]
    sizes = [1 + int(left * s / sum(share)) for s in share]
    sizes[-1] += case["elements"] - sum(sizes)
    names = {"bf16": ["bf16"], "f32": ["f32"], "mixed": ["bf16", "bf16", "f32"]}[case["dtype"]]
    return [(n, names[i % len(names)]) for i, n in enumerate(sizes)]


def _views(sizes, buffers):
    at = dict.fromkeys(buffers, 0)
    for n, t in sizes:
        yield buffers[t][at[t]:at[t] + n], t
        at[t] += n


def _inputs(case, seed):
    gen = _gen(seed)
    if case["op"] == "grad_norm":
        # the gradients of a training program: views into one buffer per type, one tensor behind the other
        sizes = _tensor_sizes(case)
        buffers = {t: torch.randn(sum(n for n, u in sizes if u == t), generator=gen, device="cuda")
                   for t in ("bf16", "f32") if any(u == t for _, u in sizes)}
        for i, (piece, _) in enumerate(_views(sizes, buffers)):
            piece *= 1e-3 * (1 + i % 7)
        buffers = {t: b.to(DTYPES[t]) for t, b in buffers.items()}
        total = sum(n * (1 + i % 7) ** 2 for i, (n, _) in enumerate(sizes)) ** 0.5 * 1e-3
        return {"buffers": buffers, "grads": [g for g, _ in _views(sizes, buffers)], "max_norm": float(total / case["ratio"])}
    dt = DTYPES[case["dtype"]]
    t = {}
    if case["op"] == "gated":
        n, K, cols = case["n"], case["K"], case["cols"]
        t["x"] = _randn(gen, (n, K), dt)
        t["w"] = _randn(gen, (K, 2 * cols), dt, K ** -0.5)
        if case["direction"] == "backward":
            t["pre"] = _randn(gen, (n, 2 * cols), dt)          # what the forward kept: unit-variance projections
            t["dh"] = _randn(gen, (n, cols), dt)
        return t
    B, Tq, Tk, H, Hkv, D = (case[k] for k in ("B", "Tq", "Tk", "H", "Hkv", "D"))
    t["q"] = _randn(gen, (B, Tq, H, D), dt)
    # a few directions of the keys are larger than the rest, so that some rows attend to a handful of keys
    feature = torch.where(torch.randn(Hkv, D, generator=gen, device="cuda").abs() > 2.0, 2.5, 1.0)
    if case["fused"]:
        kv = torch.randn(B, Tk, 2, Hkv, D, generator=gen, device="cuda")
        kv[:, :, 0] *= feature
        t["kv"] = kv.to(dt)
        t["k"], t["v"] = t["kv"][:, :, 0], t["kv"][:, :, 1]
    else:
        t["k"] = (torch.randn(B, Tk, Hkv, D, generator=gen, device="cuda") * feature).to(dt)
        t["v"] = _randn(gen, (B, Tk, Hkv, D), dt)
    shortest = 0 if case["empty"] else 1
    lengths = torch.randint(max(shortest, Tk // 2), Tk + 1, (B,), generator=gen, device="cuda")
    if case["empty"]:
        lengths = torch.where(torch.rand(B, generator=gen, device="cuda") < 0.1, 0, lengths)
    t["lengths"] = lengths.to(torch.int32)
    if case["direction"] == "backward":
        t["dout"] = _randn(gen, (B, Tq, H, D), dt)
        # what the forward kept
        t["o"], t["lse"] = torch.empty_like(t["q"]), torch.empty(B, H, Tq, device="cuda")
        for b in range(B):
            o, lse = _exact_attention_forward(case, t, b)
            t["o"][b], t["lse"][b] = o.to(dt), lse.float()
    return t


def prepare(case, seed):
    t = _inputs(case, seed)
    if not own:
        return {"case": case, "t": t}
    from paper_2006_16668_b200 import binding as B
    empty = lambda shape, dtype: torch.empty(shape, dtype=dtype, device="cuda")
    out = {}
    if case["op"] == "grad_norm":
        out = {"sumsq": empty(1, torch.float64), "norm": empty(1, torch.float32),
               "buffers": t["buffers"] if case["in_place"] else {u: torch.empty_like(b) for u, b in t["buffers"].items()}}
        out["list"] = B.make_grad_list(t["grads"], [g for g, _ in _views(_tensor_sizes(case), out["buffers"])])
        ws_bytes = B.gshard_grad_norm_workspace_bytes(out["list"])
    elif case["op"] == "gated":
        n, K, cols, dt = case["n"], case["K"], case["cols"], DTYPES[case["dtype"]]
        back = case["direction"] == "backward"
        if back:
            out = {"dx": empty((n, K), dt), "dw": empty((K, 2 * cols), dt)}
        else:
            out = {"h": empty((n, cols), dt), "pre": empty((n, 2 * cols), dt) if case["pre"] else None}
        ws_bytes = B.gshard_gated_linear_workspace_bytes(n, K, cols, dt, for_backward=back)
    else:
        dt = DTYPES[case["dtype"]]
        B_, Tq, Tk, H, Hkv, D = (case[k] for k in ("B", "Tq", "Tk", "H", "Hkv", "D"))
        back = case["direction"] == "backward"
        if back:
            out["dq"] = empty((B_, Tq, H, D), dt)
            if case["fused"]:
                out["dkv"] = empty((B_, Tk, 2, Hkv, D), dt)
                out["dk"], out["dv"] = out["dkv"][:, :, 0], out["dkv"][:, :, 1]
            else:
                out["dk"], out["dv"] = empty((B_, Tk, Hkv, D), dt), empty((B_, Tk, Hkv, D), dt)
        else:
            out = {"o": empty((B_, Tq, H, D), dt), "lse": empty((B_, H, Tq), torch.float32) if case["lse"] else None}
        ws_bytes = B.gshard_cross_attention_workspace_bytes(B_, Tq, Tk, H, Hkv, D, dt, for_backward=back)
    return {"case": case, "t": t, "out": out, "workspace": empty(ws_bytes, torch.uint8)}


# ---- the operators through the library ----------------------------------------------------------

def _present(*tensors):
    return tuple(x for x in tensors if x is not None)


def _run_own(state):
    from paper_2006_16668_b200 import binding as B
    case, t, o, ws = state["case"], state["t"], state["out"], state["workspace"]
    if case["op"] == "grad_norm":
        B.gshard_grad_norm(o["list"], o["sumsq"], workspace=ws)
        B.gshard_grad_clip(o["list"], o["sumsq"], t["max_norm"], norm=o["norm"])
        return (o["norm"], *o["buffers"].values())
    forward = case["direction"] == "forward"
    if case["op"] == "gated":
        if forward:
            B.gshard_gated_linear_forward(t["x"], t["w"], o["h"], pre=o["pre"], activation=case["act"], workspace=ws)
            return _present(o["h"], o["pre"])
        B.gshard_gated_linear_backward(t["x"], t["w"], t["pre"], t["dh"], o["dx"], o["dw"], activation=case["act"], workspace=ws)
        return o["dx"], o["dw"]
    if forward:
        B.gshard_cross_attention_forward(t["q"], t["k"], t["v"], o["o"], lse=o["lse"], k_lengths=t["lengths"], workspace=ws)
        return _present(o["o"], o["lse"])
    B.gshard_cross_attention_backward(t["q"], t["k"], t["v"], o=t["o"], lse=t["lse"], dout=t["dout"], dq=o["dq"], dk=o["dk"],
                                      dv=o["dv"], k_lengths=t["lengths"], workspace=ws)
    return (o["dq"], o["dkv"]) if case["fused"] else (o["dq"], o["dk"], o["dv"])


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


def _heads_first(x, heads):
    """[B, T, h, D] to float32 [B, heads, T, D], shared heads repeated."""
    x = x.float().transpose(1, 2)
    return x if x.shape[1] == heads else x.repeat_interleave(heads // x.shape[1], 1)


def _attention_scores(case, t):
    q, k = _heads_first(t["q"], case["H"]), _heads_first(t["k"], case["H"])
    s = torch.matmul(q, k.transpose(-1, -2)) * case["D"] ** -0.5
    behind = torch.arange(case["Tk"], device=s.device) >= t["lengths"][:, None]
    return q, k, s.masked_fill_(behind[:, None, None, :], -math.inf)


def _attention_plain(case, t):
    q, k, s = _attention_scores(case, t)
    v = _heads_first(t["v"], case["H"])
    dt = DTYPES[case["dtype"]]
    if case["direction"] == "forward":
        top = s.amax(-1, keepdim=True)
        top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
        p = s.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p, v) / torch.where(total > 0, total, torch.ones_like(total))
        lse = (top + torch.log(total)).squeeze(-1) if case["lse"] else None
        return _present(o.transpose(1, 2).to(dt).contiguous(), lse)
    scale = case["D"] ** -0.5
    dout = _heads_first(t["dout"], case["H"])
    delta = (dout * _heads_first(t["o"], case["H"])).sum(-1, keepdim=True)
    p = s.sub_(t["lse"][..., None]).exp_()
    dv = torch.matmul(p.transpose(-1, -2), dout)
    ds = torch.matmul(dout, v.transpose(-1, -2)).sub_(delta).mul_(p).mul_(scale)
    dq = torch.matmul(ds, k)
    dk = torch.matmul(ds.transpose(-1, -2), q)
    share = lambda g: g.unflatten(1, (case["Hkv"], -1)).sum(2).transpose(1, 2).to(dt)
    dq = dq.transpose(1, 2).to(dt).contiguous()
    if case["fused"]:
        return dq, torch.stack((share(dk), share(dv)), 2)
    return dq, share(dk).contiguous(), share(dv).contiguous()


def _gated_plain(case, t):
    x, w = t["x"].float(), t["w"].float()
    dt, cols = t["x"].dtype, case["cols"]
    if case["direction"] == "forward":
        pre = x @ w
        h = _act(pre[:, :cols], case["act"]) * pre[:, cols:]
        return _present(h.to(dt), pre.to(dt) if case["pre"] else None)
    gate, up, dh = t["pre"][:, :cols].float(), t["pre"][:, cols:].float(), t["dh"].float()
    dpre = torch.cat((dh * up * _act_grad(gate, case["act"]), dh * _act(gate, case["act"])), 1)
    return (dpre @ w.T).to(dt), (x.T @ dpre).to(dt)


def _norm_plain(case, t):
    norm = torch.stack([g.double().square().sum() for g in t["grads"]]).sum().sqrt()
    factor = torch.where(norm > t["max_norm"], t["max_norm"] / norm, torch.ones_like(norm)).float()
    return (norm.float().reshape(1), *[(b.float() * factor).to(b.dtype) for b in t["buffers"].values()])


def run(state):
    if own:
        return _run_own(state)
    case = state["case"]
    return {"attention": _attention_plain, "gated": _gated_plain, "grad_norm": _norm_plain}[case["op"]](case, state["t"])


# ---- what a pass cannot do without ----------------------------------------------------------------

def work(case):
    if case["op"] == "grad_norm":
        read = sum(n * (2 if t == "bf16" else 4) for n, t in _tensor_sizes(case))
        return {"bytes": read if case["ratio"] < 1 and case["in_place"] else 2 * read, "flops": 3 * case["elements"]}
    es = 4 if case["dtype"] == "f32" else 2
    forward = case["direction"] == "forward"
    if case["op"] == "gated":
        n, K, cols = case["n"], case["K"], case["cols"]
        if forward:
            return {"bytes": (n * K + 2 * K * cols + n * cols * (3 if case["pre"] else 1)) * es, "flops": 4 * n * K * cols}
        return {"bytes": (2 * n * K + 4 * K * cols + 3 * n * cols) * es, "flops": 8 * n * K * cols}
    B, Tq, Tk, H, Hkv, D = (case[k] for k in ("B", "Tq", "Tk", "H", "Hkv", "D"))
    # sources are 3/4 of the padded length on average, less the empty ones
    keys = max(1, int(0.75 * Tk * (0.9 if case["empty"] else 1.0)))
    rows, states = B * Tq * H * D, B * keys * Hkv * D
    if forward:
        return {"bytes": (2 * rows + 2 * states) * es + (4 * B * H * Tq if case["lse"] else 0), "flops": 4 * rows * keys}
    return {"bytes": (4 * rows + 2 * states + 2 * B * Tk * Hkv * D) * es + 4 * B * H * Tq, "flops": 10 * rows * keys}


# ---- the definitions in 64 bits -------------------------------------------------------------------

def _exact_attention_forward(case, t, b):
    """One batch element: o [Tq, H, D] and lse [H, Tq]; keys behind the length left out."""
    length, group = int(t["lengths"][b]), case["H"] // case["Hkv"]
    q = t["q"][b].double().unflatten(1, (case["Hkv"], group))
    k, v = t["k"][b, :length].double(), t["v"][b, :length].double()
    s = torch.einsum("qhgd,khd->hgqk", q, k) / math.sqrt(case["D"])
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)[..., None])
    o = torch.einsum("hgqk,khd->qhgd", p, v)
    return o.flatten(1, 2), lse.flatten(0, 1)


def _exact_attention_backward(case, t, b):
    length, Hkv = int(t["lengths"][b]), case["Hkv"]
    split = lambda x: x[b].double().unflatten(1, (Hkv, -1))
    q, dout, o = split(t["q"]), split(t["dout"]), split(t["o"])
    k, v = t["k"][b, :length].double(), t["v"][b, :length].double()
    scale = 1.0 / math.sqrt(case["D"])
    s = torch.einsum("qhgd,khd->hgqk", q, k) * scale
    p = torch.exp(s - t["lse"][b].double().unflatten(0, (Hkv, -1))[..., None])
    delta = torch.einsum("qhgd,qhgd->hgq", dout, o)
    ds = p * (torch.einsum("qhgd,khd->hgqk", dout, v) - delta[..., None]) * scale
    dq = torch.einsum("hgqk,khd->qhgd", ds, k).flatten(1, 2)
    dk = torch.zeros(case["Tk"], Hkv, case["D"], dtype=torch.float64, device=q.device)
    dv = torch.zeros_like(dk)
    dk[:length] = torch.einsum("hgqk,qhgd->khd", ds, q)
    dv[:length] = torch.einsum("hgqk,qhgd->khd", p, dout)
    return dq, dk, dv


def exact(case, seed):
    t = _inputs(case, seed)
    if case["op"] == "attention":
        one = _exact_attention_forward if case["direction"] == "forward" else _exact_attention_backward
        parts = [torch.stack(p) for p in zip(*[one(case, t, b) for b in range(case["B"])])]
        if case["direction"] == "forward":
            return _present(parts[0], parts[1] if case["lse"] else None)
        return (parts[0], torch.stack(parts[1:], 2)) if case["fused"] else tuple(parts)
    if case["op"] == "grad_norm":
        norm = math.sqrt(math.fsum(float(torch.linalg.vector_norm(g, dtype=torch.float64)) ** 2 for g in t["grads"]))
        factor = t["max_norm"] / norm if norm > t["max_norm"] else 1.0
        return (torch.tensor([norm], dtype=torch.float64, device="cuda"), *[b.double() * factor for b in t["buffers"].values()])
    x, w, act = t["x"].double(), t["w"].double(), case["act"]
    f = torch.nn.functional
    value = {"none": lambda u: u, "relu": f.relu, "gelu": f.gelu, "gelu_tanh": lambda u: f.gelu(u, approximate="tanh"),
             "silu": f.silu}[act]
    if case["direction"] == "forward":
        pre = torch.matmul(x, w)
        gate, up = pre.chunk(2, 1)
        return _present(value(gate) * up, pre if case["pre"] else None)
    pre = t["pre"].double().requires_grad_()
    gate, up = pre.chunk(2, 1)
    dpre = torch.autograd.grad(value(gate) * up, pre, t["dh"].double())[0]
    return torch.matmul(dpre, w.t()), torch.matmul(x.t(), dpre)
