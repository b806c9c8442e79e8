"""64-bit definitions of layer norm, linear and routing for the tests, and the unit roundings that the
tolerances count.  Nothing here calls the library."""
from __future__ import annotations

import math

import torch

U32 = 2.0 ** -24                       # half a step of float32, relative
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def within(got, want, bound, what):
    """Every element of got is finite where want is, and within bound (a float64 tensor) of want."""
    got = got.double()
    assert torch.equal(torch.isfinite(got), torch.isfinite(want)), f"{what}: not finite"
    err = (got - want).abs()
    bad = err > bound
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} out of bounds, worst error "
                           f"{float((err / bound.clamp(min=1e-300)).max()):.3g} of its bound")


# ---- layer norm -------------------------------------------------------------------------------

def layer_norm(x, gamma, beta, eps):
    x = x.double()
    mean = x.mean(1)
    rstd = 1.0 / torch.sqrt((x - mean[:, None]).square().mean(1) + eps)
    y = (x - mean[:, None]) * rstd[:, None] * gamma.double()
    return (y if beta is None else y + beta.double()), mean, rstd


def layer_norm_grad(x, gamma, mean, rstd, dy, dskip):
    x, dy, r = x.double(), dy.double(), rstd.double()[:, None]
    z = (x - mean.double()[:, None]) * r
    g = dy * gamma.double()
    dx = r * (g - g.mean(1, keepdim=True) - z * (g * z).mean(1, keepdim=True))
    if dskip is not None:
        dx = dx + dskip.double()
    return dx, (dy * z).sum(0), dy.sum(0)


# ---- linear -----------------------------------------------------------------------------------

def activation(v, act):
    if act == "relu":
        return v.clamp(min=0)
    if act == "gelu":
        return 0.5 * v * torch.special.erfc(-v / math.sqrt(2.0))
    if act == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)))
    if act == "silu":
        return v * torch.sigmoid(v)
    return v.clone()


def slope(v, act):
    if act == "none":
        return torch.ones_like(v)
    if act == "relu":
        return (v > 0).to(v.dtype)
    v = v.detach().clone().requires_grad_()
    return torch.autograd.grad(activation(v, act).sum(), v)[0]


# ---- routing ----------------------------------------------------------------------------------

def usable(logits):
    l = logits.double()
    l = torch.where(torch.isnan(l), torch.full_like(l, -math.inf), l)
    return l.clamp(max=torch.finfo(torch.float32).max)


def scores(l, score):
    if score == "sigmoid":
        return torch.sigmoid(l)
    top = l.amax(-1, keepdim=True)
    e = torch.exp(l - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = e.sum(-1, keepdim=True)
    return e / torch.where(total > 0, total, torch.ones_like(total))


def choose(logits, bias, *, k, score="softmax", groups=1, groups_kept=1, group_top=1):
    """[N, k] int64 in order of preference, -1 where nothing is left; row by row, by sorting."""
    l = usable(logits).cpu()
    s = scores(l, score)
    c = l if bias is None else torch.where(l == -math.inf, l, s + bias.double().cpu())
    c = torch.where(torch.isnan(c), torch.full_like(c, -math.inf), c)
    by_value = c if (bias is not None or group_top == 1) else torch.where(l == -math.inf, l, s)
    out = torch.full((l.shape[0], k), -1, dtype=torch.int64)
    E = l.shape[1]
    size = E // groups
    for n in range(l.shape[0]):
        allowed = range(E)
        if groups_kept < groups:
            worth = []
            for g in range(groups):
                best = sorted((v for v in by_value[n, g * size:(g + 1) * size].tolist() if v != -math.inf),
                              reverse=True)[:group_top]
                worth.append(sum(best) if best else -math.inf)
            keep = sorted(range(groups), key=lambda g: (-worth[g], g))[:groups_kept]
            allowed = [e for g in sorted(keep) for e in range(g * size, (g + 1) * size)]
        row = c[n].tolist()
        order = sorted((e for e in allowed if row[e] != -math.inf), key=lambda e: (-row[e], e))[:k]
        out[n, :len(order)] = torch.tensor(order, dtype=torch.int64)
    return out


def log_scores(l, score):
    if score == "sigmoid":
        return torch.nn.functional.logsigmoid(l)
    nothing = (l == -math.inf).all(-1, keepdim=True)
    return torch.log_softmax(torch.where(nothing, torch.zeros_like(l), l), -1).masked_fill(nothing, -math.inf)


def route_weights(l, idx, score, renormalise, scale):
    """Weights [N, k] of chosen experts idx (int64, -1 absent) from logits l [N, E] in 64 bits."""
    gone = idx < 0
    # a softmax's normaliser cancels in renormalised weights: the logits themselves keep their differences
    # also where another expert's logit is the largest float
    logs = l if renormalise and score == "softmax" else log_scores(l, score)
    pick = logs.gather(-1, idx.clamp(min=0)).masked_fill(gone, -math.inf)
    if renormalise:
        none = gone.all(-1, keepdim=True)
        top = pick.amax(-1, keepdim=True)
        pick = pick - torch.where(none, torch.zeros_like(top), top)
        pick = pick - torch.logsumexp(pick.masked_fill(none, 0.0), -1, keepdim=True)
    return scale * pick.exp().masked_fill(gone, 0.0)
