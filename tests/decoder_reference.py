"""64-bit definitions of cross attention and gated linear for the tests, with bounds that count the roundings of the
kernels.  Nothing here calls the library.

Cross attention.  A score is a product over D accumulated in fp32: `steps` roundings of 2^-24 of the absolute sum (bf16:
the tensor core rounds once per 16 products, by up to 2^-23; fp32: once per product), times the scale, plus two roundings
of the scaling itself.  exp turns an absolute error of a score into a relative one of p; numerator and denominator each
carry it.  The exponential itself is off by a few units (2^-22 counted).  With bf16 p (backward: P and dS) is rounded to
8 bits as an operand, 2^-8 of each entry counted at most.  Outputs add half a step of their type."""
from __future__ import annotations

import math

import torch

from operator_reference import HALF, U32, activation, slope

EXP = 2.0 ** -22
HALF = {**HALF, torch.float64: 2.0 ** -53}      # the definitions also take 64-bit operands, for differences
BF = torch.bfloat16


def _steps(dtype, depth):
    return (depth / 16 + 16) * 2 * U32 if dtype == BF else (depth + 16) * U32


def _heads(x, H):
    """[B, T, h, D] to 64-bit [B, H, T, D]"""
    x = x.double().transpose(1, 2)
    return x.repeat_interleave(H // x.shape[1], 1)


def _clean(x, lengths):
    """Keys behind a source's length as zeros, whatever they hold."""
    behind = torch.arange(x.shape[1], device=x.device) >= lengths[:, None]
    return torch.where(behind[:, :, None, None], torch.zeros_like(x), x)


def _scores(q, k, lengths, scale):
    H, D = q.shape[2], q.shape[3]
    Q, K = _heads(q, H), _heads(_clean(k, lengths), H)
    s = torch.matmul(Q, K.transpose(-1, -2)) * scale
    size = torch.matmul(Q.abs(), K.abs().transpose(-1, -2)) * scale
    live = (torch.arange(k.shape[1], device=q.device) < lengths[:, None])[:, None, None, :].expand_as(s)
    off = (_steps(q.dtype, D) * size + 4 * U32 * s.abs()).masked_fill(~live, 0.0)
    return s.masked_fill(~live, -math.inf), off, live


def attention(q, k, v, lengths, scale):
    """(o, bound), (lse, bound)"""
    s, off, live = _scores(q, k, lengths, scale)
    some = live.any(-1)
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - torch.where(some, lse, torch.zeros_like(lse))[..., None])
    V = _heads(_clean(v, lengths), q.shape[2])
    o = torch.matmul(p, V)
    worst = off.amax(-1, keepdim=True) if off.shape[-1] else torch.zeros_like(lse)[..., None]
    rel = 2 * worst + 4 * EXP + _steps(q.dtype, k.shape[1]) * 2 + (HALF[BF] if q.dtype == BF else 0)
    bound = rel * torch.matmul(p, V.abs())
    bound = bound + HALF[q.dtype] * (o.abs() + bound) + 1e-30
    # the running maximum and the logarithm: a few roundings of the largest score and of log(k_len)
    top = s.amax(-1) if s.shape[-1] else torch.zeros_like(lse)
    lse_bound = worst[..., 0] + 4 * EXP + (k.shape[1] / 32 + 16) * U32 + 8 * U32 * torch.where(some, lse.abs() + top.abs(), torch.ones_like(lse))
    return (o.transpose(1, 2), bound.transpose(1, 2)), (lse, lse_bound)


def attention_grad(q, k, v, lengths, scale, o, lse, dout):
    """(value, bound) of dq, dk, dv, with o and lse as given."""
    H, Hkv, D = q.shape[2], k.shape[2], q.shape[3]
    s, off, live = _scores(q, k, lengths, scale)
    P = torch.exp(s - torch.where(torch.isinf(lse), torch.zeros_like(lse), lse).double()[..., None])
    rel = off + 4 * EXP + 4 * U32 * (torch.where(torch.isinf(lse), torch.zeros_like(lse), lse).double().abs()[..., None] + s.abs().masked_fill(~live, 0.0))
    G, O, Q = _heads(dout, H), _heads(o, H), _heads(q, H)
    K, V = _heads(_clean(k, lengths), H), _heads(_clean(v, lengths), H)
    delta = (G * O).sum(-1, keepdim=True)
    delta_off = (D + 16) * U32 * (G * O).abs().sum(-1, keepdim=True)
    dP = torch.matmul(G, V.transpose(-1, -2))
    dP_off = _steps(q.dtype, D) * torch.matmul(G.abs(), V.abs().transpose(-1, -2))
    half = HALF[BF] if q.dtype == BF else U32
    dS = scale * P * (dP - delta)
    dS_off = scale * P * (rel * (dP - delta).abs() + (1 + rel) * (dP_off + delta_off + 2 * U32 * (dP.abs() + delta.abs())))
    dS_off = dS_off + half * (dS.abs() + dS_off)
    P_off = P * (rel + half * (1 + rel))
    out = []
    share = lambda x: x.unflatten(1, (Hkv, H // Hkv)).sum(2)
    T = lambda x: x.transpose(-1, -2)
    for value, terms, slack, depth in ((torch.matmul(dS, K), torch.matmul(dS.abs() + dS_off, K.abs()), torch.matmul(dS_off, K.abs()), k.shape[1]),
                                       (share(torch.matmul(T(dS), Q)), share(torch.matmul(T(dS.abs() + dS_off), Q.abs())),
                                        share(torch.matmul(T(dS_off), Q.abs())), q.shape[1] * (H // Hkv)),
                                       (share(torch.matmul(T(P), G)), share(torch.matmul(T(P + P_off), G.abs())),
                                        share(torch.matmul(T(P_off), G.abs())), q.shape[1] * (H // Hkv))):
        bound = _steps(q.dtype, depth) * terms + slack + 2 * U32 * value.abs()
        bound = bound + HALF[q.dtype] * (value.abs() + bound) + 1e-30
        out.append((value.transpose(1, 2), bound.transpose(1, 2)))
    return out


def gated(x, w, act):
    """(h, bound), (pre, bound): bounds as for the linear operator, one product of two factors more."""
    x, w, dtype = x.double(), w.double(), x.dtype
    cols = w.shape[1] // 2
    pre = x @ w
    off = _steps(dtype, x.shape[1]) * (x.abs() @ w.abs()) + 1e-30
    half = HALF[dtype]
    g, u = pre[:, :cols], pre[:, cols:]
    a = activation(g, act)
    a_off = 1.2 * off[:, :cols] + (0 if act in ("none", "relu") else 24 * U32 * (g.abs() + 1))
    h = a * u
    bound = a_off * (u.abs() + off[:, cols:]) + a.abs() * off[:, cols:] + 2 * U32 * h.abs()
    return (h, bound + half * (h.abs() + bound)), (pre, off + half * (pre.abs() + off))


def gated_grad(x, w, pre, dh, act):
    """(dx, bound), (dw, bound)"""
    dtype = x.dtype
    x, w, pre, dh = x.double(), w.double(), pre.double(), dh.double()
    cols = dh.shape[1]
    g, u = pre[:, :cols], pre[:, cols:]
    smooth = 0 if act in ("none", "relu") else 24 * U32
    dpre = torch.cat((dh * u * slope(g, act), dh * activation(g, act)), 1)
    off = torch.cat((dh.abs() * u.abs(), dh.abs()), 1) * torch.cat((1 + g.abs(), 1 + g.abs()), 1) * (smooth + 4 * U32)
    slack = off + (HALF[BF] if dtype == BF else U32) * (dpre.abs() + off)
    out = []
    for value, terms, extra, depth in ((dpre @ w.t(), (dpre.abs() + slack) @ w.abs().t(), slack @ w.abs().t(), 2 * cols),
                                       (x.t() @ dpre, x.abs().t() @ (dpre.abs() + slack), x.abs().t() @ slack, x.shape[0])):
        bound = _steps(dtype, depth) * terms + extra + 1e-30
        out.append((value, bound + HALF[dtype] * (value.abs() + bound)))
    return out
