"""CPU oracle for the operators of quantised transformer blocks.

TEST INFRASTRUCTURE ONLY, like the rest of this package: plain torch on the
CPU, in 64 bits, written from the operators' definitions (``include/miquant.h``)
and sharing no code with the HIP path.  Results in 8 and 4 bits are defined by
fp32 operations whose order does not matter, so they are unique; the others
come with a bound on the error that the kernels' stated roundings allow.
"""
from __future__ import annotations

import math

import torch

E2M1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
U = 2.0 ** -24            # unit roundoff of fp32
U16 = 2.0 ** -8           # of bf16: 8 significant bits


# ------------------------------------------------------------------ rows in 8 bits

def rows_i8(x, weight=None, residual=None, eps=1e-6, norm=True):
    """(q int8, scale fp64, h in x's type)."""
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    t = h.float()
    if weight is not None:
        t = t * weight.float()
    top = t.abs().max(1).values                      # a NaN stays
    bad = ~torch.isfinite(top)
    zero = ~bad & (top < 2.0 ** -100)
    f = torch.where(bad | zero, torch.zeros_like(top), torch.full_like(top, 127.0) / top)
    q = torch.where((f == 0)[:, None], torch.zeros_like(t), torch.round(t * f[:, None])).to(torch.int8)
    scale = top.double() / 127
    if norm:
        scale = scale / torch.sqrt(h.double().square().mean(1) + eps)
    scale = torch.where(zero, torch.zeros_like(scale), torch.where(bad, torch.full_like(scale, math.nan), scale))
    return q, scale, h


# ------------------------------------------------------------------ product of 8-bit integers

def matmul_i8(a, a_scale, w, w_scale, bias=None, residual=None, relu=False, bf16=True):
    """(y fp64, bound of the error): one rounding for the sum as fp32, one for each factor and addend, one for y."""
    y = (a.double() @ w.double().t()) * a_scale.double()[:, None] * w_scale.double()
    size, steps = y.abs(), 3
    for extra in (None if bias is None else bias.double(), None if residual is None else residual.double()):
        if extra is not None:
            y = y + extra
            size = size + extra.abs()
            steps += 1
    if relu:
        y = y.clamp_min(0)
    return y, (steps + 1) * U * size + (U16 * y.abs() * (1 + U16) if bf16 else U * y.abs())


# ------------------------------------------------------------------ the 4-bit cache

def kv4_encode(x):
    """x [..., D] -> (codes uint8 [..., D / 2], exponent bytes uint8 [..., D / 32])."""
    g = x.double().reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    top = g.abs().amax(-1)
    bad = ~torch.isfinite(top)
    e = torch.full_like(top, -126)
    # smallest e with top <= 7 * 2^e, found by counting: exact in 64 bits
    for k in range(-126, 125):
        e = torch.where(top > 7.0 * 2.0 ** k, torch.full_like(e, k + 1), e)
    u = (g.abs() / torch.exp2(e)[..., None]).clamp_max(6.0)
    u = torch.where(bad[..., None], torch.zeros_like(u), u)
    dist = (u[..., None] - E2M1).abs()
    best = dist.amin(-1, keepdim=True)
    near = dist == best                              # one level, or two at a tie: then the even code
    even = torch.arange(8) % 2 == 0
    pick = torch.where(near.sum(-1) > 1, (near & even).to(torch.int64).argmax(-1), near.to(torch.int64).argmax(-1))
    sign = torch.signbit(g) & ~bad[..., None]
    code = (pick + 8 * sign).reshape(*x.shape[:-1], x.shape[-1] // 2, 2)
    byte = torch.where(bad, torch.full_like(e, 255), e + 127)
    return (code[..., 0] + 16 * code[..., 1]).to(torch.uint8), byte.to(torch.uint8)


def kv4_decode(codes, exps):
    """fp64 [..., D]; NaN in a group whose exponent byte is above 252."""
    c = torch.stack((codes.long() % 16, codes.long() // 16), -1).flatten(-2)
    v = E2M1[c % 8] * torch.where(c >= 8, -1.0, 1.0)
    s = torch.exp2(exps.double() - 127)
    s = torch.where(exps > 252, torch.full_like(s, math.nan), s)
    return (v.reshape(*exps.shape, 32) * s[..., None]).reshape(v.shape)


# ------------------------------------------------------------------ attention

def attention(q, k, v, news, lens, scale, causal=True, window=0):
    """q [tokens][heads][D], the queries of the sequences one after another (news[s] of them); k, v lists of fp64
    [lens[s]][key heads][D].  Returns (out fp64, bound of the error).

    The bound: with weights p, a relative error r of each weight changes sum(p v) / sum(p) by at most
    r sum(p |v - out|) / sum(p).  r is that of the rounding to bf16, of the score (fp32 sums of D products, the
    factor, the difference to the maximum) and of the exponential; the result is rounded to bf16.  A weight below fp32's
    smallest normal number, 2^-126 of one that counts, may be taken as 0."""
    out = torch.zeros(q.shape, dtype=torch.float64)
    tol = torch.zeros(q.shape, dtype=torch.float64)
    heads, d = q.shape[1:]
    row = 0
    for s, n in enumerate(news):
        L = lens[s]
        g = heads // k[s].shape[1]
        for i in range(n):
            p = L - n + i
            hi = min(L, p + 1) if causal else L
            lo = max(0, p - window + 1) if window > 0 else 0
            if hi > lo:
                kk = k[s][lo:hi].repeat_interleave(g, 1)          # [T][heads][D]
                vv = v[s][lo:hi].repeat_interleave(g, 1)
                qq = q[row].double()
                sc = (kk * qq).sum(-1) * scale                    # [T][heads]
                w = torch.exp(sc - sc.max(0).values)
                w = w / w.sum(0)
                o = (w[..., None] * vv).sum(0)
                size = (kk.abs() * qq.abs()).sum(-1).amax(0) * abs(scale)
                r = U16 * (1 + U16) + 2 * U * ((d + 4) * size + (hi - lo) / 4 + 16)
                spread = (w[..., None] * (vv - o).abs()).sum(0)
                bad = ~torch.isfinite(kk).all(-1) | ~torch.isfinite(vv).all(-1)   # a NaN anywhere makes the head's row NaN
                out[row] = torch.where(bad.any(0)[:, None], torch.full_like(o, math.nan), o)
                tol[row] = r[:, None] * spread * 1.01 + U16 * o.abs() * 1.01 + 2.0 ** -126 * vv.abs().sum(0)
            row += 1
    return out, tol
