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


# ------------------------------------------------------------------ 8-bit floats in blocks

# Codes 0 .. 126 in order: subnormal steps of 2^-9, then eight steps to each power of two, up to 448.
E4M3 = torch.tensor([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127],
                    dtype=torch.float64)
F8_LO, F8_HI = -117, 119


def f8_exponent(top):
    """The smallest e in -117 .. 119 with top <= 448 * 2^e, found by counting: exact in 64 bits.  top fp64, finite."""
    e = torch.full(top.shape, F8_LO, dtype=torch.int64)
    for k in range(F8_LO, F8_HI):
        e = torch.where(top > 448.0 * 2.0 ** k, torch.full_like(e, k + 1), e)
    return e


def f8_round(x, e):
    """Codes uint8 of x fp64 over 2^e (broadcast): the nearest of the 127 magnitudes, ties to the even code."""
    y = (x.abs() / torch.exp2(e.double())).clamp_max(448.0)
    hi = torch.searchsorted(E4M3, y.contiguous()).clamp(1, 126)       # E4M3[hi - 1] < y <= E4M3[hi], but for y = 0
    up, down = E4M3[hi] - y, y - E4M3[hi - 1]
    code = torch.where(up < down, hi, torch.where(up > down, hi - 1, hi - hi % 2))
    return (code + 128 * torch.signbit(x)).to(torch.uint8)


def f8_value(code, byte):
    """fp64 values of codes with exponent bytes (broadcast); NaN for the codes that are none."""
    c = code.long() % 128
    v = torch.where(c == 127, torch.full(c.shape, math.nan, dtype=torch.float64), E4M3[c.clamp_max(126)])
    return torch.where(code >= 128, -v, v) * torch.exp2(byte.double() - 127)


def rows_f8(x, weight=None, residual=None, eps=1e-6):
    """(codes uint8 [rows][cols], exponent bytes [rows][blocks], scale fp64 [rows], h in x's type)."""
    h = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    t = h.float()
    if weight is not None:
        t = t * weight.float()
    rows, cols = t.shape
    g = torch.nn.functional.pad(t, (0, -cols % 128)).double().reshape(rows, -1, 128)
    bad = ~torch.isfinite(g).all(-1)
    g = torch.where(bad[..., None], torch.zeros_like(g), g)
    e = f8_exponent(g.abs().amax(-1))
    codes = f8_round(g, e[..., None])
    byte = torch.where(bad, torch.full_like(e, 255), e + 127).to(torch.uint8)
    scale = 1 / torch.sqrt(h.double().square().mean(1) + eps)
    scale = torch.where(torch.isfinite(h).all(1), scale.clamp_max(torch.finfo(torch.float32).max),
                        torch.full_like(scale, math.nan))
    return codes.reshape(rows, -1)[:, :cols], byte, scale, h


def rows_f8_value(codes, byte):
    """fp64 values of rows; NaN in a block whose byte is 255."""
    b = byte.repeat_interleave(128, 1)[:, :codes.shape[1]]
    v = f8_value(codes, b)
    return torch.where(b == 255, torch.full_like(v, math.nan), v)


def matmul_f8(a, w, a_scale=None, bias=None, residual=None, relu=False, bf16=True):
    """(y fp64, bound of the error) of fp64 values a, w.  The sum: as many additions as products, in any order, each off by
    2^-23 at most of a partial sum's size (fp32, cut off or rounded); one rounding for each factor and addend, one for y.
    For bf16 outputs eight neighbouring products are added aligned to the largest, 2^E <= |p| < 2^(E + 2), the other seven
    cut to multiples of 2^(E - 13): each off by less than 2^-13 |p|, and |p| is at most the product of the eight's largest
    factors."""
    y, size = a @ w.t(), a.abs() @ w.abs().t()
    tol = (a.shape[1] + 4) * 2 * U * size
    if bf16:
        top = lambda t: torch.nn.functional.pad(t.abs(), (0, -t.shape[1] % 8)).unflatten(1, (-1, 8)).amax(-1)  # noqa: E731
        tol = tol + 7 * 2.0 ** -13 * (top(a) @ top(w).t())
    if a_scale is not None:
        y, size, tol = (t * a_scale.double().abs()[:, None] for t in (y * torch.sign(a_scale.double())[:, None], size, tol))
    steps = 2
    for extra in (None if bias is None else bias.double(), None if residual is None else residual.double()):
        if extra is not None:
            y = y + extra
            size = size + extra.abs()
            steps += 1
    if relu:
        y = torch.where(y < 0, torch.zeros_like(y), y)
    return y, tol + steps * U * size + (U16 * (y.abs() + tol) * (1 + U16) if bf16 else U * y.abs())


class KV8:
    """An 8-bit cache as lists of what is written: codes uint8 [pages][heads][page][D], bytes uint8 [pages][heads][blocks],
    for keys (0) and values (1)."""

    def __init__(self, codes, byte):
        self.codes, self.byte = [c.clone() for c in codes], [b.clone() for b in byte]
        self.page = self.codes[0].shape[2]
        self.block = self.page // self.byte[0].shape[2]

    def write(self, k, v, news, lens, table, max_new=None):
        """k, v fp64 [tokens][heads][D], the new tokens of the sequences one after another; a block and a head at a time."""
        pages = self.codes[0].shape[0]
        row = 0
        for s, n in enumerate(news):
            places = [(lens[s] - n + i, row + i) for i in range(n if max_new is None else min(n, max_new))]
            places = [(p, r) for p, r in places if 0 <= p < table.shape[1] * self.page]
            row += n
            for b in sorted({p // self.block for p, _ in places}):
                mine = [(p, r) for p, r in places if p // self.block == b]
                page, at = int(table[s, b * self.block // self.page]), b * self.block % self.page
                if not 0 <= page < pages:
                    continue
                held = mine[0][0] - b * self.block
                for h in range(k.shape[1]):
                    good = [bool(torch.isfinite(k[r, h]).all() and torch.isfinite(v[r, h]).all()) for _, r in mine]
                    for i, x in enumerate((k, v)):
                        codes, byte = self.codes[i][page, h], self.byte[i][page, h]
                        tops = [x[r, h].abs().max() for (_, r), ok in zip(mine, good) if ok]
                        e = int(f8_exponent(torch.stack(tops).max() if tops else torch.zeros((), dtype=torch.float64)))
                        was = min(int(byte[at // self.block]) - 127, F8_HI)
                        if held and was >= e:
                            e = was
                        elif held:
                            old = codes[at:at + held]
                            new = f8_round(torch.nan_to_num(f8_value(old, torch.tensor(was + 127))), torch.tensor(e))
                            codes[at:at + held] = torch.where(old % 128 == 127, old, new)
                        byte[at // self.block] = e + 127
                        for (p, r), ok in zip(mine, good):
                            codes[p % self.page] = f8_round(x[r, h], torch.tensor(e)) if ok else (127 if i == 0 else 0)

    def values(self, i, slots):
        """fp64 [tokens][heads][D] of keys (i = 0) or values at slots."""
        p, at = slots.long() // self.page, slots.long() % self.page
        return f8_value(self.codes[i][p, :, at], self.byte[i][p, :, at // self.block][..., None])
