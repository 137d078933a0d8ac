"""The operators of transformer blocks in 8-bit floating point, and the pick of a token, whose speed is tracked.

A block served in 8-bit floating point holds what it multiplies, and the keys and values of past
tokens, as e4m3 values in blocks that share a power of two (a byte, exponent plus 127):

  rows     residual addition, root-mean-square norm and the 8-bit output with a byte for each 128 values of a row
  matmul   product of such rows, with bias, residual addition and ReLU in the epilogue
  cache    the keys and values of new tokens written to the paged 8-bit cache, and tokens read back
  attend   attention of queries over that cache: single tokens, chunks of a prompt, whole prompts
  sample   a token drawn from each row of logits: temperature, top-k, top-p, min-p, a given random number

A block's exponent is the smallest e with max|x| <= 448 * 2^e, held to -117 .. 119.  A cache is
values [pages][heads][page size][head size] and exponents [pages][heads][page size / block], for
keys and for values: a block is `block` places of a page and a head.  Tokens that are added to a
block raise its exponent where they need it, and the values it holds are rounded again.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6
GROUP = 128
F8 = torch.float8_e4m3fn


# ------------------------------------------------------------------ the cases

def _rows(M, C, dtype, residual):
    return {"op": "rows", "M": M, "C": C, "dtype": dtype, "residual": residual}


def _matmul(M, K, N, out, scaled, bias, residual, relu):
    return {"op": "matmul", "M": M, "K": K, "N": N, "out": out, "scaled": scaled, "bias": bias, "residual": residual,
            "relu": relu}


def _cache(seqs, new, old, heads, D, page, block, dtype):
    return {"op": "cache", "seqs": seqs, "new": new, "old": old, "heads": heads, "D": D, "page": page, "block": block,
            "dtype": dtype}


def _attend(seqs, new, longest, heads, kv_heads, D, page, block, window):
    return {"op": "attend", "seqs": seqs, "new": new, "longest": longest, "heads": heads, "kv_heads": kv_heads,
            "D": D, "page": page, "block": block, "window": window}


def _sample(rows, vocab, dtype, top_k, top_p, min_p, masked):
    return {"op": "sample", "rows": rows, "vocab": vocab, "dtype": dtype, "top_k": top_k, "top_p": top_p,
            "min_p": min_p, "masked": masked}


def listed():
    return [
        # One token of one stream through a small block: latency.
        {"name": "rows_token", **_rows(1, 1024, "bf16", True)},
        # A long batch of prompt tokens: bandwidth.
        {"name": "rows_prompt", **_rows(16384, 4096, "bf16", True)},
        # A serving batch, one token each, straight from the norm: the weights' bandwidth.
        {"name": "matmul_batch", **_matmul(16, 4096, 4096, "bf16", True, False, False, False)},
        # Features of a picture's patches into a thousand classes in fp32: no extent fills a tile or a block.
        {"name": "matmul_ragged_f32", **_matmul(333, 1999, 1000, "f32", False, True, False, True)},
        # The widening projection of a long batch of prompt tokens: the matrix cores' rate.
        {"name": "matmul_prompt", **_matmul(8192, 4096, 8192, "bf16", True, True, False, True)},
        # One new token for each sequence of a serving batch, its block read back.
        {"name": "cache_token", **_cache(64, 1, 1000, 8, 128, 64, 16, "bf16")},
        # Whole prompts written, and read back for a program that wants them in bf16.
        {"name": "cache_prompt", **_cache(4, 4000, 0, 8, 128, 64, 64, "bf16")},
        # A serving batch, one token each, over caches of ragged lengths: bandwidth.
        {"name": "attend_tokens", **_attend(16, 1, 32768, 32, 8, 128, 64, 64, 0)},
        # A short chunk over a window of its context, pages, blocks and heads of another size.
        {"name": "attend_chunk", **_attend(3, 17, 5000, 12, 4, 64, 48, 16, 1000)},
        # Whole prompts: the matrix cores' rate.
        {"name": "attend_prompt", **_attend(2, 4096, 4096, 32, 8, 128, 64, 64, 0)},
        # The next token of one stream, with every filter: latency.
        {"name": "sample_token", **_sample(1, 32000, "f32", 50, 0.9, 0.02, False)},
        # The next tokens of a serving batch over a large vocabulary, some of it forbidden: bandwidth.
        {"name": "sample_batch", **_sample(256, 128000, "bf16", 0, 0.9, 0.0, True)},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the same ranges, none dearer than the listed ones of its operator."""
    while True:
        op = rng.choice(("rows", "matmul", "matmul", "cache", "attend", "attend", "sample", "sample"))
        if op == "rows":
            C = _log(rng, 64, 8192)
            C = C if rng.random() < 0.3 else -(-C // 64) * 64
            c = _rows(_log(rng, 1, 16384), C, rng.choice(("bf16", "bf16", "f32")), rng.random() < 0.7)
            ok = c["M"] * C * (1 if c["dtype"] == "bf16" else 2) <= 16384 * 4096
        elif op == "matmul":
            K, N = _log(rng, 64, 16384), _log(rng, 64, 16384)
            if rng.random() < 0.7:
                K, N = -(-K // 64) * 64, -(-N // 64) * 64
            c = _matmul(_log(rng, 1, 8192), K, N, rng.choice(("bf16", "bf16", "f32")), rng.random() < 0.5,
                        rng.random() < 0.5, rng.random() < 0.3, rng.random() < 0.4)
            ok = c["M"] * K * N <= 8192 * 4096 * 8192 and c["M"] * N <= 8192 * 8192 and K * N <= 1 << 27
        elif op == "cache":
            new = 1 if rng.random() < 0.4 else _log(rng, 2, 8000)
            block = rng.choice((8, 16, 16, 32, 64))
            c = _cache(_log(rng, 1, 64), new, _log(rng, 1, 4000), rng.choice((1, 2, 4, 8, 16)),
                       rng.choice((64, 64, 96, 128, 128, 128, 256)), block * rng.choice((1, 2, 3)), block,
                       rng.choice(("bf16", "bf16", "f32")))
            ok = c["seqs"] * (2 * new + c["old"]) * c["heads"] * c["D"] * (1 if c["dtype"] == "bf16" else 2) <= \
                4 * 8000 * 8 * 128
        elif op == "attend":
            kv = rng.choice((1, 2, 4, 8, 8))
            new = rng.choice((1, 1, 1, _log(rng, 2, 64), _log(rng, 65, 4096)))
            block = rng.choice((8, 16, 16, 32, 64, 64))
            c = _attend(_log(rng, 1, 64), new, new + _log(rng, 1, 32768), kv * rng.choice((1, 2, 4, 4, 8)), kv,
                        rng.choice((64, 64, 96, 128, 128, 128, 256)), block * rng.choice((1, 2, 3)), block,
                        0 if rng.random() < 0.8 else _log(rng, 100, 4000))
            tokens, scores = c["seqs"] * c["longest"], c["seqs"] * c["heads"] * new * c["longest"]
            ok = tokens * kv * c["D"] <= 16 * 32768 * 8 * 128 and scores * c["D"] <= 2 * 32 * 4096 * 4096 * 128 and \
                scores <= 2 * 32 * 4096 * 4096
        else:
            vocab = _log(rng, 100, 260000)
            c = _sample(_log(rng, 1, 512), vocab, rng.choice(("bf16", "f32")),
                        rng.choice((0, 0, _log(rng, 1, 1000))), rng.choice((0.0, 0.9, 0.95)), rng.choice((0.0, 0.0, 0.02)),
                        rng.random() < 0.3)
            ok = c["rows"] * vocab * (1 if c["dtype"] == "bf16" else 2) <= 256 * 128000
        if ok:
            return c


# ------------------------------------------------------------------ the inputs

def _exponent(top):
    """The smallest e in -117 .. 119 with top <= 448 * 2^e."""
    m, x = torch.frexp(top)
    e = torch.where(m > 0.875, x - 8, x - 9).clamp(-117, 119)
    return torch.where(top == 0, torch.full_like(e, -117), e)


def _encode(x, e):
    """x fp32 as e4m3 values of the power e (int32, broadcast): the nearest, ties to even."""
    return torch.ldexp(x, -e).clamp(-448, 448).to(F8)


def _decode(codes, byte):
    """The values of e4m3 codes with exponent bytes (broadcast), fp32."""
    return torch.ldexp(codes.float(), byte.int() - 127)


def _encode_rows(x):
    """x fp32 [M][K] in blocks of 128 along a row: codes [M][K] and exponent bytes [M][K / 128, rounded up]."""
    M, K = x.shape
    g = torch.nn.functional.pad(x, (0, -K % GROUP)).reshape(M, -1, GROUP)
    e = _exponent(g.abs().amax(-1))
    return _encode(g, e.unsqueeze(-1)).reshape(M, -1)[:, :K].contiguous(), (e + 127).to(torch.uint8)


def _decode_rows(codes, byte):
    K = codes.shape[1]
    return _decode(codes, byte.repeat_interleave(GROUP, 1)[:, :K])


def _activations(g, *shape):
    """Values as hidden states have them: normal, a few channels many times larger than the rest."""
    x = torch.randn(*shape, generator=g, device="cuda")
    gain = 1 + 15 * (torch.rand(shape[-1], generator=g, device="cuda") < 0.01)
    return x * gain


def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _new_cache(g, pages, heads, page, block, D):
    """A cache of `pages` pages that hold earlier tokens: values and exponents of keys, and of values."""
    held = []
    for _ in range(2):
        x = _activations(g, pages * page, heads, D).reshape(pages, page // block, block, heads, D)
        e = _exponent(x.abs().amax((2, 4)))                                   # [pages][blocks][heads]
        codes = _encode(x, e[:, :, None, :, None]).reshape(pages, page, heads, D)
        held += [codes.transpose(1, 2).contiguous(), (e + 127).to(torch.uint8).transpose(1, 2).contiguous()]
    return tuple(held)


def _lengths(case):
    """Cached tokens of each sequence, the new ones among them: the longest, then ever shorter by a fixed pattern."""
    n, top, new = case["seqs"], case["longest"], case["new"]
    return [top if i == 0 else max(new, int(top * (1.0 - 0.6 * ((i * 7) % 11) / 11.0)) - i) for i in range(n)]


def _news(case, lens):
    """New tokens of each sequence: prompts of one batch differ in length."""
    new = case["new"]
    return [new if i == 0 else max(1, min(n, new - (new * ((i * 5) % 7)) // 16)) for i, n in enumerate(lens)]


def _starts(news):
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    return torch.tensor(starts, dtype=torch.int32, device="cuda")


def _paged(g, lens, page):
    """A page table for sequences of these lengths, pages in no order, and the number of pages."""
    pages = [-(-x // page) for x in lens]
    order = torch.randperm(sum(pages), generator=g, device="cuda").to(torch.int32)
    table = torch.zeros(len(lens), max(pages), dtype=torch.int32, device="cuda")
    row = torch.repeat_interleave(torch.arange(len(lens)), torch.tensor(pages))
    col = torch.cat([torch.arange(p) for p in pages])
    table[row.cuda(), col.cuda()] = order
    return table, sum(pages)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    s = dict(case)
    rand = lambda *shape: torch.rand(*shape, generator=g, device="cuda")  # noqa: E731
    if case["op"] == "rows":
        M, C, t = case["M"], case["C"], _type(case["dtype"])
        s["x"] = (0.2 * _activations(g, M, C)).to(t)
        s["residual"] = _activations(g, M, C).to(t) if case["residual"] else None
        s["weight"] = 0.5 + rand(C)
    elif case["op"] == "matmul":
        M, K, N = case["M"], case["K"], case["N"]
        s["a"], s["a_exps"] = _encode_rows(_activations(g, M, K))
        s["w"], s["w_exps"] = _encode_rows(torch.randn(N, K, generator=g, device="cuda") * math.sqrt(2.0 / K))
        s["a_scale"] = 0.3 + 0.7 * rand(M) if case["scaled"] else None
        s["bias_v"] = 0.1 * torch.randn(N, generator=g, device="cuda") if case["bias"] else None
        s["res"] = torch.randn(M, N, generator=g, device="cuda").to(_type(case["out"])) if case["residual"] else None
    elif case["op"] == "cache":
        n, H, D, page, block = (case[k] for k in ("seqs", "heads", "D", "page", "block"))
        lens = [case["new"] + max(0, case["old"] - 5 * i) for i in range(n)]
        s["table"], pages = _paged(g, lens, page)
        s["kv"] = _new_cache(g, pages, H, page, block, D)
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        s["starts"] = torch.arange(n + 1, dtype=torch.int32, device="cuda") * case["new"]
        # read back: the new tokens and up to 16 before them
        at = torch.cat([torch.arange(max(0, x - case["new"] - 16), x) for x in lens]).cuda()
        seq = torch.repeat_interleave(torch.arange(n), torch.tensor([min(x, case["new"] + 16) for x in lens])).cuda()
        s["read"] = (s["table"][seq, at // page] * page + at % page).to(torch.int32)
        kv = _activations(g, n * case["new"], 2 * H * D).to(_type(case["dtype"]))   # as a fused projection leaves them
        s["k"], s["v"] = (kv[:, i * H * D:(i + 1) * H * D].unflatten(1, (H, D)) for i in (0, 1))
    elif case["op"] == "attend":
        H, KV, D, page, block = (case[k] for k in ("heads", "kv_heads", "D", "page", "block"))
        lens = _lengths(case)
        s["table"], pages = _paged(g, lens, page)
        s["kv"] = _new_cache(g, pages, KV, page, block, D)
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        news = _news(case, lens)
        s["starts"] = _starts(news)
        s["q"] = (1.5 * torch.randn(sum(news), H * D, generator=g, device="cuda")).to(torch.bfloat16).unflatten(1, (H, D))
        s["scale"] = 1.0 / math.sqrt(D) / 2.0
    else:
        R, V = case["rows"], case["vocab"]
        x = 2.5 * torch.randn(R, V, generator=g, device="cuda")
        # as a trained head gives them: some rows sure of a few tokens, some of none
        liked = torch.randint(0, V, (R, 8), generator=g, device="cuda")
        x.scatter_add_(1, liked, 10 * rand(R, 8) * (rand(R, 1) < 0.7))
        if case["masked"]:   # a grammar forbids a part of the vocabulary
            x.masked_fill_(rand(V) < 0.3, float("-inf"))
        s["logits"] = x.to(_type(case["dtype"]))
        s["u"] = rand(R)
        s["temperature"] = 0.6 + 0.6 * rand(R)
        s["temperature"] = s["temperature"] * (rand(R) >= 0.05)               # 0: a request that wants the best token
        k = case["top_k"]
        s["k"] = (1 + (k * (0.5 + 0.5 * rand(R))).int()).clamp_max(k).to(torch.int32) if k else None
        s["p"] = case["top_p"] + 0.04 * rand(R) if case["top_p"] else None
        s["m"] = case["min_p"] * (0.5 + rand(R)) if case["min_p"] else None
    return s


# ------------------------------------------------------------------ one pass

def _plain_rows(s):
    h = s["x"].float() if s["residual"] is None else s["x"].float() + s["residual"].float()
    h = h.to(s["x"].dtype)
    f = h.float()
    codes, byte = _encode_rows(f * s["weight"])
    out = {"codes": codes, "exps": byte, "scale": torch.rsqrt(f.square().mean(-1) + EPS)}
    if s["residual"] is not None:
        out["h"] = h
    return out


def _plain_matmul(s):
    y = _decode_rows(s["a"], s["a_exps"]) @ _decode_rows(s["w"], s["w_exps"]).t()
    if s["a_scale"] is not None:
        y = y * s["a_scale"].unsqueeze(1)
    if s["bias_v"] is not None:
        y = y + s["bias_v"]
    if s["res"] is not None:
        y = y + s["res"].float()
    if s["relu"]:
        y = y.clamp_min(0.0)
    return y.to(_type(s["out"]))


def _plain_cache(s):
    page, block, new = s["page"], s["block"], s["new"]
    lens, table = s["lens"].long(), s["table"].long()
    begin = lens - new                                                       # place of a sequence's first new token
    blocks = (new + block - 2) // block + 1                                  # at most so many blocks are touched
    place = (begin // block * block).unsqueeze(1) + torch.arange(blocks * block, device="cuda")   # [n][blocks * block]
    fresh = (place >= begin.unsqueeze(1)) & (place < lens.unsqueeze(1))
    live = place < lens.unsqueeze(1)                                         # fresh, or held in the same block
    pg = table.gather(1, (place // page).clamp_max(table.shape[1] - 1))
    src = (s["starts"][:-1].long().unsqueeze(1) + place - begin.unsqueeze(1)).clamp(0, s["k"].shape[0] - 1)
    group = lambda t: t.unflatten(1, (blocks, block))  # noqa: E731
    for codes, exps, x in ((*s["kv"][:2], s["k"]), (*s["kv"][2:], s["v"])):
        at = group(pg)[:, :, 0], group(place)[:, :, 0] % page // block       # the blocks' places: [n][blocks]
        e0 = exps[at[0], :, at[1]].int() - 127                               # [n][blocks][heads]
        held = group(codes[pg, :, place % page].float())                     # [n][blocks][block][heads][D]
        held = torch.ldexp(held, e0.unsqueeze(2).unsqueeze(-1))
        is_new = group(fresh).unsqueeze(-1).unsqueeze(-1)
        x = group(x[src].float())
        e1 = _exponent(torch.where(is_new, x.abs(), torch.zeros_like(x)).amax((2, 4)))
        has_old = (group(live) & ~group(fresh)).any(-1).unsqueeze(-1)
        e1 = torch.where(has_old, torch.maximum(e1, e0), e1)
        out = _encode(torch.where(is_new, x, held), e1.unsqueeze(2).unsqueeze(-1)).flatten(1, 2)
        codes.view(torch.uint8)[pg[live], :, place[live] % page] = out.view(torch.uint8)[live]
        touched = group(fresh).any(-1)
        exps[at[0][touched], :, at[1][touched]] = (e1 + 127).to(torch.uint8)[touched]
    r = s["read"].long()
    k, v = (_decode(codes[r // page, :, r % page], exps[r // page, :, r % page // block].unsqueeze(-1))
            for codes, exps in (s["kv"][:2], s["kv"][2:]))
    return {"k": k.to(torch.bfloat16), "v": v.to(torch.bfloat16)}


def _plain_attend(s):
    page, block, KV, H, D = s["page"], s["block"], s["kv_heads"], s["heads"], s["D"]
    table, lens, starts = s["table"].long(), s["lens"].long(), s["starts"].long()
    n, longest, most = s["seqs"], s["longest"], s["new"]
    news = starts[1:] - starts[:-1]
    at = torch.arange(longest, device="cuda")
    pages, place = table[:, at // page], (at % page).expand(n, -1)

    def held(codes, exps):   # [sequence][key head][place][D]
        return _decode(codes[pages, :, place], exps[pages, :, place // block].unsqueeze(-1)).transpose(1, 2).contiguous()

    # queries as rows of [sequence][key head][token * query head of the group]
    tok = torch.arange(most, device="cuda")
    row = (starts[:-1].unsqueeze(1) + tok).clamp_max(s["q"].shape[0] - 1)
    q = s["q"].float()[row].reshape(n, most, KV, H // KV, D).transpose(1, 2).reshape(n, KV, most * (H // KV), D)
    p = torch.matmul(q, held(*s["kv"][:2]).transpose(2, 3)).mul_(s["scale"])
    pos = (lens - news).unsqueeze(1) + tok                                  # place of each query in its sequence
    seen = (at <= pos.unsqueeze(2)) & (at < lens.view(n, 1, 1))
    if s["window"]:
        seen &= at > pos.unsqueeze(2) - s["window"]
    seen = seen.unsqueeze(1).unsqueeze(3)
    p = p.view(n, KV, most, H // KV, longest).masked_fill_(~seen, float("-inf"))
    top = p.amax(-1, keepdim=True)
    p = p.sub_(torch.where(top == float("-inf"), torch.zeros_like(top), top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(n, KV, most * (H // KV), longest), held(*s["kv"][2:])).view(n, KV, most, H // KV, D)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    o = o.transpose(1, 2).reshape(n, most, H, D)
    return o[tok < news.unsqueeze(1)].to(torch.bfloat16)


def _plain_sample(s):
    x = s["logits"].double() + 0.0                                          # -0 and 0 are one value
    best, order = x.sort(dim=1, descending=True, stable=True)
    rank = torch.arange(x.shape[1], device="cuda").unsqueeze(0)
    t = s["temperature"].double().unsqueeze(1)
    greedy = t <= 0
    w = torch.exp((best - best[:, :1]) / torch.where(greedy, torch.ones_like(t), t))
    keep = rank < torch.where(greedy, 1, x.shape[1] if s["k"] is None else s["k"].long().unsqueeze(1))
    if s["p"] is not None:
        in_k = w * keep
        before = in_k.cumsum(1).roll(1, 1)
        before[:, 0] = 0
        keep = keep & (before < s["p"].double().unsqueeze(1) * in_k.sum(1, keepdim=True))
    if s["m"] is not None:
        keep = keep & (w >= s["m"].double().unsqueeze(1))
    w = torch.zeros_like(w).scatter_(1, order, w * keep)                    # in the vocabulary's order
    total = w.sum(1, keepdim=True)
    hit = (w.cumsum(1) > s["u"].double().unsqueeze(1) * total) & (w > 0)
    token = hit.to(torch.uint8).argmax(1, keepdim=True)
    return {"token": token.squeeze(1).to(torch.int32), "logprob": torch.log(w.gather(1, token) / total).squeeze(1).float()}


def run(s):
    op = s["op"]
    if not own:
        return {"rows": _plain_rows, "matmul": _plain_matmul, "cache": _plain_cache, "attend": _plain_attend,
                "sample": _plain_sample}[op](s)
    from paper_1907_02154_amd import quant, sample
    if op == "rows":
        codes, exps, scale, h = quant.rmsnorm_f8(s["x"], s["weight"], residual=s["residual"], eps=EPS)
        out = {"codes": codes, "exps": exps, "scale": scale}
        return out if h is None else {**out, "h": h}
    if op == "matmul":
        return quant.matmul_f8(s["a"], s["a_exps"], s["w"], s["w_exps"], a_scale=s["a_scale"], bias=s["bias_v"],
                               residual=s["res"], relu=s["relu"], out_dtype=_type(s["out"]))
    if op == "sample":
        token, logprob = sample.tokens(s["logits"], s["u"], temperature=s["temperature"], top_k=s["k"], top_p=s["p"],
                                       min_p=s["m"])
        return {"token": token, "logprob": logprob}
    cache = quant.KV8Cache(*s["kv"])
    if op == "cache":
        quant.kv8_write(s["k"], s["v"], cache, s["table"], s["lens"], starts=s["starts"], max_new=s["new"])
        k, v = quant.kv8_read(s["read"], cache)
        return {"k": k, "v": v}
    return quant.attention_kv8(s["q"], cache, s["table"], s["lens"], starts=s["starts"], max_new=s["new"],
                               max_len=s["longest"], scale=s["scale"], window=s["window"])


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    if case["op"] == "rows":
        M, C, b = case["M"], case["C"], 2 if case["dtype"] == "bf16" else 4
        return {"bytes": M * (C * (b + 1 + (2 * b if case["residual"] else 0)) + -(-C // GROUP) + 4) + 4 * C,
                "flops": 6 * M * C}
    if case["op"] == "matmul":
        M, K, N, b = case["M"], case["K"], case["N"], 2 if case["out"] == "bf16" else 4
        return {"bytes": (M + N) * (K + -(-K // GROUP)) + M * N * b * (2 if case["residual"] else 1) +
                4 * (M * case["scaled"] + N * case["bias"]), "flops": 2 * M * K * N}
    if case["op"] == "cache":
        H, D, b = case["heads"], case["D"], 2 if case["dtype"] == "bf16" else 4
        new = case["seqs"] * case["new"]
        back = sum(min(case["new"] + max(0, case["old"] - 5 * i), case["new"] + 16) for i in range(case["seqs"]))
        return {"bytes": 2 * H * D * (new * (b + 1) + back * (1 + 2)) + 2 * H * (new + back) // case["block"] + 4 * back,
                "flops": 2 * H * D * (4 * new + back)}
    if case["op"] == "sample":
        R, V, b = case["rows"], case["vocab"], 2 if case["dtype"] == "bf16" else 4
        return {"bytes": R * V * b + 28 * R, "flops": 4 * R * V}
    H, KV, D, win = case["heads"], case["kv_heads"], case["D"], case["window"]
    lens = _lengths(case)
    news = _news(case, lens)
    reads = sum(min(n, win + new - 1) if win else n for n, new in zip(lens, news))
    pairs = sum(min(n - new + j + 1, win) if win else n - new + j + 1 for n, new in zip(lens, news) for j in range(new))
    return {"bytes": sum(news) * H * D * 4 + 2 * reads * KV * D + 2 * reads * KV // case["block"],
            "flops": 4 * pairs * H * D}


# ------------------------------------------------------------------ the same in 64 bits

def _power64(top):
    """2^e of a block by its largest magnitude, in 64 bits."""
    return torch.exp2(torch.ceil(torch.log2(top.double().clamp_min(2.0 ** -130) / 448.0)).clamp(-117, 119))


def _near64(x, power):
    """x rounded to the e4m3 grid of a power of two: steps of an eighth of the leading bit, 2^-9 at least."""
    y = x.double() / power
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -20))).clamp_min(-6) - 3)
    return torch.round(y / step) * step * power


def _held64(codes, byte):
    """Values by the format's fields: sign, four bits of exponent, three of mantissa."""
    c = codes.view(torch.uint8).to(torch.int64)
    e, m = (c // 8) % 16, (c % 8).double()
    v = torch.where(e == 0, m / 512, (8 + m) * torch.exp2(e.double() - 10))
    return (1.0 - 2.0 * (c // 128)) * v * torch.exp2(byte.double() - 127)


def _exact_rows(case, s):
    h = s["x"].double()
    if s["residual"] is not None:
        h = h + s["residual"].double()
    kept = h.to(s["x"].dtype).double()              # the stream is held in its own type
    t = (kept.float() * s["weight"]).double()       # and so is what the exponents go by
    blocks = t.split(GROUP, 1)
    out = {"codes": torch.cat([b / _power64(b.abs().amax(1, keepdim=True)) for b in blocks], 1), "exps": None,
           "scale": (torch.einsum("mc,mc->m", kept, kept) / kept.shape[1] + EPS).sqrt().reciprocal()}
    if s["residual"] is not None:
        out["h"] = h
    return out


def _exact_matmul(case, s):
    a, w = (torch.cat([_held64(c, b) for c, b in zip(codes.split(GROUP, 1), byte.split(1, 1))], 1)
            for codes, byte in ((s["a"], s["a_exps"]), (s["w"], s["w_exps"])))
    if s["a_scale"] is not None:
        a = a * s["a_scale"].double()[:, None]
    y = torch.mm(a, w.t())
    for extra in (s["bias_v"], s["res"]):
        y = y if extra is None else y + extra.double()
    return torch.relu(y) if case["relu"] else y


def _exact_cache(case, s):
    """Each sequence's blocks one after another: what a block held, rounded to its new power, and the new tokens."""
    page, block, new = case["page"], case["block"], case["new"]
    table, read = s["table"].long(), s["read"].long()
    out = {}
    for name, codes, exps in (("k", *s["kv"][:2]), ("v", *s["kv"][2:])):
        value = _held64(codes, exps.repeat_interleave(block, 2).unsqueeze(-1))     # [pages][heads][page][D]
        power = torch.exp2(exps.double() - 127)                                    # [pages][heads][page / block]
        for i, n in enumerate(s["lens"].tolist()):
            x = s[name][i * new:(i + 1) * new].double()                            # [new][heads][D]
            first = (n - new) // block
            padded = torch.zeros(-(-n // block) * block - first * block, *x.shape[1:], dtype=torch.float64, device="cuda")
            padded[n - new - first * block:n - first * block] = x
            b = padded.unflatten(0, (-1, block))                                   # [blocks][block][heads][D]
            at = torch.arange(first, first + b.shape[0], device="cuda")
            pg, slot = table[i, at * block // page], at * block % page // block
            p = _power64(b.abs().amax((1, 3)))                                     # [blocks][heads]
            if n - new > first * block:
                p[0] = torch.maximum(p[0], power[pg[0], :, slot[0]])
            power[pg, :, slot] = p
            t = torch.arange(first * block, n, device="cuda")
            tp, tq = table[i, t // page], t % page
            fill = torch.cat((value[tp, :, tq][:n - new - first * block], x))
            fill = _near64(fill, p.repeat_interleave(block, 0)[:len(t)].unsqueeze(-1))
            value[tp, :, tq] = fill
        out[name] = value[read // page, :, read % page]
    return out


def _exact_attend(case, s):
    H, KV, page, block = case["heads"], case["kv_heads"], case["page"], case["block"]
    starts, lens, table = s["starts"].tolist(), s["lens"].tolist(), s["table"].long()
    out = torch.zeros(starts[-1], H, case["D"], dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        q = s["q"][starts[b]:starts[b + 1]].double()
        at = torch.arange(n, device="cuda")
        pg, place = table[b, at // page], at % page
        pos = n - q.shape[0] + torch.arange(q.shape[0], device="cuda")
        bad = at[None, :] > pos[:, None]
        if case["window"]:
            bad |= pos[:, None] - at[None, :] >= case["window"]
        for h in range(KV):
            k, v = (_held64(codes[pg, h, place], exps[pg, h, place // block].unsqueeze(-1))
                    for codes, exps in (s["kv"][:2], s["kv"][2:]))
            for j in range(h * (H // KV), (h + 1) * (H // KV)):
                score = (q[:, j] @ k.t() * s["scale"]).masked_fill(bad, -math.inf)
                out[starts[b]:starts[b + 1], j] = torch.softmax(score, -1) @ v
    return out


def _exact_sample(case, s):
    """Row by row: the tokens ordered, the filters as the lengths of a prefix, the pick by its place in the kept ones."""
    out = torch.zeros(case["rows"], dtype=torch.float64, device="cuda")
    for i in range(case["rows"]):
        x, t = s["logits"][i].double(), float(s["temperature"][i])
        if t <= 0:
            continue                                                         # the best token, with probability 1
        order = torch.argsort(-x, stable=True)
        k = len(order) if s["k"] is None else int(s["k"][i])
        order = order[:k]
        p = torch.softmax(x[order] / t, 0)
        n = k
        if s["p"] is not None:
            n = min(n, 1 + int((p.cumsum(0) < float(s["p"][i])).sum()))
        if s["m"] is not None:
            n = min(n, int((x[order] - x[order[0]] >= t * math.log(float(s["m"][i]))).sum()))
        kept = order[:n].sort().values
        p = torch.softmax(x[kept] / t, 0)
        at = int(torch.searchsorted(p.cumsum(0), s["u"][i].double(), right=True).clamp_max(n - 1))
        out[i] = torch.log_softmax(x[kept] / t, 0)[at]
    return {"token": None, "logprob": out}


def exact(case, seed):
    s = prepare(case, seed)
    return {"rows": _exact_rows, "matmul": _exact_matmul, "cache": _exact_cache, "attend": _exact_attend,
            "sample": _exact_sample}[case["op"]](case, s)
