"""GPU: the pick of a token (include/misample.h) against the oracle
(oracle/sample.py), through the binding.

Tokens are whole numbers and compared as such.  A row may only differ where the
oracle's own number lies within MARGIN of a border: weights are multiples of
2^-45 of the largest at least for the vocabularies here, each off by half of
that and by 2^-46 of itself, and 2^18 of them are added.
"""
import math

import numpy as np
import pytest
import torch

from oracle import sample as ref
from paper_1907_02154_amd import miconv, sample

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
MARGIN = 2.0 ** (18 - 45)


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sample.lib()


def gen(seed):
    return torch.Generator().manual_seed(seed)


def check(x, u, strict=True, **k):
    """x [rows][vocab] on the host; temperature, top_k, top_p, min_p lists or None."""
    dev = {n: torch.tensor(v, dtype=torch.int32 if n == "top_k" else F32, device="cuda") for n, v in k.items() if v is not None}
    token, logprob = sample.tokens(x.cuda(), torch.tensor(u, device="cuda"), **dev)
    token, logprob = token.cpu(), logprob.cpu()
    u32 = np.asarray(u, dtype=np.float32).astype(np.float64)
    off = 0
    for r in range(x.shape[0]):
        one = {n: (int(v[r]) if n == "top_k" else float(np.float32(v[r]))) for n, v in k.items() if v is not None}
        t, lp, margin = ref.pick(x[r].double().numpy(), float(u32[r]), **one)
        if int(token[r]) != t:
            assert not strict or margin < MARGIN, (r, int(token[r]), t, margin, one, float(u32[r]))
            off += 1
            continue
        if math.isnan(lp):
            assert math.isnan(float(logprob[r])), r
        else:
            assert abs(float(logprob[r]) - lp) <= 2.0 ** -23 * abs(lp) + 2.0 ** -24, (r, float(logprob[r]), lp)   # 64 bits, rounded once
    assert off <= 0.02 * x.shape[0]
    return token, logprob


def logits(g, rows, vocab, dtype, spread=2.5):
    x = spread * torch.randn(rows, vocab, generator=g)
    x[:, :min(5, vocab)] += 8 * torch.rand(rows, min(5, vocab), generator=g)
    return x[:, torch.randperm(vocab, generator=g)].contiguous().to(dtype)


FILTERS = [dict(), dict(top_k=True), dict(top_p=True), dict(min_p=True), dict(top_k=True, top_p=True),
           dict(top_p=True, min_p=True), dict(top_k=True, top_p=True, min_p=True)]
VOCABS = [1, 2, 5, 64, 511, 512, 513, 1000, 4096, 4097, 8191, 20000, 32000, 50001]


def ids(f):
    return "-".join(f) or "none"


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("filters", FILTERS, ids=ids)
@pytest.mark.parametrize("vocab", VOCABS)
def test_draws(vocab, filters, dtype):
    g = gen(vocab + len(filters))
    rows = 40 if vocab < 4000 else 12
    x = logits(g, rows, vocab, dtype)
    rand = lambda: torch.rand(rows, generator=g)  # noqa: E731
    k = {"temperature": (0.1 + 1.5 * rand()).tolist()}
    if "top_k" in filters:
        k["top_k"] = (1 + (rand() * min(vocab, 300)).int()).tolist()
        k["top_k"][0] = 1
    if "top_p" in filters:
        k["top_p"] = (0.05 + 0.94 * rand()).tolist()
    if "min_p" in filters:
        k["min_p"] = (0.3 * rand()).tolist()
    check(x, rand().tolist(), **k)


@pytest.mark.parametrize("vocab", [130000, 260000])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_large_vocabularies(vocab, dtype):
    g = gen(vocab)
    x = logits(g, 6, vocab, dtype)
    u = torch.rand(6, generator=g).tolist()
    for k in (dict(), dict(top_p=[.5, .9, .95, .99, .999, .1]), dict(top_k=[50, 1000, 5000, 20000, 100000, 3]),
              dict(top_k=[50, 1000, 5000, 20000, 100000, 3], top_p=[.9] * 6), dict(min_p=[.05] * 6), dict(top_p=[.9] * 6, min_p=[.001] * 6)):
        check(x, u, temperature=[.2, .7, 1, 1.5, 3, .05], **k)


@pytest.mark.parametrize("vocab", [7, 1000, 6000, 40000])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_equal_logits(vocab, dtype):
    """Nothing but ties, of one value and of a few, and of 0 and -0: the lowest indexes are kept, whatever does not fit a list."""
    g = gen(vocab)
    few = torch.tensor([0.0, -0.0, 1.0, -3.0])
    x = torch.stack([torch.full((vocab,), 0.3), torch.zeros(vocab), few[torch.randint(0, 2, (vocab,), generator=g)],
                     few[torch.randint(0, 4, (vocab,), generator=g)], torch.full((vocab,), -1e30), torch.full((vocab,), 1e30)]).to(dtype)
    for frac in (0.0, 0.1, 0.5, 0.77, 1 - 2.0 ** -24):
        u = [frac] * 6
        check(x, u)
        kk = [1, 3, max(1, vocab // 2), vocab - 1, vocab, 5]
        t, _ = check(x, u, top_k=kk)
        assert int(t[1]) <= 2                                    # the first three of equal ones
        check(x, u, top_p=[0.25, 0.5, 0.75, 0.5, 0.125, 0.9])
        check(x, u, top_k=kk, top_p=[0.5] * 6)
        check(x, u, min_p=[1.0] * 6)


@pytest.mark.parametrize("vocab", [4097, 40000, 70001])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_the_first_few(vocab, dtype):
    """k around what one wavefront finishes, of rows with more candidates than k (ties, and a thread's own), with fewer tokens
    than k, with logits of every size; and the first alone."""
    g = gen(vocab)
    base = logits(g, 1, vocab, F32)
    tied = torch.randn(1, vocab, generator=g)
    tied[0, torch.randperm(vocab, generator=g)[:90]] = 7.0
    near = torch.randn(1, vocab, generator=g)
    near[0, 512:1024] = 9 + torch.rand(512, generator=g)         # the largest in one unit
    left = torch.full((1, vocab), -math.inf)
    left[0, torch.randperm(vocab, generator=g)[:20]] = torch.randn(20, generator=g)
    tiny, huge = 1e-4 * base, 1e4 * base
    x = torch.cat([base, tied, near, left, tiny, huge]).to(dtype)
    for k in (1, 2, 19, 20, 48, 55, 56, 57, 64, 65, 128):
        for u in (0.0, 0.4, 0.93):
            check(x, [u] * 6, top_k=[k] * 6)
        check(x, [0.7] * 6, top_k=[k] * 6, top_p=[0.9, 0.5, 0.0, 0.9, 1.0, 0.3], min_p=[0.0, 0.1, 0.0, 0.2, 0.0, 1.0], temperature=[0.9] * 6)
    t, lp = check(x, [0.5] * 6, temperature=[0.0, -1.0, 0.0, 0.0, 1.0, math.nan], top_k=[5, 0, 1, 70, 0, 0])
    assert lp[:4].tolist() == [0.0] * 4 and t[1] == int((x[1] == 7).nonzero()[0])


def test_masks_and_extremes():
    g = gen(3)
    low = torch.finfo(F32).min
    x = 3 * torch.randn(14, 5000, generator=g)
    x[0, 100:] = -math.inf                                       # most of it forbidden
    x[1] = -math.inf                                             # all of it
    x[2], x[2, 4321] = -math.inf, -5.0                           # one left
    x[3, 10:] = low                                              # forbidden by the type's lowest value
    x[4] = low                                                   # all equal
    x[5, 7] = math.nan
    x[6, 4999] = math.inf
    x[7], x[7, 77] = -1e38, 3e38                                 # differences pass fp32
    x[8] *= 1e30
    x[9] *= 1e-30
    x[10] = torch.arange(5000).float() * 1e-3
    x[11, 2:] = -math.inf
    x[12] *= 200
    x[13, :4990] = low
    none = [1, 5, 6]
    for u in (0.0, 0.3, 0.999):
        for k in (dict(), dict(top_k=[200] * 14), dict(top_p=[.9] * 14), dict(top_k=[4999] * 14, top_p=[.99] * 14, min_p=[1e-4] * 14),
                  dict(min_p=[.2] * 14), dict(temperature=[1e-3] * 14), dict(temperature=[1e4] * 14, top_p=[.5] * 14),
                  dict(temperature=[math.inf] * 14), dict(temperature=[1e-44] * 14), dict(temperature=[3e38] * 14, top_k=[30] * 14)):
            t, lp = check(x, [u] * 14, **k)
            assert all(int(t[i]) == -1 and math.isnan(float(lp[i])) for i in none)
            assert int(t[2]) == 4321 and float(lp[2]) == 0 and 0 <= int(t[0]) < 100
        check(x.to(BF16), [u] * 14)


def test_parameters_at_their_ends():
    g = gen(4)
    x = logits(g, 12, 3001, F32)
    best = x.argmax(1)
    inf, nan = math.inf, math.nan
    t, lp = check(x, [.5] * 12, temperature=[0.0, -0.0, -1.0, nan, -inf, 0.0] * 2, top_k=[3] * 12)
    assert torch.equal(t.long(), best) and (lp == 0).all()
    plain = check(x, [.7] * 12)[0]
    for k in (dict(top_k=[0, -1, -2 ** 31, 3001, 2 ** 31 - 1, 3002] * 2), dict(top_p=[1.0, 1.5, inf, nan, 1.0, 2.0] * 2),
              dict(min_p=[0.0, -1.0, -inf, nan, 0.0, -0.0] * 2)):
        assert torch.equal(check(x, [.7] * 12, **k)[0], plain)
    for k in (dict(top_k=[1] * 12), dict(top_p=[0.0, -1.0, -inf, 1e-45] * 3), dict(min_p=[1.0, 2.0, inf] * 4),
              dict(top_k=[40] * 12, top_p=[0.0, -1.0, -inf, 1e-45] * 3)):
        t, lp = check(x, [.7] * 12, **k)
        assert torch.equal(t.long(), best) and (lp == 0).all()
    first = check(x, [0.0] * 12)[0]
    assert torch.equal(check(x, [-1.0, -inf, nan, -0.0] * 3)[0], first)
    last = check(x, [1 - 2.0 ** -24] * 12)[0]
    assert torch.equal(check(x, [1.0, 2.0, inf] * 4)[0], last)


@pytest.mark.parametrize("vocab", [12000, 70000])
def test_more_candidates_than_a_list_holds(vocab):
    """Logits so close that a bin holds most of the row, beside one far above or below."""
    g = gen(vocab)
    for far in (40.0, -40.0, 0.0, -3e38):
        for dtype in (F32, BF16):
            x = (1 + 1e-3 * torch.randn(4, vocab, generator=g))
            x[:, 17] += far
            x = x.to(dtype)
            u = torch.rand(4, generator=g).tolist()
            kk = [4097, 5000, vocab // 2, vocab - 1]
            check(x, u, top_k=kk)
            check(x, u, top_p=[.5, .9, .3, .999], temperature=[1.0, 20.0, 5.0, 40.0])
            check(x, u, top_k=kk, top_p=[.5, .9, .3, .999], temperature=[1.0, 20.0, 5.0, 40.0])


@pytest.mark.parametrize("vocab", [5000, 30011])
@pytest.mark.parametrize("share", [0.01, 0.05, 0.5])
def test_bf16_logits_outside_the_range_of_the_counters(vocab, share):
    """Large and tiny magnitudes of either sign among the others, a few and more than a list holds, at every filter's end."""
    g = gen(vocab + int(100 * share))
    x = 2 * torch.randn(8, vocab, generator=g)
    kind = torch.rand(8, vocab, generator=g)
    tiny = torch.randn(8, vocab, generator=g) * 2.0 ** -12
    huge = (130 + 5 * torch.rand(8, vocab, generator=g)) * torch.sign(torch.randn(8, vocab, generator=g))
    x = torch.where(kind < share, tiny, x)
    for part in (x, torch.where((kind > 1 - share) & (torch.arange(8)[:, None] % 2 == 0), huge, x), x * 1e-4,
                 x.clamp(max=0), torch.where(kind > share, torch.full_like(x, -math.inf), x), 100 * x):
        part = part.to(BF16)
        u = torch.rand(8, generator=g).tolist()
        t = [0.3, 1.0, 2.0, 5.0, 0.0, 1.0, 30.0, 0.05]
        for k in (dict(), dict(top_k=[1, 2, 40, vocab // 3, 5, vocab // 2, vocab - 1, 4000]),
                  dict(top_p=[.1, .5, .9, .99, .5, .3, .7, .95]), dict(min_p=[.5, .1, .01, .9, .5, 1.0, .99, 1e-6]),
                  dict(top_k=[1, 2, 40, vocab // 3, 5, vocab // 2, vocab - 1, 4000], top_p=[.1, .5, .9, .99, .5, .3, .7, .95],
                       min_p=[.5, .1, .01, .9, .5, .2, .99, 1e-6])):
            check(part, u, temperature=t, **k)


def test_every_token_is_reached():
    """u over a fine grid: each token as often as its weight says, in the vocabulary's order."""
    x = torch.tensor([[0.0, math.log(3.0), -math.inf, math.log(2.0), 0.0, math.log(0.5)]])
    n = 7500
    u = (torch.arange(n) + 0.5) / n
    t, _ = sample.tokens(x.expand(n, 6).contiguous().cuda(), u.cuda())
    assert torch.bincount(t.cpu().long(), minlength=6).tolist() == [1000, 3000, 0, 2000, 1000, 500]
    assert (t.cpu()[1:] >= t.cpu()[:-1]).all()


def test_strides_and_outputs():
    g = gen(6)
    for dtype in (F32, BF16):
        wide = torch.randn(9, 1300, generator=g).to(dtype)
        wide[:, :3], wide[:, 3 + 1201:] = math.nan, math.nan
        d = wide.cuda()
        u = torch.rand(9, generator=g)
        out, lp = torch.full((11,), 7, dtype=torch.int32, device="cuda"), torch.full((11,), 7.0, device="cuda")
        got = sample.tokens(d[:, 3:3 + 1201], u.cuda(), out=out[1:10], logprob=lp[1:10])
        want = sample.tokens(wide[:, 3:3 + 1201].contiguous().cuda(), u.cuda())
        assert got[0].data_ptr() == out[1:].data_ptr() and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert int(out[0]) == int(out[10]) == 7 and float(lp[0]) == float(lp[10]) == 7
    e = sample.tokens(torch.empty(0, 50, device="cuda"), torch.empty(0, device="cuda"))
    assert e[0].shape == (0,) and e[1].shape == (0,)


def test_many_rows_are_the_same_bits_on_another_stream_and_in_a_graph():
    g = gen(8)
    rows, vocab = 300, 9000
    x = logits(g, rows, vocab, BF16).cuda()
    u, p = torch.rand(rows, generator=g).cuda(), (0.5 + 0.5 * torch.rand(rows, generator=g)).cuda()
    k = torch.randint(-5, 9000, (rows,), generator=g).to(torch.int32).cuda()
    first = sample.tokens(x, u, top_k=k, top_p=p)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream, 0, None):
        again = sample.tokens(x, u, top_k=k, top_p=p, stream=stream)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, again))
    out, lp = torch.empty_like(first[0]), torch.empty_like(first[1])
    with torch.cuda.stream(side):
        sample.tokens(x, u, top_k=k, top_p=p, out=out, logprob=lp)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sample.tokens(x, u, top_k=k, top_p=p, out=out, logprob=lp)
    for _ in range(4):
        u.copy_(torch.rand(rows, generator=g))
        graph.replay()
        torch.cuda.synchronize()
        want = sample.tokens(x, u, top_k=k, top_p=p)
        assert torch.equal(out, want[0]) and torch.equal(lp, want[1])


def test_binding_refusals():
    x, u = torch.zeros(4, 64, device="cuda"), torch.zeros(4, device="cuda")
    i = torch.ones(4, dtype=torch.int32, device="cuda")
    bad = [lambda: sample.tokens(x.half(), u), lambda: sample.tokens(x.t(), u), lambda: sample.tokens(x[0], u),
           lambda: sample.tokens(x, u[:3]), lambda: sample.tokens(x, u.double()), lambda: sample.tokens(x, u, temperature=i),
           lambda: sample.tokens(x, u, top_k=u), lambda: sample.tokens(x, u, top_k=i.long()), lambda: sample.tokens(x, u, top_p=0.9),
           lambda: sample.tokens(x, u, min_p=u[:2]), lambda: sample.tokens(x, u, out=i.long()), lambda: sample.tokens(x, u, logprob=i),
           lambda: sample.tokens(x[:, :0], u), lambda: sample.tokens(x.cpu(), u.cpu()), lambda: sample.tokens(x, u.cpu()),
           lambda: sample.tokens(x[:1].expand(4, 64), u)]
    for n, f in enumerate(bad):
        with pytest.raises((ValueError, TypeError, miconv.MiconvError)):
            f()
            print("case", n)
