"""GPU: the pick of a token from vocabularies of 2^19 to 2^25 tokens, whose partial sums are more than one wavefront
looks through, of runs of 8 and of 16 units."""
import math

import numpy as np
import pytest
import torch

from oracle import sample as ref
from paper_1907_02154_amd import sample

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
DRAWS = [0.0, 0.25, 0.6180339, 0.9, 1 - 2.0 ** -24]


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sample.lib()


def drawn(x, u, **k):
    rows = x.shape[0]
    dev = {n: torch.full((rows,), v, dtype=torch.int32 if n == "top_k" else F32, device="cuda") for n, v in k.items()}
    token, logprob = sample.tokens(x, torch.full((rows,), u, dtype=F32, device="cuda"), **dev)
    return token.tolist(), logprob.tolist()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("vocab", [2 ** 19 + 77, 2 ** 24 + 5000, 2 ** 25])
def test_ties_over_many_runs(vocab, dtype):
    """Equal logits, every third or in two stretches, among forbidden tokens and ones 40 below, whose weights are less than
    half of what weights are multiples of.  All numbers here have 48 bits at most, so that the token follows by counting."""
    i = torch.arange(vocab, device="cuda")
    for top in (2.5, -300.0):                                    # within and outside the range of bf16's counters
        for equal in (i % 3 == 1, (i < 700) | (i > vocab - 9000)):
            for rest in (-math.inf, top - 40):
                x = torch.where(equal, top, rest).to(dtype)[None]
                at = equal.nonzero()[:, 0].cpu()
                n = len(at)
                for u in DRAWS if vocab < 2 ** 20 else DRAWS[2::2]:
                    u = float(np.float32(u))
                    for kept, k in ((n, dict()), (n // 2, dict(top_k=n // 2)), (3, dict(top_k=3)), (n, dict(top_k=n + 5)),
                                    (math.ceil(float(np.float32(0.3)) * n), dict(top_p=0.3)), (n, dict(min_p=1.0)),
                                    (math.ceil(0.5 * (n - 1)), dict(top_k=n - 1, top_p=0.5))):
                        token, lp = drawn(x, u, **k)
                        assert token == [int(at[math.floor(u * kept)])], (top, rest, u, kept, k)
                        assert abs(lp[0] + math.log(kept)) <= 2.0 ** -23 * math.log(kept), (top, rest, u, kept, k)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_draws_from_600001_tokens(dtype):
    """Against the oracle.  Each of n weights may be off by one of the 2^-42 that they are multiples of, where it lies next to a
    half of it, and by 2^-50 of itself; so may a sum of theirs, by n times that, as a share of their sum."""
    vocab, rows = 600001, 2
    g = torch.Generator().manual_seed(5)
    x = 2.5 * torch.randn(rows, vocab, generator=g)
    x[:, torch.randperm(vocab, generator=g)[:8]] += 12
    x = x.to(dtype)
    d, host = x.cuda(), x.double().numpy()
    for f in (dict(), dict(temperature=0.5), dict(top_k=50), dict(top_k=40000), dict(top_p=0.9), dict(min_p=0.001),
              dict(top_k=100000, top_p=0.95, min_p=1e-5, temperature=1.5), dict(temperature=3.0, top_p=0.5)):
        k = {n: v if n == "top_k" else float(np.float32(v)) for n, v in f.items()}
        for u in DRAWS:
            token, lp = drawn(d, u, **f)
            for r in range(rows):
                want, want_lp, margin = ref.pick(host[r], float(np.float32(u)), **k)
                w = np.sort(np.exp((host[r] - host[r].max()) / k.get("temperature", 1.0)))[::-1][:k.get("top_k", vocab)]
                off = (2 * len(w) * 2.0 ** -42 + w.sum() * 2.0 ** -49) / (min(1.0, k.get("top_p", 1.0)) * w.sum())
                if token[r] != want:
                    assert margin < off and 0 < u < 0.95, (f, u, r, token[r], want, margin, off)
                else:
                    assert abs(lp[r] - want_lp) <= 2.0 ** -23 * abs(want_lp) + 2.0 ** -24 + off, (f, u, r, lp[r], want_lp)
