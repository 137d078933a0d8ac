"""GPU: the pick of a token where min_p ends what is kept, against the oracle (oracle/sample.py), through the binding."""
import math

import pytest
import torch

from paper_1907_02154_amd import sample
from test_gpu_sample import BF16, F32, check, gen

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sample.lib()


def near_zero(step, dtype):
    """(temperature, largest logit, min_p) with the logit that min_p stands for, top + T ln(min_p), within rounding of 0,
    where floats lie closer than weights can tell apart."""
    out = [(1.0, float.fromhex("0x1.3684f8p+2"), float.fromhex("0x1.000ac8p-7"))] if dtype is F32 else []
    for t in (0.25, 0.5, 0.7, 1.0, 1.25, 2.0):
        for i in range(math.ceil(2 ** -4 / step), int(12 / step)):
            top = i * step
            m = math.exp(-top / float(torch.tensor(t)))
            if m > 1e-6 and float(torch.tensor(top).to(dtype)) == top:
                out.append((t, top, m))
    return out


def rows_below(g, tops, vocab, dtype):
    """Rows of logits from -1 to their largest, none nearer to 0 than 2^-6, which no rounding of a threshold at 0 reaches."""
    x = torch.rand(len(tops), vocab, generator=g) * (tops[:, None] + 1) - 1
    x = torch.where(x.abs() < 2.0 ** -6, torch.full_like(x, -0.5), torch.minimum(x, 0.97 * tops[:, None]))
    x[:, vocab // 3] = tops
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("vocab", [5, 40])
def test_a_min_p_whose_logit_is_zero(vocab, dtype):
    """Every token of a positive logit stays, each of a negative one goes."""
    t, top, m = zip(*near_zero(1 / 128, dtype))
    g = gen(vocab)
    x = rows_below(g, torch.tensor(top), vocab, dtype)
    u = torch.rand(len(t), generator=g).tolist()
    check(x, u, temperature=t, min_p=m)
    check(x, u, temperature=t, min_p=m, top_k=[4] * len(t))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("filters", [dict(), dict(top_k=50), dict(top_k=200), dict(top_p=0.999), dict(top_k=3000, top_p=0.98)],
                         ids=lambda f: "-".join(f"{n}{v}" for n, v in f.items()) or "none")
def test_a_min_p_whose_logit_is_zero_in_long_rows(filters, dtype):
    t, top, m = zip(*near_zero(1 / 32, dtype))
    g = gen(len(filters))
    x = rows_below(g, torch.tensor(top), 4500, dtype)
    x = torch.where((torch.arange(4500) % 23 > 0) & (x > 0), -x, x)   # 196 above the threshold at most, so that filters reach it
    x[:, 1500] = torch.tensor(top).to(dtype)
    u = torch.rand(len(t), generator=g).tolist()
    check(x, u, temperature=t, min_p=m, **{n: [v] * len(t) for n, v in filters.items()})


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("vocab", [5, 900, 4500, 40000])
def test_a_min_p_above_one_keeps_one_of_equal_tokens(vocab, dtype):
    """The largest logit many times, within and outside the range of the counters of bf16 rows; of min_p = 1 all of them stay."""
    g = gen(vocab)
    x = torch.rand(6, vocab, generator=g) - 1.5
    tops = torch.tensor([3.0, 200.0, 2.0 ** -12, -2.0 ** -12, 0.25, 0.0])
    equal = torch.rand(vocab, generator=g) < 0.3
    equal[[1, 3]] = True
    x[:, equal] = tops[:, None]
    x[5, equal] *= torch.where(torch.arange(int(equal.sum())) % 2 == 0, -1.0, 1.0)      # -0 and 0
    x = x.to(dtype)
    first = int(equal.nonzero()[0])
    above = [math.nextafter(1.0, 2.0) + 2.0 ** -23, 2.0, math.inf, 1e30, 1.5, 4.0]
    for u in (0.0, 0.6, 0.999):
        for k in (dict(), dict(top_k=[2, 3, 4, 50, 4000, 60]), dict(top_p=[0.9] * 6), dict(top_k=[4, 50, 200, 5000, 4, 300], top_p=[0.99] * 6)):
            for t in ([1.0] * 6, [0.3, 2.0, 1e-3, 50.0, 1.0, 0.7]):
                token, lp = check(x, [u] * 6, temperature=t, min_p=above, **k)
                assert token.tolist() == [first] * 6 and (lp == 0).all()
                check(x, [u] * 6, temperature=t, min_p=[1.0] * 6, **k)
