"""Host-side checks of the pick of a token (no GPU needed): refusals before any launch, and the oracle by hand."""
import math

import numpy as np
import pytest
import torch

from oracle import sample as ref
from paper_1907_02154_amd import miconv, sample
from test_quant_host import FAKE, call, placed


@pytest.fixture(scope="module")
def L():
    return sample.lib()


def test_refusals(L):
    d = [("rows", 2), ("vocab", 100), ("dtype", 1), ("x", FAKE), ("stride", 100), ("u", FAKE), ("t", None), ("k", None), ("p", None),
         ("m", None), ("token", FAKE), ("lp", None), ("ws", None), ("wsb", 0), ("st", None)]
    f = lambda **k: call(L.sample_tokens, d, **k)  # noqa: E731
    for n in ("sample_tokens", "sample_tokens_workspace_bytes"):
        assert n in miconv.header_functions() and hasattr(L, n)
    for k in (dict(rows=-1), dict(vocab=0), dict(stride=99)):
        assert f(**k) == miconv.ERR_SHAPE, k
    for k in (dict(x=None), dict(u=None), dict(token=None)):
        assert f(**k) == miconv.ERR_NULL, k
    for n in ("u", "t", "k", "p", "m", "token", "lp"):
        assert f(**{n: FAKE + 2}) == miconv.ERR_ALIGN, n
    assert f(x=FAKE + 1) == f(dtype=0, x=FAKE + 2) == miconv.ERR_ALIGN
    assert f(dtype=2) == miconv.ERR_UNSUPPORTED
    big = (1 << 25) + 1
    assert f(vocab=big, stride=big) == f(rows=1 << 22) == miconv.ERR_TOO_LARGE
    assert f(rows=0, x=None, u=None, token=None) == miconv.OK
    w = L.sample_tokens_workspace_bytes
    assert w(-1, 5, 0) == w(1, 0, 0) == miconv.ERR_SHAPE and w(1, 5, 3) == miconv.ERR_UNSUPPORTED
    assert w(1, big, 0) == miconv.ERR_TOO_LARGE and w(0, 5, 0) == 0
    with pytest.raises(TypeError):
        sample.tokens_workspace_bytes(1, 5, torch.float16)


def test_binding_refuses_operands_on_another_device(monkeypatch):
    from paper_1907_02154_amd import quant
    monkeypatch.setattr(quant, "_getdevice", lambda: 0)

    class Called(Exception):
        pass

    class Library:
        def __getattr__(self, name):
            if name.endswith("_workspace_bytes"):
                return lambda *a: 0
            raise Called(name)
    monkeypatch.setattr(sample, "lib", Library)
    f32, i32 = torch.float32, torch.int32
    kinds = [((4, 64), torch.bfloat16), ((4,), f32), ((4,), f32), ((4,), i32), ((4,), f32), ((4,), f32), ((4,), i32), ((4,), f32)]
    make = lambda at: [placed(d, *k[0], dtype=k[1]) for k, d in zip(kinds, at)]  # noqa: E731
    f = lambda x, u, t, k, p, m, o, lp: sample.tokens(x, u, t, k, p, m, out=o, logprob=lp, stream=0)  # noqa: E731
    with pytest.raises(Called):
        f(*make([0] * 8))
    for i in range(8):
        with pytest.raises(ValueError, match="device"):
            f(*make([int(i == j) for j in range(8)]))
    with pytest.raises(ValueError, match="device"):
        sample.tokens(torch.zeros(2, 8), torch.zeros(2))


def test_oracle_by_hand():
    x = np.log(np.array([1.0, 4.0, 2.0, 4.0, 1.0]))      # 12 in all; order 1, 3, 2, 0, 4
    pick = lambda u, **k: ref.pick(x, u, **k)[0]  # noqa: E731
    assert [pick(u / 12 + 1e-6) for u in range(12)] == [0, 1, 1, 1, 1, 2, 2, 3, 3, 3, 3, 4]
    assert [pick(u, top_k=1) for u in (0.0, 0.99)] == [1, 1]
    assert [pick(u, top_k=2) for u in (0.0, 0.49, 0.51)] == [1, 1, 3]
    assert [pick(u, top_k=4) for u in (0.0, 0.08, 0.1, 0.5, 0.99)] == [0, 0, 1, 2, 3]        # of 11
    assert [pick(u, top_p=0.3) for u in (0.0, 0.99)] == [1, 1]                             # 4 of 12 pass .3
    assert [pick(u, top_p=0.34) for u in (0.0, 0.99)] == [1, 3]
    assert [pick(u, top_k=3, top_p=0.39) for u in (0.0, 0.99)] == [1, 1]                   # 4 of 10
    assert [pick(u, top_k=3, top_p=0.41) for u in (0.0, 0.99)] == [1, 3]
    assert [pick(u, min_p=0.4) for u in (0.0, 0.41, 0.99)] == [1, 2, 3]                    # 1, 2, 3 stay: 4 + 2 + 4
    assert [pick(u, temperature=0.5) for u in (0.0, 0.03, 0.99)] == [0, 1, 4]              # weights 1 16 4 16 1
    assert ref.pick(x, 0.5, temperature=0.0)[:2] == (1, 0.0)
    t, lp, _ = ref.pick(x, 0.5, top_k=3)
    assert t == 2 and abs(lp - math.log(0.2)) < 1e-15
    for bad in ([1.0, math.nan], [1.0, math.inf], [-math.inf, -math.inf]):
        t, lp, _ = ref.pick(np.array(bad), 0.5)
        assert t == -1 and math.isnan(lp)
    assert ref.pick(np.array([-math.inf, 2.0, -math.inf]), 0.9)[0] == 1
    # against a draw from the softmax in its own words
    g = np.random.default_rng(0)
    x = g.normal(size=200) * 2
    p = np.exp(x) / np.exp(x).sum()
    for u in g.random(50):
        assert ref.pick(x, u)[0] == int(np.searchsorted(p.cumsum(), u, side="right"))
