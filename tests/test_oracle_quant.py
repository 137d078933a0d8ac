"""Pins of the oracle of the quantised operators (oracle/quant.py): hand-worked
values, and the definitions checked another way."""
import math

import pytest
import torch

from oracle import quant as ref


def test_rows_by_hand():
    x = torch.tensor([[3.0, -4.0, 0.0, 0.0], [0.0, 0.0, 0.0, 0.0], [1.0, math.nan, 2.0, 0.0], [1.0, -math.inf, 2.0, 0.0]])
    q, scale, h = ref.rows_i8(x, eps=0.0)
    # rms of the first row is 2.5, its largest magnitude 4: q = 127 x / 4 (95.25 -> 95), scale = 4 / 2.5 / 127
    assert q[0].tolist() == [95, -127, 0, 0] and abs(float(scale[0]) - 1.6 / 127) < 1e-12
    assert q[1:].abs().sum() == 0
    assert scale[1] == 0 and torch.isnan(scale[2:]).all() and h is x
    q, scale, _ = ref.rows_i8(x[:1], norm=False)
    assert q[0].tolist() == [95, -127, 0, 0] and abs(float(scale[0]) - 4 / 127) < 1e-12
    q, scale, h = ref.rows_i8(x[:1], weight=torch.tensor([2.0, 0.5, 1.0, 1.0]), residual=torch.ones(1, 4), eps=0.0)
    assert h[0].tolist() == [4, -3, 1, 1]                       # t = 8, -1.5, 1, 1
    assert q[0].tolist() == [127, -24, 16, 16]
    assert abs(float(scale[0]) - 8 / math.sqrt(27 / 4) / 127) < 1e-12


def test_rows_ties_go_to_even():
    x = torch.tensor([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5]])
    assert ref.rows_i8(x, norm=False)[0][0].tolist() == [127, 0, 2, 2, 0, -2]


def test_matmul_by_hand():
    a = torch.tensor([[1, -2, 3]], dtype=torch.int8)
    w = torch.tensor([[4, 5, 6], [-128, 0, 127]], dtype=torch.int8)
    y, tol = ref.matmul_i8(a, torch.tensor([0.5]), w, torch.tensor([2.0, 1.0]), bias=torch.tensor([1.0, -200.0]), relu=True)
    assert y.tolist() == [[13.0, 0.0]] and (tol >= 0).all()


@pytest.mark.parametrize("top,e", [(7.0, 0), (7.0001, 1), (6.0, 0), (3.5, -1), (3.5001, 0), (1.75, -2), (2.0 ** -126, -126),
                                   (0.0, -126), (3.0e38, 125)])
def test_shared_exponent(top, e):
    x = torch.zeros(1, 32, dtype=torch.float64)
    x[0, 5] = -top
    assert ref.kv4_encode(x)[1].item() == e + 127


def test_codes_by_hand():
    x = torch.zeros(1, 32, dtype=torch.float64)
    # with 6 as the largest the exponent is 0; the ties go to the even code
    vals = [6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.26, -5.1, 4.9, 0.1]
    x[0, :12] = torch.tensor(vals, dtype=torch.float64)
    codes, exps = ref.kv4_encode(x)
    assert exps.item() == 127
    want = [6.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, -0.5, -6.0, 4.0, 0.0]
    assert ref.kv4_decode(codes, exps)[0, :12].tolist() == want
    assert codes[0, 0].item() == 7 and codes[0, 4].item() == 9 + 16 * 15   # the lower channel in the lower bits


def test_encode_is_idempotent_and_nearest():
    g = torch.Generator().manual_seed(3)
    x = torch.randn(50, 64, generator=g, dtype=torch.float64) * torch.exp2(torch.randint(-20, 20, (50, 1), generator=g).double())
    codes, exps = ref.kv4_encode(x)
    y = ref.kv4_decode(codes, exps)
    step = torch.exp2(exps.double() - 127).repeat_interleave(32, 1)
    assert ((x - y).abs() <= step).all()          # the widest half step, and what lies between 6 and 7
    again = ref.kv4_decode(*ref.kv4_encode(y))
    assert torch.equal(again, y)


def test_groups_that_are_not_finite():
    x = torch.ones(2, 64, dtype=torch.float64)
    x[0, 3], x[1, 40] = math.inf, math.nan
    codes, exps = ref.kv4_encode(x)
    assert exps.tolist() == [[255, 125], [125, 255]]   # 1 = 4 * 2^-2
    y = ref.kv4_decode(codes, exps)
    assert torch.isnan(y[0, :32]).all() and torch.equal(y[0, 32:], torch.ones(32, dtype=torch.float64))


def test_attention_by_hand():
    k = [torch.tensor([[[1.0, 0.0]], [[0.0, 1.0]], [[1.0, 1.0]]], dtype=torch.float64)]
    v = [torch.tensor([[[1.0, 0.0]], [[0.0, 1.0]], [[5.0, 5.0]]], dtype=torch.float64)]
    q = torch.tensor([[[0.0, math.log(3.0)], [0.0, 0.0]]] * 2, dtype=torch.float64)
    out, tol = ref.attention(q, k, v, [2], [3], 1.0)
    assert torch.allclose(out[0, 0], torch.tensor([0.25, 0.75], dtype=torch.float64))   # the first query sees two places
    assert torch.allclose(out[1, 1], torch.tensor([2.0, 2.0], dtype=torch.float64))     # equal scores: the mean
    assert (tol > 0).all()
    out, _ = ref.attention(q, k, v, [2], [3], 1.0, window=1)
    assert torch.allclose(out[0, 0], v[0][1, 0]) and torch.allclose(out[1, 0], v[0][2, 0])
    out, _ = ref.attention(q, [k[0][:1]], [v[0][:1]], [2], [1], 1.0)                    # more queries than places
    assert torch.equal(out[0], torch.zeros(2, 2, dtype=torch.float64)) and torch.allclose(out[1], v[0][0].expand(2, 2))
    out, _ = ref.attention(q, k, v, [2], [3], 1.0, causal=False)
    assert torch.allclose(out[0, 1], out[1, 1])
