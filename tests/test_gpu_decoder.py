"""GPU: a decoder of quantised blocks (paper_1907_02154_amd/decoder.py), the operators of ``quant`` run together.

Each operator's result inside a pass is held to the oracle on the exact tensors that it read, with the operator's own
bound (bit for bit where results are unique); a captured step is held to the eager one bit for bit.
"""
import pytest
import torch

from oracle import quant as ref
from paper_1907_02154_amd import decoder, quant

pytestmark = pytest.mark.gpu

SCALE_TOL = (74 / 2 + 4) * 2.0 ** -24   # of a row's scale: 74 additions, halved by the root, and four roundings


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    quant.lib()


def small():
    dec = decoder.Decoder(blocks=2, width=256, heads=4, kv_heads=2, head_dim=64, inner=520, seed=3)
    return dec, decoder.State(dec, seqs=3, max_len=150, page_size=16, seed=4)


def streams(dec, news, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(n, dec.width, generator=g, device="cuda").to(torch.bfloat16) for n in news]


def check_rows(q, s, x, weight=None, residual=None, norm=True):
    wq, ws, h = ref.rows_i8(x.cpu(), None if weight is None else weight.cpu(), None if residual is None else residual.cpu(),
                            1e-6, norm)
    assert torch.equal(q.cpu(), wq)
    assert ((s.cpu().double() - ws).abs() <= SCALE_TOL * ws.abs()).all()
    return h


def check_product(y, q, s, w, residual=None, relu=False):
    want, tol = ref.matmul_i8(q.cpu(), s.cpu(), w.q.cpu(), w.scale.cpu(), None if w.bias is None else w.bias.cpu(),
                              None if residual is None else residual.cpu(), relu)
    assert ((y.cpu().double() - want).abs() <= tol).all()


def check_pass(dec, state, trace, news, held):
    """`held`: the keys and values, by block and sequence, that the oracle's cache holds so far; this pass's are added."""
    lens = state.lens.tolist()
    for b, t, kv in zip(dec.blocks, trace, held):
        check_rows(t["q1"], t["s1"], t["x"], b.norm1)
        check_product(t["qkv"], t["q1"], t["s1"], b.wqkv)
        at = 0
        for s, n in enumerate(news):
            for i, name in enumerate("kv"):
                kv[s][i] = torch.cat([kv[s][i], ref.kv4_decode(*ref.kv4_encode(t[name][at:at + n].cpu()))])
            assert kv[s][0].shape[0] == lens[s]
            at += n
        want, tol = ref.attention(t["q"].cpu(), [x[0] for x in kv], [x[1] for x in kv], news, lens, dec.head_dim ** -0.5)
        assert ((t["att"].cpu().double() - want).abs() <= tol).all()
        check_rows(t["q2"], t["s2"], t["att"].flatten(1), norm=False)
        check_product(t["o"], t["q2"], t["s2"], b.wo)
        h = check_rows(t["q3"], t["s3"], t["o"], b.norm2, t["x"])
        assert torch.equal(h, t["x1"].cpu())
        check_product(t["u"], t["q3"], t["s3"], b.w1, relu=True)
        check_rows(t["q4"], t["s4"], t["u"], norm=False)
        check_product(t["out"], t["q4"], t["s4"], b.w2, residual=t["x1"])


def test_prompts_chunks_and_steps_against_the_oracle():
    dec, state = small()
    held = [[[torch.zeros(0, 2, 64, dtype=torch.float64) for _ in "kv"] for _ in range(3)] for _ in dec.blocks]
    out = None
    for i, news in enumerate(([40, 1, 77], [5, 30, 1])):
        trace = []
        out = dec.prompt(state, streams(dec, news, 10 + i), trace)
        check_pass(dec, state, trace, news, held)
    x = torch.stack([y[-1] for y in out])
    for _ in range(2):
        trace = []
        x = dec.step(state, x, trace)
        check_pass(dec, state, trace, [1, 1, 1], held)
    assert state.lens.tolist() == [47, 33, 80] and torch.isfinite(x).all()


def test_captured_steps_are_the_eager_ones():
    dec, state = small()
    _, twin = small()
    for st in (state, twin):
        out = dec.prompt(st, streams(dec, [30, 9, 61], 20))
    x = torch.stack([y[-1] for y in out])
    y = x.clone()
    graph, got = decoder.capture_step(dec, state, y)
    for i in range(5):
        want = dec.step(twin, x)                     # eager work between the replays
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want), i
        x = want
        y.copy_(got)
    assert state.lens.tolist() == twin.lens.tolist() == [35, 14, 66]


def test_weights_hold_a_scale_for_each_channel():
    g = torch.Generator().manual_seed(1)
    w = torch.randn(7, 100, generator=g) * torch.logspace(-3, 3, 7)[:, None]
    got = decoder.Weights(w.cuda())
    off = (got.q.cpu().float() * got.scale.cpu()[:, None] - w).abs()
    assert (off <= 0.5001 * got.scale.cpu()[:, None]).all()      # half a step of the channel's own


def test_sequences_up_to_their_last_place_and_past_it():
    """A state whose last page has room past max_len: the last token against the oracle, the next one refused, and a replay
    that goes round the refusal writes no cache."""
    dec, state = small()                             # 150 tokens of at most, pages of 16: 160 places
    held = [[[torch.zeros(0, 2, 64, dtype=torch.float64) for _ in "kv"] for _ in range(3)] for _ in dec.blocks]
    trace = []
    out = dec.prompt(state, streams(dec, [148, 140, 3], 30), trace)
    check_pass(dec, state, trace, [148, 140, 3], held)
    x = torch.stack([y[-1] for y in out])
    steps, got = decoder.capture_step(dec, state, x)
    for _ in range(2):
        steps.replay()
    torch.cuda.synchronize()
    assert state.lens.tolist() == state.held == [150, 142, 5]
    kept = [t.clone() for c in state.caches for t in (c.k_codes, c.k_exps, c.v_codes, c.v_exps)]
    for f in (steps.replay, lambda: dec.step(state, x), lambda: decoder.capture_step(dec, state, x),
              lambda: dec.prompt(state, streams(dec, [1, 0, 0], 31)), lambda: dec.prompt(state, streams(dec, [0, 9, 0], 31))):
        with pytest.raises(ValueError, match="no room"):
            f()
    assert state.lens.tolist() == state.held == [150, 142, 5]
    dec.prompt(state, streams(dec, [0, 8, 0], 32))
    for _ in range(12):
        steps.graph.replay()                         # past 150, and for the first sequence past its pages
    torch.cuda.synchronize()
    assert state.lens.tolist() == [162, 162, 17]
    pages = state.table[:2].flatten().long()         # of the full sequences: only what the prompt wrote has changed
    wrote = state.slots(torch.ones(8, dtype=torch.long, device="cuda"), torch.arange(142, 150, device="cuda")).long()
    for old, new in zip(kept, [t for c in state.caches for t in (c.k_codes, c.k_exps, c.v_codes, c.v_exps)]):
        same = (old == new).all(-1).all(1)           # [pages][place]
        same[wrote // 16, wrote % 16] = True
        assert same[pages].all()
