"""GPU: a decoder in 8-bit floats that answers with tokens (paper_1907_02154_amd/decoder.py): norm, product, cache,
attention and pick run together.

Each operator's result inside a pass is held to the oracle on the exact tensors that it read, with the operator's own
bound (bit for bit where results are unique); captured steps and answers are held to the eager ones bit for bit.
"""
import pytest
import torch

from oracle import quant as ref
from oracle import sample as ref_sample
from paper_1907_02154_amd import decoder, quant

pytestmark = pytest.mark.gpu

U8 = torch.uint8


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    quant.lib()


def small(seqs=3, vocab=5003):
    dec = decoder.Decoder(blocks=2, width=256, heads=4, kv_heads=2, head_dim=64, inner=520, seed=3, float8=True, vocab=vocab)
    return dec, decoder.State(dec, seqs=seqs, max_len=150, page_size=16, seed=4)


def streams(dec, news, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(n, dec.width, generator=g, device="cuda").to(torch.bfloat16) for n in news]


def bits(t):
    return t.view(U8).cpu()


def check_rows(q, e, x, s=None, weight=None, residual=None):
    codes, byte, scale, h = ref.rows_f8(x.cpu(), None if weight is None else weight.cpu(),
                                        None if residual is None else residual.cpu())
    assert torch.equal(bits(q), codes) and torch.equal(e.cpu(), byte)
    if s is not None:   # squares in 64 lanes at least, ten additions, halved by the root; five roundings
        assert ((s.cpu().double() - scale).abs() <= ((x.shape[1] / 64 + 20) / 2 + 5) * 2.0 ** -24 * scale).all()
    return h


def check_product(y, q, e, w, s=None, residual=None, relu=False):
    cpu = lambda t: None if t is None else t.cpu()  # noqa: E731
    want, tol = ref.matmul_f8(ref.rows_f8_value(bits(q), e.cpu()), ref.rows_f8_value(bits(w.q), w.exps.cpu()), cpu(s), cpu(w.bias),
                              cpu(residual), relu)
    assert ((y.cpu().double() - want).abs() <= tol).all()


def cache_of(cache):
    return ref.KV8([bits(cache.k_codes), bits(cache.v_codes)], [cache.k_exps.cpu(), cache.v_exps.cpu()])


def check_pass(dec, state, trace, news, before):
    """`before`: each block's cache as the oracle has it; this pass's tokens are added."""
    lens, table = state.lens.tolist(), state.table.cpu()
    for b, t, want, cache in zip(dec.blocks, trace, before, state.caches):
        check_rows(t["q1"], t["e1"], t["x"], t["s1"], b.norm1)
        check_product(t["qkv"], t["q1"], t["e1"], b.wqkv, t["s1"])
        want.write(t["k"].cpu().double(), t["v"].cpu().double(), news, lens, table)
        now = cache_of(cache)
        for i in (0, 1):
            assert torch.equal(now.codes[i], want.codes[i]) and torch.equal(now.byte[i], want.byte[i])
        slots = [table[s, torch.arange(n) // 16] * 16 + torch.arange(n) % 16 for s, n in enumerate(lens)]
        out, tol = ref.attention(t["q"].cpu(), [want.values(0, s) for s in slots], [want.values(1, s) for s in slots], news, lens,
                                 dec.head_dim ** -0.5)
        assert ((t["att"].cpu().double() - out).abs() <= tol).all()
        check_rows(t["q2"], t["e2"], t["att"].flatten(1))
        check_product(t["o"], t["q2"], t["e2"], b.wo)
        h = check_rows(t["q3"], t["e3"], t["o"], t["s3"], b.norm2, t["x"])
        assert torch.equal(h, t["x1"].cpu())
        check_product(t["u"], t["q3"], t["e3"], b.w1, t["s3"], relu=True)
        check_rows(t["q4"], t["e4"], t["u"])
        check_product(t["out"], t["q4"], t["e4"], b.w2, residual=t["x1"])


def test_prompts_chunks_and_steps_against_the_oracle():
    dec, state = small()
    before = [cache_of(c) for c in state.caches]
    out = None
    for i, news in enumerate(([40, 1, 77], [5, 30, 1])):
        trace = []
        out = dec.prompt(state, streams(dec, news, 10 + i), trace)
        check_pass(dec, state, trace, news, before)
    x = torch.stack([y[-1] for y in out])
    for _ in range(2):
        trace = []
        x = dec.step(state, x, trace)
        check_pass(dec, state, trace, [1, 1, 1], before)
    assert state.lens.tolist() == [47, 33, 80] and torch.isfinite(x).all()


@pytest.mark.parametrize("float8", [False, True], ids=["int8", "float8"])
def test_answers_are_what_the_filters_leave(float8):
    """The head's logits against the oracle's product, and every token against the oracle's pick of the logits."""
    dec = decoder.Decoder(blocks=1, width=256, heads=4, kv_heads=2, head_dim=64, inner=520, seed=3, float8=float8, vocab=5003)
    state = decoder.State(dec, seqs=3, max_len=150, page_size=16, seed=4)
    x = torch.stack([y[-1] for y in dec.prompt(state, streams(dec, [30, 9, 61], 20))])
    logits = dec.logits(x)
    if float8:
        q, e, s, _ = quant.rmsnorm_f8(x, dec.norm)
        check_product(logits, q, e, dec.head, s)
    g = torch.Generator().manual_seed(5)
    for _ in range(20):
        u = torch.rand(3, generator=g)
        t, lp = dec.pick(x, u.cuda(), temperature=torch.full((3,), 0.7).cuda(), top_k=torch.full((3,), 40, dtype=torch.int32).cuda(),
                         top_p=torch.full((3,), 0.9).cuda())
        for r in range(3):
            want, wlp, _ = ref_sample.pick(logits[r].cpu().double().numpy(), float(u[r]), float(torch.tensor(0.7)), 40,
                                           float(torch.tensor(0.9)))
            assert int(t[r]) == want and abs(float(lp[r]) - wlp) <= 2.0 ** -23 * abs(wlp) + 2.0 ** -24


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


@pytest.mark.parametrize("float8", [False, True], ids=["int8", "float8"])
def test_captured_answers_are_the_eager_ones(float8):
    def made():
        dec = decoder.Decoder(blocks=2, width=256, heads=4, kv_heads=2, head_dim=64, inner=520, seed=3, float8=float8, vocab=5003)
        return dec, decoder.State(dec, seqs=3, max_len=150, page_size=16, seed=4)
    dec, state = made()
    _, twin = made()
    filters = dict(temperature=torch.tensor([0.8, 1.0, 0.0]).cuda(), top_p=torch.full((3,), 0.95).cuda())
    first = torch.tensor([5, 4000, 17], dtype=torch.int32, device="cuda")
    for st in (state, twin):
        dec.prompt(st, streams(dec, [30, 9, 61], 20))
    tokens, u = first.clone(), torch.zeros(3, device="cuda")
    graph, logprob = decoder.capture_answer(dec, state, tokens, u, **filters)
    assert torch.equal(tokens, first) and state.held == twin.held
    g = torch.Generator(device="cuda").manual_seed(6)
    eager = first
    for i in range(6):
        r = torch.rand(3, generator=g, device="cuda")
        eager, want = dec.answer(twin, eager, r, **filters)          # eager work between the replays
        u.copy_(r)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(tokens, eager) and torch.equal(logprob, want), i
    assert state.lens.tolist() == twin.lens.tolist() == [36, 15, 67] and float(want[2]) == 0


def test_a_capture_leaves_the_cache_as_it_was():
    """Of a token far larger than those that follow: its block's exponent must not have seen it."""
    dec, state = small()
    _, twin = small()
    for st in (state, twin):
        out = dec.prompt(st, streams(dec, [30, 9, 61], 22))
    x = torch.stack([y[-1] for y in out])
    for b in dec.blocks:
        b.norm1 = b.norm1 * 300                       # keys and values of the captured step
    y = x.clone()
    before = [bits(t).clone() for c in state.caches for t in (c.k_codes, c.v_codes, c.k_exps, c.v_exps)]
    graph, got = decoder.capture_step(dec, state, y)
    decoder.capture_answer(dec, state, torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(3, device="cuda"))
    torch.cuda.synchronize()
    after = [bits(t) for c in state.caches for t in (c.k_codes, c.v_codes, c.k_exps, c.v_exps)]
    assert all(torch.equal(p, q) for p, q in zip(before, after)) and state.lens.tolist() == twin.lens.tolist()
    for i in range(3):
        want = dec.step(twin, x)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want), i
        x = want
        y.copy_(got)


def test_a_captured_answer_keeps_what_it_reads():
    """Filters that nothing else refers to, whose memory would go to the tensors made after the capture."""
    dec, state = small()
    _, twin = small()
    for st in (state, twin):
        dec.prompt(st, streams(dec, [30, 9, 61], 23))
    tokens = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda")
    eager = tokens.clone()
    u = torch.full((3,), 0.999, device="cuda")
    graph, _ = decoder.capture_answer(dec, state, tokens, u, temperature=torch.zeros(3, device="cuda"))
    other = [torch.full((3,), 50.0, device="cuda") for _ in range(200)]
    for i in range(4):
        eager, _ = dec.answer(twin, eager, u, temperature=torch.zeros(3, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(tokens, eager) and len(other) == 200, i


def test_two_captured_answers_of_one_state_take_turns():
    """Two graphs with workspaces and outputs of their own, replayed in turn on one state, against eager answers."""
    dec, state = small()
    _, twin = small()
    for st in (state, twin):
        dec.prompt(st, streams(dec, [30, 9, 61], 21))
    tokens, u = torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda"), torch.rand(3, device="cuda")
    eager = tokens.clone()
    graphs = [decoder.capture_answer(dec, state, tokens, u, **f)[0] for f in (dict(), dict(temperature=torch.zeros(3, device="cuda")))]
    for i in range(6):
        u.copy_(torch.rand(3, device="cuda"))
        torch.cuda.synchronize()
        eager, _ = dec.answer(twin, eager, u, **(dict(temperature=torch.zeros(3, device="cuda")) if i % 2 else dict()))
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(tokens, eager), i


def test_no_room_and_no_vocabulary():
    dec, state = small()
    dec.prompt(state, streams(dec, [149, 5, 150], 30))
    t, u = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(3, device="cuda")
    with pytest.raises(ValueError, match="no room"):
        dec.answer(state, t, u)
    for bad in ((t[:2], u), (t.long(), u), (t, u[:1])):
        with pytest.raises(ValueError):
            dec.answer(state, *bad)
    for capture in (lambda: decoder.capture_answer(dec, state, t, u), lambda: decoder.capture_step(dec, state, dec.embed(t))):
        with pytest.raises(ValueError, match="no room"):
            capture()
    assert state.held == [149, 5, 150] == state.lens.tolist()
    plain = decoder.Decoder(blocks=1, width=256, heads=4, kv_heads=2, head_dim=64, inner=520)
    for f in (lambda: plain.embed(t), lambda: plain.logits(torch.zeros(1, 256)), lambda: plain.answer(state, t, u)):
        with pytest.raises(ValueError, match="vocabulary"):
            f()


@pytest.mark.parametrize("float8", [False, True], ids=["int8", "float8"])
def test_a_refused_call_leaves_the_state(float8):
    """Shapes, types, devices, filters and states that do not fit: lengths and every byte of the caches stay, and the call
    that follows gives what it gives without them."""
    def made():
        dec = decoder.Decoder(blocks=2, width=256, heads=4, kv_heads=2, head_dim=64, inner=520, seed=3, float8=float8, vocab=5003)
        return dec, decoder.State(dec, seqs=3, max_len=150, page_size=16, seed=4)
    dec, state = made()
    _, twin = made()
    for st in (state, twin):
        out = dec.prompt(st, streams(dec, [30, 9, 61], 24))
    x = torch.stack([y[-1] for y in out])
    t, u = torch.tensor([5, 4000, 17], dtype=torch.int32, device="cuda"), torch.full((3,), 0.4, device="cuda")
    ones, k = torch.ones(3, device="cuda"), torch.ones(3, dtype=torch.int32, device="cuda")
    other = decoder.Decoder(blocks=1, width=256, heads=4, kv_heads=2, head_dim=64, inner=520, float8=float8, vocab=50)
    kind = decoder.Decoder(blocks=2, width=256, heads=4, kv_heads=2, head_dim=64, inner=520, float8=not float8, vocab=50)
    bad = [lambda f=f: dec.answer(state, t, u, **f) for f in (
        dict(top_p=0.9), dict(top_p=ones[:2]), dict(top_p=ones.double()), dict(temperature=ones.cpu()), dict(temperature=k),
        dict(top_k=ones), dict(top_k=k.long()), dict(min_p=ones[:2]), dict(top_q=ones), dict(stream=0), dict(out=ones),
        dict(out=k[:1]), dict(logprob=k), dict(logprob=ones.cpu()))]
    bad += [lambda f=f: decoder.capture_answer(dec, state, t, u, **f) for f in (dict(top_p=0.9), dict(top_k=ones))]
    bad += [lambda: dec.answer(state, t, u.double()), lambda: dec.answer(state, t, u.cpu()), lambda: dec.step(state, x.cpu()),
            lambda: dec.step(state, x.t().contiguous().t()), lambda: dec.prompt(state, [x.cpu()] * 3),
            lambda: dec.prompt(state, [x, x.cpu(), x]), lambda: other.step(state, x), lambda: kind.step(state, x),
            lambda: kind.answer(state, t, u), lambda: kind.prompt(state, [x] * 3)]
    held = lambda: [bits(c) for cache in state.caches for c in (cache.k_codes, cache.v_codes, cache.k_exps, cache.v_exps)]  # noqa: E731
    before = held()
    for i, f in enumerate(bad):
        with pytest.raises((ValueError, TypeError)):
            f()
        assert state.held == state.lens.tolist() == [30, 9, 61], i
        assert all(torch.equal(p, q) for p, q in zip(before, held())), i
    got, want = (dec.answer(st, t, u, temperature=ones, top_k=k * 40, top_p=0.9 * ones, out=k.clone(), logprob=ones.clone())
                 for st in (state, twin))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and state.lens.tolist() == [31, 10, 62]
    assert torch.equal(dec.step(state, x), dec.step(twin, x))


def test_the_8_bit_form_asks_for_no_slots(monkeypatch):
    """Its cache takes the page table: what the 4-bit cache's slots take would be launches for nothing."""
    dec, state = small()
    monkeypatch.setattr(decoder.State, "slots", None)
    out = dec.prompt(state, streams(dec, [30, 9, 61], 25))
    dec.step(state, torch.stack([y[-1] for y in out]))
    assert state.lens.tolist() == [31, 10, 62]
