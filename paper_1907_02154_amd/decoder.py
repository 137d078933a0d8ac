"""A decoder of transformer blocks served in few bits: the operators of ``quant`` as a program uses them.

A block keeps its residual stream in bf16 and everything that is multiplied in 8 bits:

    q, s    = rows of rmsnorm(x) in 8 bits
    qkv     = q wqkv, scaled                                  keys and values of the new tokens into the 4-bit cache
    o       = attention of the queries over the cache         its rows in 8 bits
    x, q, s = x + o wo, and the rows of its rmsnorm in 8 bits (one kernel)
    x       = x + relu(q w1 + b1) w2 + b2                     the rows between in 8 bits

or, with ``float8``, in 8-bit floats whose blocks share a power of two, and an 8-bit cache:

    q, e, s = rmsnorm(x) in blocks of 128 and, apart, the norm's factor of each row
    qkv     = s (q wqkv)                                      keys and values into the 8-bit cache, blocks of tokens
    o       = attention over it, in blocks; and so on

With a vocabulary it answers with tokens: logits = the last rmsnorm's rows times the head's weights, from which
``pick`` draws with temperature, top-k, top-p and min-p by random numbers that the caller gives.

Weights are synthetic (seeded, He-normal); they are quantised once, a scale for each output channel or an exponent for
each 128 of its weights, by the same operator that quantises activations.  The order of tokens enters through the causal
mask alone.  A step of single tokens reads and writes only tensors that the ``State`` keeps, so it can be captured into a
HIP graph and replayed.

    python -m paper_1907_02154_amd.decoder        # prompts, then steps as a graph: tokens a second of each
"""
from __future__ import annotations

import math
import time
from typing import List, Optional

import torch

from . import quant, sample


class Weights:
    """An output channel's weights in a row of 8-bit integers, with a scale for each."""

    def __init__(self, w: torch.Tensor, bias: Optional[torch.Tensor] = None):
        self.q, self.scale = quant.rows_i8(w)
        self.bias = bias

    def __call__(self, q, scale, **k):
        return quant.matmul_i8(q, scale, self.q, self.scale, bias=self.bias, **k)


class Weights8:
    """An output channel's weights in a row of 8-bit floats, with an exponent for each 128."""

    def __init__(self, w: torch.Tensor, bias: Optional[torch.Tensor] = None):
        self.q, self.exps = quant.rows_f8(w)
        self.bias = bias

    def __call__(self, q, exps, scale=None, **k):
        return quant.matmul_f8(q, exps, self.q, self.exps, a_scale=scale, bias=self.bias, **k)


class State:
    """What `seqs` sequences of up to `max_len` tokens keep between calls: their pages in each block's cache, and their
    lengths, on the device (`lens`) and on the host (`held`: what a call is checked against before it launches anything)."""

    def __init__(self, dec: "Decoder", seqs: int, max_len: int, page_size: int = 64, seed: int = 0):
        if seqs < 1 or max_len < 1 or page_size < 1:
            raise ValueError("a state holds one sequence of one token at least, in pages of one at least")
        pages = -(-max_len // page_size)
        g = torch.Generator().manual_seed(seed)      # pages in no order, as a server that reuses them has them
        table = torch.randperm(seqs * pages, generator=g).reshape(seqs, pages).to(torch.int32)
        self.table = table.cuda()
        self.slot = None if dec.float8 else self.slots_of(table, max_len, page_size).cuda()   # the 8-bit cache takes the table
        cache = quant.KV8Cache if dec.float8 else quant.KV4Cache
        self.caches = [cache.allocate(seqs * pages, dec.kv_heads, page_size, dec.head_dim) for _ in dec.blocks]
        self.lens = torch.zeros(seqs, dtype=torch.int32, device="cuda")
        self.held = [0] * seqs
        self.max_len, self.page_size = max_len, page_size

    def room(self, news: List[int]) -> List[int]:
        """How many tokens each sequence s holds with news[s] more, if all have room for theirs."""
        if len(news) != len(self.held):
            raise ValueError(f"the state has {len(self.held)} sequences, got tokens of {len(news)}")
        after = [h + n for h, n in zip(self.held, news)]
        if max(after) > self.max_len:
            s = after.index(max(after))
            raise ValueError(f"sequence {s} holds {self.held[s]} tokens of {self.max_len} at most: no room for {news[s]} more")
        return after

    def take(self, news: List[int]) -> None:
        """Counts news[s] more tokens of each sequence s, if all have room for theirs."""
        self.held = self.room(news)

    @staticmethod
    def slots_of(table: torch.Tensor, max_len: int, page_size: int) -> torch.Tensor:
        """The slot of every place of each sequence, and -1, which is not written, behind the last one."""
        place = torch.arange(max_len)
        slot = table.long()[:, place // page_size] * page_size + place % page_size
        return torch.nn.functional.pad(slot, (0, 1), value=-1).to(torch.int32)

    def slots(self, seq: torch.Tensor, place: torch.Tensor) -> torch.Tensor:
        """Cache slots of the tokens at `place` of sequences `seq`; -1 past max_len."""
        return self.slot[seq, place.clamp(max=self.max_len)]


class Block:
    def __init__(self, dec: "Decoder", g: torch.Generator):
        width, inner = dec.width, dec.inner
        qkv = (dec.heads + 2 * dec.kv_heads) * dec.head_dim

        def make(n, k, bias=False):
            w = torch.randn(n, k, generator=g, device="cuda") * math.sqrt(2.0 / k)
            return dec.weights(w, 0.01 * torch.randn(n, generator=g, device="cuda") if bias else None)

        self.norm1 = 0.5 + torch.rand(width, generator=g, device="cuda")
        self.norm2 = 0.5 + torch.rand(width, generator=g, device="cuda")
        self.wqkv, self.wo = make(qkv, width), make(width, dec.heads * dec.head_dim)
        self.w1, self.w2 = make(inner, width, True), make(width, inner, True)


class Decoder:
    """`blocks` blocks on a residual stream of `width` channels: `heads` query heads on `kv_heads` key heads of
    `head_dim` channels, and a ReLU layer of `inner` channels.  float8: in 8-bit floats with an 8-bit cache, in place of
    8-bit integers with a 4-bit one.  vocab > 0: tokens have an embedding, and logits."""

    def __init__(self, blocks: int = 2, width: int = 1024, heads: int = 16, kv_heads: int = 4, head_dim: int = 64,
                 inner: int = 4096, seed: int = 0, float8: bool = False, vocab: int = 0):
        self.width, self.heads, self.kv_heads, self.head_dim, self.inner = width, heads, kv_heads, head_dim, inner
        self.float8, self.vocab = float8, vocab
        self.weights = Weights8 if float8 else Weights
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.blocks: List[Block] = [Block(self, g) for _ in range(blocks)]
        if vocab:
            self.embedding = torch.randn(vocab, width, generator=g, device="cuda").to(torch.bfloat16)
            self.norm = 0.5 + torch.rand(width, generator=g, device="cuda")
            self.head = self.weights(torch.randn(vocab, width, generator=g, device="cuda") * math.sqrt(2.0 / width))

    def _block(self, b: Block, cache, x, slots, table, lens, starts, max_new, max_len, trace=None):
        if self.float8:
            return self._block8(b, cache, x, table, lens, starts, max_new, max_len, trace)
        h, kv, d = self.heads, self.kv_heads, self.head_dim
        q1, s1, _ = quant.rmsnorm_i8(x, b.norm1)
        qkv = b.wqkv(q1, s1)
        q, k, v = (t.unflatten(1, (-1, d)) for t in qkv.split((h * d, kv * d, kv * d), 1))
        quant.kv4_write(k, v, slots, cache)
        att = quant.attention_kv4(q, cache, table, lens, starts=starts, max_new=max_new, max_len=max_len)
        q2, s2 = quant.rows_i8(att.flatten(1))
        o = b.wo(q2, s2)
        q3, s3, x1 = quant.rmsnorm_i8(o, b.norm2, residual=x)
        u = b.w1(q3, s3, relu=True)
        q4, s4 = quant.rows_i8(u)
        out = b.w2(q4, s4, residual=x1)
        if trace is not None:
            trace.append(dict(x=x, q1=q1, s1=s1, qkv=qkv, q=q, k=k, v=v, att=att, q2=q2, s2=s2, o=o, x1=x1, q3=q3, s3=s3,
                              u=u, q4=q4, s4=s4, out=out))
        return out

    def _block8(self, b: Block, cache, x, table, lens, starts, max_new, max_len, trace=None):
        h, kv, d = self.heads, self.kv_heads, self.head_dim
        q1, e1, s1, _ = quant.rmsnorm_f8(x, b.norm1)
        qkv = b.wqkv(q1, e1, s1)
        q, k, v = (t.unflatten(1, (-1, d)) for t in qkv.split((h * d, kv * d, kv * d), 1))
        quant.kv8_write(k, v, cache, table, lens, starts=starts, max_new=max_new)
        att = quant.attention_kv8(q, cache, table, lens, starts=starts, max_new=max_new, max_len=max_len)
        q2, e2 = quant.rows_f8(att.flatten(1))
        o = b.wo(q2, e2)
        q3, e3, s3, x1 = quant.rmsnorm_f8(o, b.norm2, residual=x)
        u = b.w1(q3, e3, s3, relu=True)
        q4, e4 = quant.rows_f8(u)
        out = b.w2(q4, e4, residual=x1)
        if trace is not None:
            trace.append(dict(x=x, q1=q1, e1=e1, s1=s1, qkv=qkv, q=q, k=k, v=v, att=att, q2=q2, e2=e2, o=o, x1=x1, q3=q3,
                              e3=e3, s3=s3, u=u, q4=q4, e4=e4, out=out))
        return out

    def _tokens(self) -> None:
        if not self.vocab:
            raise ValueError("the decoder has no vocabulary")

    def _device(self, state: State, t: torch.Tensor, name: str) -> int:
        """The device of a pass over a state, where t has to be, with caches as the decoder's blocks have them."""
        dev = quant._here(t, name)
        if state.lens.get_device() != dev:
            raise ValueError(f"the state is on device {state.lens.get_device()}, {name} is on device {dev}")
        cache = quant.KV8Cache if self.float8 else quant.KV4Cache
        if len(state.caches) != len(self.blocks) or any(
                not isinstance(c, cache) or c.heads != self.kv_heads or c.head_dim != self.head_dim for c in state.caches):
            raise ValueError("the state is of another decoder")
        return dev

    def embed(self, tokens: torch.Tensor) -> torch.Tensor:
        """The stream of tokens int32 [tokens], bf16 [tokens][width]; of -1 (no token was drawn) token 0's."""
        self._tokens()
        return self.embedding[tokens.clamp(0, self.vocab - 1)]

    def logits(self, x: torch.Tensor) -> torch.Tensor:
        """bf16 [tokens][vocab] of the stream x after the last block."""
        self._tokens()
        if self.float8:
            q, e, s, _ = quant.rmsnorm_f8(x, self.norm)
            return self.head(q, e, s)
        q, s, _ = quant.rmsnorm_i8(x, self.norm)
        return self.head(q, s)

    def pick(self, x: torch.Tensor, u: torch.Tensor, temperature=None, top_k=None, top_p=None, min_p=None, out=None,
             logprob=None, ws=None):
        """(tokens, logprob) drawn for the stream x after the last block by u, as ``sample.tokens`` has it; on the current
        stream, as the logits are."""
        return sample.tokens(self.logits(x), u, temperature, top_k, top_p, min_p, out=out, logprob=logprob, ws=ws)

    def prompt(self, state: State, xs: List[torch.Tensor], trace=None) -> List[torch.Tensor]:
        """New tokens of every sequence, xs[s] bf16 [tokens][width] behind what the sequence holds: the stream after the
        last block, a tensor for each sequence.  What is refused for want of room, or for a shape, type or device, leaves
        the state as it was."""
        if any(x.dim() != 2 or x.shape[1] != self.width or x.dtype != torch.bfloat16 for x in xs):
            raise ValueError(f"tokens must be bf16 [tokens][{self.width}]")
        news = [x.shape[0] for x in xs]
        after = state.room(news)
        if not any(news):
            return list(xs)
        dev = self._device(state, xs[0], "a sequence's tokens")
        for x in xs:
            quant._tensor(x, "a sequence's tokens", dev, torch.bfloat16)
        state.held = after
        starts = torch.tensor([0, *torch.tensor(news).cumsum(0).tolist()], dtype=torch.int32).cuda()
        slots = None
        if not self.float8:
            seq = torch.repeat_interleave(torch.arange(len(xs)), torch.tensor(news)).cuda()
            slots = state.slots(seq, torch.arange(sum(news), device="cuda") - starts[seq] + state.lens[seq])
        state.lens += (starts[1:] - starts[:-1])
        x = torch.cat(xs)
        for b, cache in zip(self.blocks, state.caches):
            x = self._block(b, cache, x, slots, state.table, state.lens, starts, max(news), state.max_len, trace)
        return list(x.split(news))

    def step(self, state: State, x: torch.Tensor, trace=None) -> torch.Tensor:
        """One new token of every sequence, x bf16 [seqs][width]: the stream after the last block.  What is refused leaves
        the state as it was, as of ``prompt``."""
        if x.dim() != 2 or x.shape[1] != self.width or x.dtype != torch.bfloat16:
            raise ValueError(f"tokens must be bf16 [sequences][{self.width}]")
        after = state.room([1] * x.shape[0])
        quant._matrix(x, "x", self._device(state, x, "x"), None, None, torch.bfloat16)
        state.held = after
        return self._step(state, x, trace)

    def _step(self, state: State, x: torch.Tensor, trace=None) -> torch.Tensor:
        slots = None if self.float8 else state.slots(torch.arange(x.shape[0], device="cuda"), state.lens)
        state.lens += 1
        for b, cache in zip(self.blocks, state.caches):
            x = self._block(b, cache, x, slots, state.table, state.lens, None, 1, state.max_len, trace)
        return x

    def answer(self, state: State, tokens: torch.Tensor, u: torch.Tensor, **filters):
        """One step on a token of every sequence, tokens int32 [seqs]: the (tokens, logprob) drawn to follow them, as
        ``pick`` has it.  What is refused leaves the state as it was, as of ``prompt``."""
        self._tokens()
        if tokens.shape != (len(state.held),) or tokens.dtype != torch.int32 or u.shape != tokens.shape:
            raise ValueError(f"there are {len(state.held)} sequences: one int32 token and one random number for each")
        after = state.room([1] * len(state.held))
        sample._operands(self._device(state, u, "u"), len(state.held), u, **filters)
        x = self.embed(tokens)
        state.held = after
        return self.pick(self._step(state, x), u, **filters)


class Steps:
    """A captured step: each replay takes the sequences of its state one token further.  It keeps what a replay reads."""

    def __init__(self, state: State, graph: "torch.cuda.CUDAGraph", reads=()):
        self.state, self.graph, self.reads = state, graph, reads

    def replay(self) -> None:
        """A ValueError, and nothing done, where a sequence has no room for a token more."""
        self.state.take([1] * len(self.state.held))
        self.graph.replay()


def _capture(state: State, reads, once, again):
    """`again` as a HIP graph, after `once` outside it, for kernels are loaded on their first launch.  The state stays as it
    was: `once` finds the pages full, so that its tokens, which might raise an exponent of the cache, are not written."""
    lens, held = state.lens.clone(), state.held
    state.lens.fill_(state.table.shape[1] * state.page_size)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    try:
        with torch.cuda.stream(side):
            once()
    finally:
        torch.cuda.current_stream().wait_stream(side)
        state.lens.copy_(lens)
        state.held = held
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = again()
    return Steps(state, graph, reads), out


def capture_step(dec: Decoder, state: State, x: torch.Tensor):
    """A step on the tensor x as a HIP graph: (``Steps`` to replay, its output)."""
    return _capture(state, (dec, x), lambda: dec.step(state, x), lambda: dec._step(state, x))


def capture_answer(dec: Decoder, state: State, tokens: torch.Tensor, u: torch.Tensor, **filters):
    """An answer to the tensor of tokens as a HIP graph: (``Steps`` to replay, logprob).  A replay puts the tokens drawn by
    u in the place of those that it read, for the next one, whose u the caller fills in before."""
    quant._vector(tokens, "tokens", quant._here(tokens, "tokens"), len(state.held), torch.int32)   # replays write it

    def again():
        drawn, logprob = dec.pick(dec._step(state, dec.embed(tokens)), u, **filters)
        tokens.copy_(drawn)
        return logprob
    return _capture(state, (dec, tokens, u, filters), lambda: dec.answer(state, tokens, u, **filters), again)


def main(seqs: int = 16, prompt: int = 1000, steps: int = 64) -> None:
    for float8 in (False, True):
        print("8-bit floats, 8-bit cache" if float8 else "8-bit integers, 4-bit cache")
        run(float8, seqs, prompt, steps)


def run(float8: bool, seqs: int, prompt: int, steps: int) -> None:
    dec = Decoder(blocks=4, width=2048, heads=16, kv_heads=4, head_dim=128, inner=8192, float8=float8, vocab=32000)
    state = State(dec, seqs, prompt + 2 * steps + 1)
    g = torch.Generator(device="cuda").manual_seed(1)
    xs = [torch.randn(prompt, dec.width, generator=g, device="cuda").to(torch.bfloat16) for _ in range(seqs)]
    dec.prompt(State(dec, seqs, prompt), xs)
    torch.cuda.synchronize()
    t = time.perf_counter()
    last = torch.stack([y[-1] for y in dec.prompt(state, xs)])
    torch.cuda.synchronize()
    t = time.perf_counter() - t
    print(f"prompts: {seqs} of {prompt} tokens in {t * 1e3:.2f} ms, {seqs * prompt / t:.0f} tokens/s")
    u = torch.rand(seqs, generator=g, device="cuda")
    filters = dict(temperature=torch.full_like(u, 0.8), top_p=torch.full_like(u, 0.95))
    tokens, _ = dec.pick(last, u, **filters)
    graph, out = capture_step(dec, state, last)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(steps):
        graph.replay()
        last.copy_(out)
    torch.cuda.synchronize()
    t = time.perf_counter() - t
    held = sum(c.nbytes() for c in state.caches)
    bf16 = sum(c.k_codes.numel() for c in state.caches) * (1 if float8 else 2) * 4
    print(f"steps: {steps} of {seqs} sequences in {t * 1e3:.2f} ms, {seqs * steps / t:.0f} tokens/s; "
          f"cache {held / 1e6:.1f} MB (bf16: {bf16 / 1e6:.1f})")
    graph, _ = capture_answer(dec, state, tokens, u, **filters)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(steps):
        graph.replay()
        u.uniform_(generator=g)
    torch.cuda.synchronize()
    t = time.perf_counter() - t
    print(f"answers: {steps} tokens for {seqs} sequences, {dec.vocab} to choose from, in {t * 1e3:.2f} ms, "
          f"{seqs * steps / t:.0f} tokens/s")


if __name__ == "__main__":
    main()
