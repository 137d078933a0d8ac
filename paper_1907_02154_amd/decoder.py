"""A decoder of transformer blocks served in few bits: the operators of ``quant`` as a program uses them.

A block keeps its residual stream in bf16 and everything that is multiplied in 8 bits:

    q, s    = rows of rmsnorm(x) in 8 bits
    qkv     = q wqkv, scaled                                  keys and values of the new tokens into the 4-bit cache
    o       = attention of the queries over the cache         its rows in 8 bits
    x, q, s = x + o wo, and the rows of its rmsnorm in 8 bits (one kernel)
    x       = x + relu(q w1 + b1) w2 + b2                     the rows between in 8 bits

Weights are synthetic (seeded, He-normal); they are quantised once, a scale for each output channel, by the same
operator that quantises activations.  The order of tokens enters through the causal mask alone.  A step of single
tokens reads and writes only tensors that the ``State`` keeps, so it can be captured into a HIP graph and replayed.

    python -m paper_1907_02154_amd.decoder        # prompts, then steps as a graph: tokens a second of each
"""
from __future__ import annotations

import math
import time
from typing import List, Optional

import torch

from . import quant


class Weights:
    """An output channel's weights in a row of 8-bit integers, with a scale for each."""

    def __init__(self, w: torch.Tensor, bias: Optional[torch.Tensor] = None):
        self.q, self.scale = quant.rows_i8(w)
        self.bias = bias

    def __call__(self, q, scale, **k):
        return quant.matmul_i8(q, scale, self.q, self.scale, bias=self.bias, **k)


class State:
    """What `seqs` sequences of up to `max_len` tokens keep between calls: their pages in each block's cache, and their
    lengths, on the device (`lens`) and on the host (`held`: what a call is checked against before it launches anything)."""

    def __init__(self, dec: "Decoder", seqs: int, max_len: int, page_size: int = 64, seed: int = 0):
        if seqs < 1 or max_len < 1 or page_size < 1:
            raise ValueError("a state holds one sequence of one token at least, in pages of one at least")
        pages = -(-max_len // page_size)
        g = torch.Generator().manual_seed(seed)      # pages in no order, as a server that reuses them has them
        table = torch.randperm(seqs * pages, generator=g).reshape(seqs, pages).to(torch.int32)
        self.table, self.slot = table.cuda(), self.slots_of(table, max_len, page_size).cuda()
        self.caches = [quant.KV4Cache.allocate(seqs * pages, dec.kv_heads, page_size, dec.head_dim) for _ in dec.blocks]
        self.lens = torch.zeros(seqs, dtype=torch.int32, device="cuda")
        self.held = [0] * seqs
        self.max_len, self.page_size = max_len, page_size

    def take(self, news: List[int]) -> None:
        """Counts news[s] more tokens of each sequence s, if all have room for theirs."""
        if len(news) != len(self.held):
            raise ValueError(f"the state has {len(self.held)} sequences, got tokens of {len(news)}")
        after = [h + n for h, n in zip(self.held, news)]
        if max(after) > self.max_len:
            s = after.index(max(after))
            raise ValueError(f"sequence {s} holds {self.held[s]} tokens of {self.max_len} at most: no room for {news[s]} more")
        self.held = after

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
            return Weights(w, 0.01 * torch.randn(n, generator=g, device="cuda") if bias else None)

        self.norm1 = 0.5 + torch.rand(width, generator=g, device="cuda")
        self.norm2 = 0.5 + torch.rand(width, generator=g, device="cuda")
        self.wqkv, self.wo = make(qkv, width), make(width, dec.heads * dec.head_dim)
        self.w1, self.w2 = make(inner, width, True), make(width, inner, True)


class Decoder:
    """`blocks` blocks on a residual stream of `width` channels: `heads` query heads on `kv_heads` key heads of
    `head_dim` channels, and a ReLU layer of `inner` channels."""

    def __init__(self, blocks: int = 2, width: int = 1024, heads: int = 16, kv_heads: int = 4, head_dim: int = 64,
                 inner: int = 4096, seed: int = 0):
        self.width, self.heads, self.kv_heads, self.head_dim, self.inner = width, heads, kv_heads, head_dim, inner
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.blocks: List[Block] = [Block(self, g) for _ in range(blocks)]

    def _block(self, b: Block, cache, x, slots, table, lens, starts, max_new, max_len, trace=None):
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

    def prompt(self, state: State, xs: List[torch.Tensor], trace=None) -> List[torch.Tensor]:
        """New tokens of every sequence, xs[s] bf16 [tokens][width] behind what the sequence holds: the stream after the
        last block, a tensor for each sequence.  A ValueError, and nothing done, where a sequence has no room for its own."""
        if any(x.dim() != 2 or x.shape[1] != self.width or x.dtype != torch.bfloat16 for x in xs):
            raise ValueError(f"tokens must be bf16 [tokens][{self.width}]")
        news = [x.shape[0] for x in xs]
        state.take(news)
        if not any(news):
            return list(xs)
        starts = torch.tensor([0, *torch.tensor(news).cumsum(0).tolist()], dtype=torch.int32).cuda()
        seq = torch.repeat_interleave(torch.arange(len(xs)), torch.tensor(news)).cuda()
        place = torch.arange(sum(news), device="cuda") - starts[seq] + state.lens[seq]
        slots = state.slots(seq, place)
        state.lens += (starts[1:] - starts[:-1])
        x = torch.cat(xs)
        for b, cache in zip(self.blocks, state.caches):
            x = self._block(b, cache, x, slots, state.table, state.lens, starts, max(news), state.max_len, trace)
        return list(x.split(news))

    def step(self, state: State, x: torch.Tensor, trace=None) -> torch.Tensor:
        """One new token of every sequence, x bf16 [seqs][width]: the stream after the last block.  A ValueError, and
        nothing done, where a sequence has no room for it."""
        if x.dim() != 2 or x.shape[1] != self.width or x.dtype != torch.bfloat16:
            raise ValueError(f"tokens must be bf16 [sequences][{self.width}]")
        state.take([1] * x.shape[0])
        return self._step(state, x, trace)

    def _step(self, state: State, x: torch.Tensor, trace=None) -> torch.Tensor:
        seq = torch.arange(x.shape[0], device="cuda")
        slots = state.slots(seq, state.lens)
        state.lens += 1
        for b, cache in zip(self.blocks, state.caches):
            x = self._block(b, cache, x, slots, state.table, state.lens, None, 1, state.max_len, trace)
        return x


class Steps:
    """A captured step: each replay takes the sequences of its state one token further."""

    def __init__(self, state: State, graph: "torch.cuda.CUDAGraph"):
        self.state, self.graph = state, graph

    def replay(self) -> None:
        """A ValueError, and nothing done, where a sequence has no room for a token more."""
        self.state.take([1] * len(self.state.held))
        self.graph.replay()


def capture_step(dec: Decoder, state: State, x: torch.Tensor):
    """A step on the tensor x as a HIP graph: (``Steps`` to replay, its output)."""
    lens, held = state.lens.clone(), state.held
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):      # once outside the graph: kernels are loaded on their first launch
        dec.step(state, x)
    torch.cuda.current_stream().wait_stream(side)
    state.lens.copy_(lens)
    state.held = held
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = dec._step(state, x)
    return Steps(state, graph), out


def main(seqs: int = 16, prompt: int = 1000, steps: int = 64) -> None:
    dec = Decoder(blocks=4, width=2048, heads=16, kv_heads=4, head_dim=128, inner=8192)
    state = State(dec, seqs, prompt + steps + 1)
    g = torch.Generator(device="cuda").manual_seed(1)
    xs = [torch.randn(prompt, dec.width, generator=g, device="cuda").to(torch.bfloat16) for _ in range(seqs)]
    dec.prompt(State(dec, seqs, prompt), xs)
    torch.cuda.synchronize()
    t = time.perf_counter()
    last = torch.stack([y[-1] for y in dec.prompt(state, xs)])
    torch.cuda.synchronize()
    t = time.perf_counter() - t
    print(f"prompts: {seqs} of {prompt} tokens in {t * 1e3:.2f} ms, {seqs * prompt / t:.0f} tokens/s")
    graph, out = capture_step(dec, state, last)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(steps):
        graph.replay()
        last.copy_(out)
    torch.cuda.synchronize()
    t = time.perf_counter() - t
    held = sum(c.nbytes() for c in state.caches)
    print(f"steps: {steps} of {seqs} sequences in {t * 1e3:.2f} ms, {seqs * steps / t:.0f} tokens/s; "
          f"cache {held / 1e6:.1f} MB (bf16: {held * 64 / 17 / 1e6:.1f})")


if __name__ == "__main__":
    main()
