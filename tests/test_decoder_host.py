"""A decoder's state on the host: what has no room is refused before anything is launched (no GPU needed)."""
import pytest
import torch

from paper_1907_02154_amd import decoder


def made(held, max_len, width=8):
    """A decoder and a state without their device tensors: a call that gets as far as these fails otherwise."""
    dec, state = decoder.Decoder.__new__(decoder.Decoder), decoder.State.__new__(decoder.State)
    dec.width, dec.blocks = width, []
    state.held, state.max_len, state.page_size = held, max_len, 4
    return dec, state


def tokens(n, width=8, dtype=torch.bfloat16):
    return torch.zeros(n, width, dtype=dtype)


def test_prompts_and_steps_past_the_capacity():
    dec, state = made([3, 10], 10)
    with pytest.raises(ValueError, match="sequence 1 holds 10 tokens of 10"):
        dec.step(state, tokens(2))
    with pytest.raises(ValueError, match="sequence 0 holds 3 tokens of 10 at most: no room for 8 more"):
        dec.prompt(state, [tokens(8), tokens(0)])
    with pytest.raises(ValueError, match="no room"):
        decoder.Steps(state, None).replay()
    with pytest.raises(ValueError, match="no room"):
        dec.prompt(state, [tokens(7), tokens(1)])
    assert state.held == [3, 10]
    state.take([7, 0])                       # to the last place
    assert state.held == [10, 10]


def test_tokens_of_other_sequences_widths_and_types():
    dec, state = made([0, 0], 10)
    for xs in ([tokens(1)], [tokens(1)] * 3, [tokens(1), tokens(1, 7)], [tokens(1), tokens(1, dtype=torch.float32)],
               [tokens(1), tokens(1)[0]]):
        with pytest.raises(ValueError):
            dec.prompt(state, xs)
    for x in (tokens(1), tokens(3), tokens(2, 7), tokens(2, dtype=torch.float32), tokens(2)[0]):
        with pytest.raises(ValueError):
            dec.step(state, x)
    assert state.held == [0, 0]


@pytest.mark.parametrize("seqs,max_len,page", [(0, 8, 4), (1, 0, 4), (1, 8, 0)])
def test_states_that_hold_nothing(seqs, max_len, page):
    with pytest.raises(ValueError):
        decoder.State(None, seqs, max_len, page)


def test_slots_past_the_capacity_are_none():
    _, state = made([0, 0], 10)
    state.slot = state.slots_of(torch.tensor([[5, 0, 3], [1, 2, 4]], dtype=torch.int32), state.max_len, state.page_size)
    assert state.slot.dtype == torch.int32
    seq = torch.tensor([0, 0, 0, 1, 1, 1, 1])
    place = torch.tensor([0, 9, 10, 4, 11, 12, 1000])
    assert state.slots(seq, place).tolist() == [20, 13, -1, 8, -1, -1, -1]


def test_prompts_of_no_tokens():
    dec, state = made([3, 10], 10)
    out = dec.prompt(state, [tokens(0), tokens(0)])
    assert [tuple(x.shape) for x in out] == [(0, 8), (0, 8)] and state.held == [3, 10]
