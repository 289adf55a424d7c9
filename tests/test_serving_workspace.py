"""Scratch of prompts' recurrence: states between a request's blocks, for requests that can have several.  No GPU."""
import pytest

from paper_2506_23906_amd import binding as B


@pytest.mark.parametrize("n,length,heads,dk,dv", [(1000, 100, 16, 128, 128), (1000, 100, 32, 128, 256), (4000, 30, 8, 64, 64), (100000, 3, 4, 128, 128)])
def test_many_short_prompts_take_little(libmmvseg_path, n, length, heads, dk, dv):
    """No more than the keys, values, queries and outputs of the tokens themselves, whose states these are; a state for every request was up to 4 GB."""
    need = B.mmv_decay_attention_workspace_bytes(n, n * length, heads, dk, dv)
    assert 0 < need <= n * length * heads * (2 * dk + 2 * dv) * 2, need


@pytest.mark.parametrize("n,tokens,heads,dk,dv", [(1, 257, 1, 8, 8), (3, 1000, 8, 64, 64), (12, 63000, 16, 128, 128), (64, 100000, 2, 64, 64), (65, 100000, 2, 64, 64), (300, 400000, 32, 128, 256)])
def test_there_is_room_for_any_lengths(libmmvseg_path, n, tokens, heads, dk, dv):
    """A request of all the tokens has as many blocks as there are tokens for; one state for each block of every request of several, whatever the lengths."""
    slots = B.mmv_decay_attention_workspace_bytes(n, tokens, heads, dk, dv) // (4 * heads * dk * dv)
    assert slots >= 2
    if n <= 64:
        assert slots <= 2 * tokens // 64
