"""What paper_2506_23906_amd/serving_step.py keeps between steps: its list of free pages and its workspaces.  The calls are replaced by plain ones on the CPU."""
import types

import pytest
import torch

from paper_2506_23906_amd import serving_step as M
from serving_util import plain_tables


@pytest.fixture
def calls(monkeypatch):
    """Stands in for the binding: page tables as they are, attention and recurrence of zeros; keeps the slots of every append and the scratch of every attention."""
    seen = types.SimpleNamespace(slots=[], scratch=[])

    def tables(cached, new, free, table, page, max_tokens, ws=None):
        got = plain_tables(cached.tolist(), new.tolist(), free.tolist(), table.tolist(), page, max_tokens)
        table.copy_(torch.tensor(got["table"], dtype=torch.int32))
        return types.SimpleNamespace(**{n: torch.tensor(got[n], dtype=torch.int64 if n in ("slots", "used") else torch.int32) for n in ("offsets", "context", "slots", "positions", "used")})

    def attention(q, cache, table, context, ws=None):
        seen.scratch.append(ws)
        return torch.zeros_like(q)

    def compress(x, mask, n, out=None, count=None, ws=None):
        kept = x[mask.bool()]
        out[:kept.numel()] = kept
        return out, count

    monkeypatch.setattr(M, "B", types.SimpleNamespace(
        PagedCache=lambda *a: a, workspace=lambda nbytes, device=None: torch.empty(max(256, nbytes), dtype=torch.uint8), new_workspace=lambda *a: torch.empty(256, dtype=torch.uint8),
        MMV_OP_COMPRESS=4, MMV_I8_I32=0, MMV_FLAGS_U8=0,
        mmv_page_tables_workspace_bytes=lambda n: 0, mmv_page_tables=tables, mmv_compress=compress,
        mmv_cache_append=lambda k, v, slots, cache: seen.slots.append(slots.tolist()),
        mmv_paged_attention_workspace_bytes=lambda n, *a: 1000 * n, mmv_paged_attention=attention,
        mmv_decay_attention_workspace_bytes=lambda *a: 0))
    return seen


def server(requests, longest):
    shape = M.Shape(layers=1, heads=4, dim=32, vocabulary=50, page=8)
    return M.Server(shape, M.weights(shape, device="cpu"), requests, longest, device="cpu")


def prompts(s, lengths):
    s.prompts(torch.zeros(sum(lengths), dtype=torch.int64), torch.tensor(lengths, dtype=torch.int32))


def test_a_request_that_grows_past_the_longest_takes_nobodys_pages(calls):
    """Two columns of eight positions for each of four requests; the first two run 25 positions past them while the others fill theirs."""
    s = server(4, 16)
    prompts(s, [15, 16, 1, 3])
    owner = {slot: r for r, slots in enumerate(torch.tensor(calls.slots[-1]).split([15, 16, 1, 3])) for slot in slots.tolist()}
    assert len(owner) == 35
    lengths = [15, 16, 1, 3]
    for _ in range(26):
        s.step()
        for r, slot in enumerate(calls.slots[-1]):
            if lengths[r] < 16:
                assert slot >= 0 and slot not in owner, (r, lengths[r], slot)
                owner[slot] = r
            else:
                assert slot == -1
            lengths[r] += 1
    held, free = s.table.flatten().tolist(), s.free[s.free >= 0].tolist()
    assert len(set(held)) == 8 and sorted(held + free) == list(range(s.free.numel())) and s.cached.tolist() == lengths
    with pytest.raises(ValueError):
        prompts(s, [1, 1, 1, 1])
    with pytest.raises(ValueError):
        prompts(server(2, 16), [3, 17])


def test_full_requests_at_the_end_of_a_page_leave_the_last_pages_to_others(calls):
    """Three of four requests are full and would open another page in the very step in which the last one opens its own."""
    s = server(4, 16)
    prompts(s, [16, 16, 16, 8])
    s.step()
    assert calls.slots[-1][:3] == [-1] * 3 and calls.slots[-1][3] >= 0


def test_the_free_pages_keep_their_order(calls):
    s = server(3, 40)
    first = s.free.tolist()
    prompts(s, [9, 1, 17])
    assert s.free.tolist() == first[6:] + [-1] * 6 and s.table[s.table >= 0].tolist() == first[:6]
    for _ in range(8):
        s.step()
    assert s.free.tolist() == first[9:] + [-1] * 9


def test_a_steps_scratch_is_its_own(calls):
    """A captured step goes on using the scratch it was recorded with: prompts of more tokens may not replace it."""
    s = server(3, 80)
    prompts(s, [2, 1, 1])
    s.step()
    own = calls.scratch[-1]
    prompts(s, [30, 20, 9])
    assert calls.scratch[-1].numel() >= 59000
    s.step()
    assert calls.scratch[-1] is own
