"""The calls of a serving step on inputs whose results nearly cancel (tests/serving_rounding.py): no term of what meets the matrix cores is missing."""
import pytest
import torch

import serving_rounding as R
from paper_2506_23906_amd import binding as B

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def close(got, want, by, what):
    off = (got.cpu().double() - want).abs()
    assert bool((off <= by).all()), "%s: %.3g off, bound %.3g" % (what, float(off.max()), float(torch.as_tensor(by).max()))


@pytest.mark.parametrize("columns", [4, 900])   # a workgroup for the segment, the list of tiles
@pytest.mark.parametrize("dtype,cache_type", [(R.BF16, R.BF16), (R.F16, R.F16), (R.BF16, R.E4M3), (R.F16, R.E4M3)])
def test_probabilities(dtype, cache_type, columns):
    print(dtype, cache_type, columns, flush=True)
    q, k, v, scale, weights, values, want, by = R.cancelling_probabilities(dtype, cache_type)
    out = B.mmv_paged_attention(q.cuda(), B.PagedCache(k.cuda(), v.cuda()), ints([[0, 1, 2, 3] + [-1] * (columns - 4)]), ints([61]), scale=scale)
    close(out, want, by, "out")


@pytest.mark.parametrize("columns", [4, 900])
def test_probabilities_of_24_bits(columns):
    q, k, v, scale, weights, values, want, by = R.probabilities_of_24_bits()
    out = B.mmv_paged_attention(q.cuda(), B.PagedCache(k.cuda(), v.cuda()), ints([[0, 1, 2, 3] + [-1] * (columns - 4)]), ints([7]), scale=scale)
    close(out, want, by, "out")


@pytest.mark.parametrize("dtype", [R.BF16, R.F16])
def test_a_flat_tail_counts_in_the_sum(dtype):
    """4096 rows, so that a wave has whole rows of 65536 positions."""
    q, k, v, scale, _, _, want_lse, lse_by = R.flat_tail(dtype, 1.0)
    n, pages = 4096, (1 << 16) // 16
    table = torch.ones(n, pages, dtype=torch.int32, device="cuda")
    table[:, 0] = 0
    lse = torch.empty(n, 1, device="cuda")
    B.mmv_paged_attention(q.expand(n, 1, 8).contiguous().cuda(), B.PagedCache(k.cuda(), v.cuda()), table, torch.full((n,), 1 << 16, dtype=torch.int32, device="cuda"), scale=scale, lse=lse)
    close(lse, want_lse, lse_by, "lse")


@pytest.mark.parametrize("dtype", [R.BF16, R.F16])
@pytest.mark.parametrize("first_value", [0.0, 1.0])
def test_a_flat_tail_keeps_its_weight(first_value, dtype):
    """4096 rows, so that a wave has whole rows of 65536 positions."""
    q, k, v, scale, want, by, _, _ = R.flat_tail(dtype, first_value)
    n, pages = 4096, (1 << 16) // 16
    table = torch.ones(n, pages, dtype=torch.int32, device="cuda")
    table[:, 0] = 0
    out = B.mmv_paged_attention(q.expand(n, 1, 8).contiguous().cuda(), B.PagedCache(k.cuda(), v.cuda()), table, torch.full((n,), 1 << 16, dtype=torch.int32, device="cuda"), scale=scale)
    close(out, want, by, "out")


@pytest.mark.parametrize("dtype", [R.BF16, R.F16])
@pytest.mark.parametrize("tokens", [70, 700])   # one block, several
def test_states(tokens, dtype):
    q, k, v, state, _, want, by = R.cancelling_state(dtype, tokens)
    given = state.cuda()
    out = B.mmv_decay_attention(q.cuda(), k.cuda(), v.cuda(), ints([0, tokens]), torch.zeros(1, device="cuda"), scale=1.0, state_in=given, state_out=given)
    close(out, want, by, "out")
    assert torch.equal(given.cpu(), state)


@pytest.mark.parametrize("dtype", [R.BF16, R.F16])
@pytest.mark.parametrize("tokens", [70, 700])
def test_scores(tokens, dtype):
    q, k, v, _, want, by = R.cancelling_scores(dtype, tokens)
    out = B.mmv_decay_attention(q.cuda(), k.cuda(), v.cuda(), ints([0, tokens]), torch.zeros(1, device="cuda"), scale=1.0)
    close(out[1:], want, by, "out")


@pytest.mark.parametrize("dtype", [R.BF16, R.F16])
@pytest.mark.parametrize("tokens", [40, 700])
def test_decayed_values(tokens, dtype):
    q, k, v, ld, values, by_decay, by = R.decayed_values(dtype, tokens)
    state = torch.zeros(1, 1, 16, 32, device="cuda")
    B.mmv_decay_attention(q.cuda(), k.cuda(), v.cuda(), ints([0, tokens]), ld.cuda(), scale=1.0, state_out=state)
    close(state[0, 0, 5], values * by_decay, by, "state")
