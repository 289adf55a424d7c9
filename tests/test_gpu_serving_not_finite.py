"""Attention over a paged cache where queries, keys or values are not finite: the same whichever waves share a segment."""
import math
import random

import pytest
import torch

from paper_2506_23906_amd import binding as B
from serving_util import check, e4m3, plain_attention

pytestmark = pytest.mark.gpu
BF16, F16, E4M3 = torch.bfloat16, torch.float16, torch.float8_e4m3fn
NAN = float("nan")
PAGE = 16
# positions of the longest row, columns of the table: one wave, the waves of a workgroup, the list of tiles (parts of a tile each; more than eight parts for every joining wave)
FORMS = {"one wave": (30, 2), "workgroup": (200, 15), "list": (700, 900), "long list": (6000, 900)}
TYPES = [(BF16, BF16), (F16, F16), (BF16, E4M3), (F16, E4M3)]


def case(form, dtype, cache_type, heads=2, group=4, dim=64, seed=1):
    """Two rows: keys and values on the CPU in the cache's type, the table, queries, contexts."""
    longest, columns = FORMS[form]
    contexts = [longest, max(1, longest - 3)]
    counts = [-(-c // PAGE) for c in contexts]
    ids = list(range(sum(counts)))
    random.Random(seed).shuffle(ids)
    table = [ids[:counts[0]] + [-1] * (columns - counts[0]), ids[counts[0]:] + [-1] * (columns - counts[1])]
    g = torch.Generator().manual_seed(seed)
    k, v = (torch.randn(len(ids), heads, PAGE, dim, generator=g) for _ in "kv")
    k, v = (e4m3(x, 1.0) if cache_type == E4M3 else x.to(cache_type) for x in (k, v))
    q = torch.randn(2, heads * group, dim, generator=g).to(dtype)
    return k, v, table, q, contexts


def run(k, v, table, q, contexts, scale=0.125):
    cache = B.PagedCache(k.cuda(), v.cuda())
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    out = B.mmv_paged_attention(q.cuda(), cache, torch.tensor(table, dtype=torch.int32, device="cuda"), torch.tensor(contexts, dtype=torch.int32, device="cuda"), scale=scale, lse=lse)
    return out.cpu(), lse.cpu()


def put(x, table, row, position, value, heads=slice(None), dims=slice(None)):
    raw = x.view(torch.uint8) if x.dtype == E4M3 else x
    raw[table[row][position // PAGE], heads, position % PAGE, dims] = 0x7F if x.dtype == E4M3 and value != value else value


@pytest.mark.parametrize("dtype,cache_type", TYPES)
@pytest.mark.parametrize("form", FORMS)
def test_a_query_that_is_not_a_number_stays_one(form, dtype, cache_type):
    print(form, dtype, cache_type, flush=True)
    k, v, table, q, contexts = case(form, dtype, cache_type)
    want, want_lse, by, lse_by = plain_attention(q, k, v, table, contexts, 0.125, 0)
    q[0, 1, 5], q[1, 6, :] = NAN, NAN
    out, lse = run(k, v, table, q, contexts)
    bad = torch.zeros(2, 8, dtype=torch.bool)
    bad[0, 1] = bad[1, 6] = True
    assert bool(out[bad].isnan().all()) and bool(lse[bad].isnan().all())
    check(out[~bad], want[~bad], by[~bad], "the other heads")
    check(lse[~bad], want_lse[~bad], lse_by[~bad], "their lse")


@pytest.mark.parametrize("dtype,cache_type", TYPES)
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("where", ["first", "last", "page"])
def test_keys_that_are_not_numbers_reach_their_row_and_head(form, where, dtype, cache_type):
    """One position, a last part of a single one, a whole page: every query of the row's head is not a number, and nothing else is."""
    print(form, where, dtype, cache_type, flush=True)
    k, v, table, q, contexts = case(form, dtype, cache_type)
    if contexts[0] > 64:   # (the last tile has one position alone)
        contexts[0] = contexts[0] // 32 * 32 + 1
    want, want_lse, by, lse_by = plain_attention(q, k, v, table, contexts, 0.125, 0)
    positions = {"first": [0], "last": [contexts[0] - 1], "page": range(PAGE * (contexts[0] // PAGE // 2), PAGE * (contexts[0] // PAGE // 2 + 1))}[where]
    for p in positions:
        if p < contexts[0]:
            put(k, table, 0, p, NAN, heads=1)
    out, lse = run(k, v, table, q, contexts)
    bad = torch.zeros(2, 8, dtype=torch.bool)
    bad[0, 4:] = True
    assert bool(out[bad].isnan().all()) and bool(lse[bad].isnan().all())
    check(out[~bad], want[~bad], by[~bad], "the other heads")
    check(lse[~bad], want_lse[~bad], lse_by[~bad], "their lse")


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("form", FORMS)
def test_a_key_of_minus_infinity_has_no_weight(form, dtype):
    print(form, dtype, flush=True)
    k, v, table, q, contexts = case(form, dtype, dtype)
    q[..., 0] = 1.0
    put(k, table, 1, 2, -1e4, dims=0)      # (exp(-1250) is 0 in 64 bits too)
    want, want_lse, by, lse_by = plain_attention(q, k, v, table, contexts, 0.125, 0)
    put(k, table, 1, 2, 0.0)
    _, _, by, lse_by = plain_attention(q, k, v, table, contexts, 0.125, 0)   # (bounds of scores of ordinary size)
    put(k, table, 1, 2, -math.inf, dims=0)
    out, lse = run(k, v, table, q, contexts)
    check(out, want, by, "out")
    check(lse, want_lse, lse_by, "lse")


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("form", FORMS)
def test_infinite_values_reach_their_component_alone(form, dtype):
    """A value of ordinary weight is that infinity; one whose weight vanishes need not be (0 times it is no number), but what comes out is not finite either."""
    print(form, dtype, flush=True)
    k, v, table, q, contexts = case(form, dtype, dtype)
    # what has all the weight of row 1 lies in its first part, what has none in its last
    q[1, :, 0] = 8.0
    put(k, table, 1, 0, 0.0)
    put(k, table, 1, 0, 1000.0, dims=0)
    want, want_lse, by, lse_by = plain_attention(q, k, v, table, contexts, 0.125, 0)
    put(v, table, 0, contexts[0] // 2, math.inf, heads=0, dims=9)
    put(v, table, 0, contexts[0] // 3, -math.inf, heads=1, dims=3)
    put(v, table, 1, contexts[1] - 1, math.inf, heads=1, dims=63)
    out, lse = run(k, v, table, q, contexts)
    assert bool((out[0, :4, 9] == math.inf).all()) and bool((out[0, 4:, 3] == -math.inf).all())
    assert not bool(out[1, 4:, 63].isfinite().any())
    keep = torch.ones_like(want, dtype=torch.bool)
    keep[0, :4, 9] = keep[0, 4:, 3] = keep[1, 4:, 63] = False
    check(out[keep], want[keep], by[keep], "the other components")
    check(lse, want_lse, lse_by, "lse")


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("form", FORMS)
def test_large_finite_values_without_weight_add_nothing(form, dtype):
    """Values near the largest of the type at positions whose probability is 0 in 32 bits."""
    print(form, dtype, flush=True)
    k, v, table, q, contexts = case(form, dtype, dtype)
    q[:, :, 0] = 8.0
    for row in (0, 1):
        put(k, table, row, 1, 0.0)
        put(k, table, row, 1, 1000.0, dims=0)     # (exp(-900) of the others beside it)
    want, want_lse, by, lse_by = plain_attention(q, k, v, table, contexts, 0.125, 0)
    large = 1e35 if dtype == BF16 else 65504.0    # (times the probabilities of a part that has no other base still finite in 32 bits)
    for row in (0, 1):
        for p in range(3, contexts[row], 5):
            put(v, table, row, p, large, dims=slice(7, 40))
    out, lse = run(k, v, table, q, contexts)
    check(out, want, by, "out")
    check(lse, want_lse, lse_by, "lse")
