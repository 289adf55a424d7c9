"""The calls of a serving step over a ragged batch against their plain forms in 64 bits (tests/serving_util.py)."""
import math
import random

import pytest
import torch

from paper_2506_23906_amd import binding as B
from serving_util import E4M3_MOST, check, e4m3, plain_attention, plain_decay, plain_tables

pytestmark = pytest.mark.gpu
BF16, F16, E4M3 = torch.bfloat16, torch.float16, torch.float8_e4m3fn
NAN = float("nan")


def ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


def normal(seed, *shape, dtype=BF16, by=1.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * by).to(dtype)


# ---- page tables --------------------------------------------------------------------------------------------------


def tables_case(rng, n, page, hi, new_hi, spare=0, short=0):
    cached, new = [rng.choice([0, 1, page - 1, page, page + 1, rng.randint(0, hi)]) for _ in range(n)], [rng.choice([0, 1, rng.randint(0, new_hi)]) for _ in range(n)]
    held, need = [-(-c // page) for c in cached], [-(-(c + m) // page) for c, m in zip(cached, new)]
    ids = list(range(sum(need) + 5))
    rng.shuffle(ids)
    width = max(1, max(need + held, default=0) + 1 - short)
    table, at = [], 0
    for r in range(n):
        table.append((ids[at:at + held[r]] + [-1] * width)[:width])
        at += held[r]
    free = ids[at:at + max(0, sum(need) - sum(held) + spare)]
    return cached, new, free, table


def run_tables(cached, new, free, table, page, max_tokens, columns=0, ws=None):
    n, width = len(new), len(table[0]) if table else 1
    buffer = torch.full((max(n, 1), width + columns), -7, dtype=torch.int32, device="cuda")
    if n:
        buffer[:n, :width] = ints(table)
    rows = buffer[:n, :width]
    got = B.mmv_page_tables(ints(cached), ints(new), ints(free), rows, page, max_tokens, ws=ws)
    want = plain_tables(cached, new, free, table, page, max_tokens)
    for name in ("offsets", "context", "slots", "positions", "used"):
        assert getattr(got, name).tolist() == want[name], name
    assert rows.tolist() == want["table"] and bool((buffer[:, width:] == -7).all())


@pytest.mark.parametrize("n,page,hi,new_hi", [(0, 16, 1, 1), (1, 16, 1, 1), (1, 1, 40, 3), (7, 8, 100, 700), (64, 16, 300, 1), (65, 13, 90, 33), (257, 64, 500, 40),
                                              (1000, 16, 50, 1), (2048, 8, 20, 3), (2049, 8, 20, 3), (5000, 256, 600, 2)])
@pytest.mark.parametrize("room", [0, 5])
def test_page_tables(n, page, hi, new_hi, room):
    print(n, page, hi, new_hi, room, flush=True)
    cached, new, free, table = tables_case(random.Random(n + page), n, page, hi, new_hi, spare=room)
    run_tables(cached, new, free, table, page, sum(new) + room, columns=room)


@pytest.mark.parametrize("n", [9, 3000])
def test_page_tables_leave_out_what_has_no_place(n):
    """Free pages used up, rows too short, fewer places for tokens than tokens, pages that the row does not have, negative lengths."""
    cached, new, free, table = tables_case(random.Random(n), n, 8, 60, 30)
    run_tables(cached, new, free[:len(free) // 2], table, 8, sum(new))
    run_tables(cached, new, [], table, 8, sum(new))
    run_tables(cached, new, free, table, 8, sum(new) // 2)
    run_tables(cached, new, free, table, 8, 0)
    cached, new, free, table = tables_case(random.Random(n + 1), n, 8, 60, 30, short=4)
    run_tables(cached, new, free, table, 8, sum(new) + 3)
    run_tables(cached, new, free, [[-1] * len(row) for row in table], 8, sum(new) + 3)
    cached[1], new[2] = -5, -2
    run_tables(cached, new, free, table, 8, sum(max(x, 0) for x in new))


def test_page_tables_of_lengths_whose_sum_passes_32_bits():
    big = 2 ** 31 - 1
    table = torch.full((3, 4), -1, dtype=torch.int32, device="cuda")
    got = B.mmv_page_tables(ints([0, 5, big]), ints([big, big, big]), ints([3, 1]), table, 16, 40)
    assert got.offsets.tolist() == [0, big, big, big] and got.context.tolist() == [big, big, big]
    assert got.used[1].item() == 3 * big and got.positions.tolist() == list(range(40))
    assert got.slots.tolist() == [48 + i for i in range(16)] + [16 + i for i in range(16)] + [-1] * 8
    assert table.tolist() == [[3, 1, -1, -1], [-1] * 4, [-1] * 4]


# ---- cache append -------------------------------------------------------------------------------------------------


def cache_pair(seed, pages, heads, page, dim, dtype, order="heads", scale=(0.03, 0.05)):
    """A cache on the GPU and its values on the CPU; "slots": a page's slots lie before its heads."""
    def one(s):
        x = normal(s, pages, heads, page, dim)
        x = e4m3(x, scale[s % 2]) if dtype == E4M3 else x.to(dtype)
        t = x.cuda()
        if order == "slots":
            t = t.view(torch.uint8 if dtype == E4M3 else dtype).transpose(1, 2).contiguous().transpose(1, 2)
            t = t.view(E4M3) if dtype == E4M3 else t
        return t, x
    (k, kc), (v, vc) = one(2 * seed), one(2 * seed + 1)
    scales = scale if dtype == E4M3 else (1.0, 1.0)
    return B.PagedCache(k, v, *scales), kc, vc


def bits(x):
    return x.cpu().contiguous().view(torch.uint8 if x.dtype == E4M3 else torch.int16)


@pytest.mark.parametrize("dtype,cache_type", [(BF16, BF16), (F16, F16), (BF16, E4M3), (F16, E4M3)])
@pytest.mark.parametrize("tokens,heads,dim,page,order", [(1, 1, 8, 16, "heads"), (3, 2, 72, 8, "slots"), (33, 8, 128, 13, "heads"), (257, 3, 160, 1, "slots"), (300, 5, 256, 64, "heads")])
def test_cache_append(dtype, cache_type, tokens, heads, dim, page, order):
    print(dtype, cache_type, tokens, heads, dim, page, order, flush=True)
    pages = tokens // page + 3
    cache, kc, vc = cache_pair(tokens, pages, heads, page, dim, cache_type, order)
    fused = normal(tokens + 9, tokens, 3 * heads * dim, dtype=dtype)
    fused.view(-1)[:6] = torch.tensor([math.inf, -math.inf, NAN, 1e4, -0.0, 1e-7]).to(dtype)
    k, v = fused[:, :heads * dim].unflatten(1, (heads, dim)), fused[:, 2 * heads * dim:].unflatten(1, (heads, dim))
    slots = torch.randperm(pages * page, generator=torch.Generator().manual_seed(5))[:tokens]
    if tokens > 4:
        slots[1], slots[tokens // 2], slots[tokens - 1] = -1, pages * page, 2 ** 40
    on_gpu = fused.cuda()
    B.mmv_cache_append(on_gpu[:, :heads * dim].unflatten(1, (heads, dim)), on_gpu[:, 2 * heads * dim:].unflatten(1, (heads, dim)), slots.cuda(), cache)
    for x, c, now, scale in ((k, kc, cache.k, cache.k_scale), (v, vc, cache.v, cache.v_scale)):
        for t, s in enumerate(slots.tolist()):
            if 0 <= s < pages * page:
                c[s // page, :, s % page] = e4m3(x[t], scale) if cache_type == E4M3 else x[t]
        now, c = now.cpu(), c
        same = bits(now) == bits(c)
        assert bool((same | (now.float().isnan() & c.float().isnan())).all())


# ---- paged attention ----------------------------------------------------------------------------------------------


def attention_case(seed, contexts, heads, group, dim, page, dtype, cache_type, order="heads"):
    rng, width = random.Random(seed), max(-(-max(contexts + [0]) // page) + 1, 1)
    counts = [-(-max(c, 0) // page) for c in contexts]
    pages = sum(counts) + 2
    ids = list(range(pages))
    rng.shuffle(ids)
    table, at = [], 0
    for c in counts:
        table.append((ids[at:at + c] + [-1] * width)[:width])
        at += c
    cache, kc, vc = cache_pair(seed, pages, heads, page, dim, cache_type, order)
    return cache, kc, vc, table, normal(seed + 1, len(contexts), heads * group, dim, dtype=dtype, by=1.5)


def run_attention(cache, kc, vc, table, q, contexts, window=0, scale=None, what="", q_on_gpu=None):
    scale = q.shape[2] ** -0.5 if scale is None else scale
    q_on_gpu = q.cuda() if q_on_gpu is None else q_on_gpu
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    out = B.mmv_paged_attention(q_on_gpu, cache, ints(table), ints(contexts), scale=scale, window=window, lse=lse)
    want, want_lse, by, lse_by = plain_attention(q, kc, vc, table, contexts, scale, window, cache.k_scale, cache.v_scale)
    check(out, want, by, what + " out")
    check(lse, want_lse, lse_by, what + " lse")
    return out


TYPES = [(BF16, BF16), (F16, F16), (BF16, E4M3), (F16, E4M3)]


@pytest.mark.parametrize("dtype,cache_type", TYPES)
@pytest.mark.parametrize("heads,group,dim,page,order", [(1, 1, 8, 8, "heads"), (2, 1, 64, 16, "heads"), (3, 5, 72, 8, "slots"), (1, 16, 80, 24, "heads"), (2, 4, 112, 32, "slots"),
                                                        (8, 4, 128, 16, "heads"), (1, 7, 136, 128, "heads"), (2, 8, 160, 64, "slots"), (1, 2, 192, 40, "heads"), (2, 3, 256, 16, "heads"),
                                                        (2, 2, 32, 8, "heads"), (1, 3, 96, 8, "heads")])
def test_attention_at_ragged_lengths(heads, group, dim, page, order, dtype, cache_type):
    contexts = [0, 1, 2, 7, 8, 9, 31, 32, 33, 63, 64, 65, 100, 257, 700]
    random.Random(dim).shuffle(contexts)
    print(heads, group, dim, page, order, dtype, cache_type, flush=True)
    run_attention(*attention_case(dim, contexts, heads, group, dim, page, dtype, cache_type, order), contexts)


@pytest.mark.parametrize("window", [1, 5, 32, 33, 100, 5000])
@pytest.mark.parametrize("dtype,cache_type", TYPES)
def test_attention_in_a_window(window, dtype, cache_type):
    contexts = [1, 33, 0, 100, 101, 640, 1500]
    print(window, dtype, cache_type, flush=True)
    run_attention(*attention_case(window, contexts, 2, 4, 128, 16, dtype, cache_type), contexts, window=window)
    run_attention(*attention_case(window, contexts, 3, 1, 64, 24, dtype, cache_type), contexts, window=window)


@pytest.mark.parametrize("n,hi", [(1, 1), (1, 20_000), (3, 9000), (70, 300), (300, 40), (1500, 9)])
def test_attention_of_few_and_many_rows(n, hi):
    """From one long context, whose parts are joined, to more rows than any list in a kernel."""
    rng = random.Random(n)
    contexts = [rng.randint(0, hi) if i else hi for i in range(n)]
    run_attention(*attention_case(n, contexts, 2, 2, 64, 16, BF16, BF16), contexts, what=str(n))


def test_attention_does_not_use_what_is_left_out():
    """NaN and infinities behind the context, before the window, in pages of nobody, and lengths that the table does not hold."""
    for heads, group, dim, page, dtype, cache_type in ((2, 4, 128, 16, BF16, BF16), (1, 3, 72, 8, F16, F16), (2, 2, 64, 32, BF16, E4M3), (1, 8, 256, 8, BF16, BF16)):
        contexts, window = [37, 5, 0, 129, 64, 200], 60
        cache, kc, vc, table, q = attention_case(3, contexts, heads, group, dim, page, dtype, cache_type)
        seen = set()
        for r, c in enumerate(contexts):
            seen |= {(table[r][p // page], p % page) for p in range(max(0, c - window), c)}
        for x, on_gpu in ((kc, cache.k), (vc, cache.v)):
            raw = x.view(torch.uint8) if cache_type == E4M3 else x
            for i in range(x.shape[0]):
                for s in range(page):
                    if (i, s) not in seen:
                        raw[i, :, s] = 0x7F if cache_type == E4M3 else (NAN, math.inf, -math.inf)[(i + s) % 3]
            (on_gpu.view(torch.uint8) if cache_type == E4M3 else on_gpu).copy_(raw)
        run_attention(cache, kc, vc, table, q, contexts, window=window)
        # pages that the cache does not have; a context beyond the table; a negative one
        table[3][5:7], table[5][-1] = [-1] * len(table[3][5:7]), 10 ** 9
        table[0] = [-5] * len(table[0])
        contexts[1] = -3
        run_attention(cache, kc, vc, table, q, contexts, window=window)
        width = max(len(row) for row in table)
        contexts[4] = contexts[5] = width * page + 1000
        out = run_attention(cache, kc, vc, table, q, contexts, window=1)
        assert bool((out[0] == 0).all())


def test_attention_of_values_that_are_not_finite_and_of_large_scores():
    """A value's infinity reaches its own component alone; scores that differ by more than fp32's exponent can say; -infinity in a key."""
    contexts = [40, 70]
    cache, kc, vc, table, q = attention_case(11, contexts, 1, 2, 64, 8, BF16, BF16)
    vc[table[0][1], 0, 3, 5] = math.inf
    kc[table[1][0], 0, 2, 0], q[1, :, 0] = -math.inf, 1.0
    cache.k.copy_(kc), cache.v.copy_(vc)
    scale = 40.0
    lse = torch.empty(2, 2, device="cuda")
    out = B.mmv_paged_attention(q.cuda(), cache, ints(table), ints(contexts), scale=0.125, lse=lse)
    want, want_lse, by, lse_by = plain_attention(q, kc, vc, table, contexts, 0.125, 0)
    assert bool((out[0, :, 5] == math.inf).all())
    by, lse_by = by.nan_to_num(nan=0.05), lse_by.nan_to_num(nan=1e-4, posinf=1e-4)   # (the bound of a row with an infinite score is not finite)
    check(out[0], want[0], by[0].nan_to_num(posinf=0.0), "infinite value")
    vc[table[0][1], 0, 3, 5] = kc[table[1][0], 0, 2, 0] = 0.5
    cache.k.copy_(kc), cache.v.copy_(vc)
    run_attention(cache, kc, vc, table, q, contexts, scale=scale)
    run_attention(cache, kc, vc, table, q, contexts, scale=0.0)
    run_attention(cache, kc, vc, table, q, contexts, scale=-0.3)


def test_attention_takes_views():
    """Queries in a fused projection, rows of a wider table, scratch full of garbage, another stream."""
    contexts = [300, 17, 64]
    cache, kc, vc, table, q = attention_case(21, contexts, 2, 4, 80, 16, F16, F16)
    fused = torch.full((3, 8 * 80 + 96), NAN, dtype=F16, device="cuda")
    fused[:, 48:48 + 640] = q.flatten(1).cuda()
    wide = torch.full((5, len(table[0]) + 9), 10 ** 9, dtype=torch.int32, device="cuda")
    wide[:3, :len(table[0])] = ints(table)
    need = B.mmv_paged_attention_workspace_bytes(3, 8, 2, 80, wide.shape[1] * 16)
    ws, side = torch.full((max(need, 256),), 0xFF, dtype=torch.uint8, device="cuda"), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = torch.full((3, 8, 80), NAN, dtype=F16, device="cuda")
    with torch.cuda.stream(side):
        B.mmv_paged_attention(fused[:, 48:688].unflatten(1, (8, 80)), cache, wide, ints(contexts), out=got, ws=ws)
    side.synchronize()
    want, _, by, _ = plain_attention(q, kc, vc, table, contexts, 80 ** -0.5, 0)
    check(got, want, by, "views")


def test_attention_and_append_beyond_32_bit_offsets():
    """A cache of 5 GB: the pages at its end hold the context."""
    heads, page, dim, pages = 2, 64, 128, 160_000
    k = torch.zeros(pages, heads, page, dim, dtype=BF16, device="cuda")
    v = torch.zeros_like(k)
    cache, contexts = B.PagedCache(k, v), [100, 64]
    table = [[pages - 1, pages - 3], [pages - 2, -1]]
    new_k, new_v = normal(1, 164, heads, dim), normal(2, 164, heads, dim)
    slots = [table[0][i // page] * page + i % page for i in range(100)] + [table[1][0] * page + i for i in range(64)]
    B.mmv_cache_append(new_k.cuda(), new_v.cuda(), ints(slots, torch.int64), cache)
    small = torch.zeros(2, 4, heads, page, dim, dtype=BF16)
    for x, c, s in ((new_k, k, small[0]), (new_v, v, small[1])):
        for t, slot in enumerate(slots):
            s[slot // page - (pages - 4), :, slot % page] = x[t]
        assert torch.equal(c[-4:].cpu(), s) and not bool(c[:-4].any())
    q = normal(3, 2, 2 * heads, dim)
    out = B.mmv_paged_attention(q.cuda(), cache, ints(table), ints(contexts))
    want, _, by, _ = plain_attention(q, small[0], small[1], [[3, 1], [2, -1]], contexts, dim ** -0.5, 0)
    check(out, want, by, "far pages")


def test_attention_of_slots_that_lie_far_apart():
    """Pages side by side, slot behind slot: 24 slots are more than 2^32 elements."""
    heads, page, dim, pages, context = 1, 32, 64, 2_900_000, 75
    k, v = (torch.empty(page, pages, heads, dim, dtype=torch.uint8, device="cuda").view(E4M3).permute(1, 2, 0, 3) for _ in "kv")
    assert 24 * k.stride(2) > 2 ** 32
    cache, table = B.PagedCache(k, v, 0.02, 0.03), [[pages - 1, 7, pages - 2]]
    new_k, new_v = normal(1, context, heads, dim), normal(2, context, heads, dim)
    slots = [table[0][i // page] * page + i % page for i in range(context)]
    B.mmv_cache_append(new_k.cuda(), new_v.cuda(), ints(slots, torch.int64), cache)
    small = torch.zeros(2, 3, heads, page, dim, dtype=torch.uint8).view(E4M3)
    for x, s, by in ((new_k, small[0], 0.02), (new_v, small[1], 0.03)):
        held = e4m3(x, by)
        for t in range(context):
            s[t // page, :, t % page] = held[t]
    q = normal(3, 1, 4, dim)
    out = B.mmv_paged_attention(q.cuda(), cache, ints(table), ints([context]))
    want, _, by, _ = plain_attention(q, small[0], small[1], [[0, 1, 2]], [context], dim ** -0.5, 0, 0.02, 0.03)
    check(out, want, by, "far slots")


# ---- linear attention with decay ----------------------------------------------------------------------------------


def decays(heads, kind="spread"):
    if kind == "none":
        return torch.zeros(heads)
    if kind == "hard":
        return torch.tensor([(-40.0, -math.inf, -3.0, -1e-3)[h % 4] for h in range(heads)])
    return torch.tensor([-(2.0 ** (-8.0 * (h + 1) / heads)) for h in range(heads)])


def run_decay(lengths, heads, group, dk, dv, dtype, kind="spread", states="both", step=False, seed=0, before=0, after=0):
    print(lengths[:20], heads, group, dk, dv, dtype, kind, states, step, flush=True)
    n, kv, tokens = len(lengths), heads // group, sum(lengths) + before + after
    q, k, v = normal(seed, tokens, heads, dk, dtype=dtype), normal(seed + 1, tokens, kv, dk, dtype=dtype), normal(seed + 2, tokens, kv, dv, dtype=dtype)
    ends = [before]
    for x in lengths:
        ends.append(ends[-1] + x)
    ld, scale = decays(heads, kind), dk ** -0.5
    first = normal(seed + 3, n + 2, heads, dk, dv, dtype=torch.float32)
    index = torch.randperm(n + 2, generator=torch.Generator().manual_seed(seed))[:n]
    kept = torch.full((n + 2, heads, dk, dv), 5.0, device="cuda")
    given, keep, state_index = first.cuda(), kept, index.int().cuda()
    if states == "none":
        given = keep = state_index = None
    elif states == "in place":
        kept = keep = given
    elif states == "by number":
        state_index, index = None, torch.arange(n)
    out = torch.full((tokens, heads, dv), 9.0, dtype=dtype, device="cuda")
    args = dict(scale=scale, state_in=given, state_out=keep, state_index=state_index, out=out)
    if step:
        B.mmv_decay_step(q.cuda(), k.cuda(), v.cuda(), ld.cuda(), args.pop("state_in"), args.pop("state_out"), **args)
    else:
        B.mmv_decay_attention(q.cuda(), k.cuda(), v.cuda(), ints(ends), ld.cuda(), **args)
    want, final, by, final_by = plain_decay(q, k, v, ends, ld.clamp(min=-1e30), scale, None if given is None else first[index])
    check(out[before:tokens - after], want[before:tokens - after], by[before:tokens - after], "out")
    assert bool((out[:before] == 9).all() and (out[tokens - after:] == 9).all())
    if given is not None:
        check(kept.cpu()[index], final, final_by, "states")
        rest = torch.ones(n + 2, dtype=torch.bool)
        rest[index] = False
        assert torch.equal(kept.cpu()[rest], first[rest] if states == "in place" else torch.full_like(first[rest], 5.0))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("heads,group,dk,dv", [(1, 1, 8, 8), (2, 1, 64, 64), (4, 2, 80, 112), (2, 2, 128, 128), (4, 4, 24, 160), (2, 1, 128, 256), (3, 1, 96, 40)])
def test_decay_over_ragged_prompts(heads, group, dk, dv, dtype):
    run_decay([0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300], heads, group, dk, dv, dtype)


@pytest.mark.parametrize("kind", ["none", "hard"])
@pytest.mark.parametrize("states", ["none", "in place", "by number"])
def test_decay_with_and_without_states(kind, states):
    run_decay([70, 0, 1, 130], 4, 2, 64, 64, BF16, kind, states)
    run_decay([70, 0, 1, 130], 4, 1, 128, 128, F16, kind, states, before=3, after=2)


@pytest.mark.parametrize("lengths", [[2500], [1025, 3, 1023], [1] * 300, [0, 0, 700, 0], []])
def test_decay_over_long_and_many_prompts(lengths):
    run_decay(lengths, 2, 1, 64, 64, BF16, seed=9)
    run_decay(lengths, 4, 1, 16, 16, BF16, "hard", "in place", seed=10)
    run_decay(lengths, 2, 2, 128, 96, BF16, "none", seed=11)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n,heads,group,dk,dv", [(1, 1, 1, 8, 8), (4, 8, 1, 64, 64), (33, 4, 4, 80, 112), (5, 2, 1, 128, 256), (130, 2, 2, 128, 128), (3, 1, 1, 120, 72), (2, 3, 3, 72, 160)])
def test_decay_step(n, heads, group, dk, dv, dtype):
    for states in ("both", "in place", "by number", "none"):
        run_decay([1] * n, heads, group, dk, dv, dtype, states=states, step=True)
    run_decay([1] * n, heads, group, dk, dv, dtype, "hard", step=True)


def test_decay_leaves_out_what_has_no_place():
    """Indices outside the states, offsets beyond the tokens or backwards."""
    heads, dk, dv = 2, 64, 64
    q, k, v = (normal(i, 100, heads, 64) for i in range(3))
    ld, first = decays(heads), normal(4, 2, heads, dk, dv, dtype=torch.float32)
    want, final, by, final_by = plain_decay(q, k, v, [0, 30, 100], ld, 1.0, [torch.zeros(heads, dk, dv), first[1]])
    state = first.cuda()
    out = B.mmv_decay_attention(q.cuda(), k.cuda(), v.cuda(), ints([-4, 30, 2 ** 31 - 1, 50]), ld.cuda(), scale=1.0, state_in=state, state_out=state,
                                state_index=ints([-1, 1, 2]))
    check(out, want, by, "out")
    check(state[1], final[1], final_by[1], "state")
    assert torch.equal(state[0].cpu(), first[0])
    out = B.mmv_decay_step(q[:3].cuda(), k[:3].cuda(), v[:3].cuda(), ld.cuda(), state, state, scale=1.0, state_index=ints([7, -1, 2 ** 30]))
    want, _, by, _ = plain_decay(q[:3], k[:3], v[:3], [0, 1, 2, 3], ld, 1.0)
    check(out, want, by, "step")
    assert torch.equal(state[0].cpu(), first[0])


@pytest.mark.parametrize("step", [False, True])
def test_decay_keeps_what_is_not_finite_in_its_request_and_head(step):
    lengths, heads, dk, dv = [1] * 4 if step else [40, 90, 5], 2, 64, 64
    tokens, n = sum(lengths), len(lengths)
    q, k, v = (normal(i, tokens, heads, 64) for i in range(3))
    bad = lengths[0] + (0 if step else 33)
    v[bad, 1, 7] = NAN
    ends = [sum(lengths[:i]) for i in range(n + 1)]
    state = torch.zeros(n, heads, dk, dv, device="cuda")
    if step:
        out = B.mmv_decay_step(q.cuda(), k.cuda(), v.cuda(), decays(heads).cuda(), state, state, scale=1.0)
    else:
        out = B.mmv_decay_attention(q.cuda(), k.cuda(), v.cuda(), ints(ends), decays(heads).cuda(), scale=1.0, state_out=state)
    want, final, by, final_by = plain_decay(q, k, v, ends, decays(heads), 1.0)
    nan = torch.isnan(want)
    assert bool(nan[bad, 1, 7]) and torch.equal(torch.isnan(out.cpu())[:, :, :7], nan[:, :, :7]) and bool(torch.isnan(out.cpu()[bad:ends[2], 1, 7]).all())
    assert not bool(torch.isnan(out.cpu()[:bad]).any()) and not bool(torch.isnan(out.cpu()[ends[2]:]).any())
    keep = ~nan & ~torch.isnan(by)
    check(out.cpu()[keep], want[keep], by[keep], "out")
    assert torch.equal(torch.isnan(state.cpu()), torch.isnan(final))


def test_decay_keeps_what_is_not_finite_however_fast_the_decay():
    """In a prompt of several blocks a NaN stays in the state as it does token by token, also where the decay since is zero in fp32."""
    lengths, heads, dk, dv = [900, 300], 4, 64, 64
    tokens, n = sum(lengths), len(lengths)
    q, k, v = (normal(i, tokens, heads, 64) for i in range(3))
    v[3, :, 7] = NAN
    k[910, 1, 5] = math.inf
    ld, ends = decays(heads, "hard"), [0, 900, 1200]
    state = torch.zeros(n, heads, dk, dv, device="cuda")
    out = B.mmv_decay_attention(q.cuda(), k.cuda(), v.cuda(), ints(ends), ld.cuda(), scale=1.0, state_out=state).cpu()
    assert bool(out[3:900, :, 7].isnan().all()) and bool(state[0, :, :, 7].isnan().all())
    assert not bool((~out[910:, 1].isfinite()).logical_not().any()) and not bool(state[1, 1, 5].isfinite().any())
    other = out.clone()
    other[3:900, :, 7], other[910:, 1] = 0, 0
    assert bool(other.isfinite().all())
    rest = state.clone()
    rest[0, :, :, 7], rest[1, 1, 5] = 0, 0
    assert bool(rest.isfinite().all())


# ---- a step in a graph --------------------------------------------------------------------------------------------


def test_what_a_call_on_another_stream_allocates_is_that_streams(monkeypatch):
    """Scratch and results of a call with `stream`: allocated where its kernels run, and the same as on the current stream."""
    made, own = [], B.workspace
    monkeypatch.setattr(B, "workspace", lambda *a: made.append(torch.cuda.current_stream()) or own(*a))
    side = torch.cuda.Stream()
    n, heads, dim, page, width = 3, 2, 64, 16, 80
    table = torch.randperm(n * width, generator=torch.Generator().manual_seed(3), dtype=torch.int64).to(torch.int32).view(n, width).cuda()
    cache = B.PagedCache(*(normal(i, n * width, heads, page, dim).cuda() for i in (1, 2)))
    q, k, v = (normal(i, 900, heads, dim).cuda() for i in (3, 4, 5))
    context, offsets, ld = ints([1200, 3, 700]), ints([0, 400, 400, 900]), decays(heads).cuda()
    many = 4000
    cached, new, free, pages = ints([5] * many), ints([1] * many), ints([]), ints(list(range(many)))[:, None]
    side.wait_stream(torch.cuda.current_stream())
    for call in (lambda **s: B.mmv_paged_attention(q[:n], cache, table, context, **s), lambda **s: B.mmv_decay_attention(q, k, v, offsets, ld, **s),
                 lambda **s: B.mmv_decay_step(q[:n], k[:n], v[:n], ld, **s),
                 lambda **s: B.mmv_page_tables(cached, new, free, pages, page, many, **s).slots):
        here = call()
        torch.cuda.synchronize()
        made.clear()
        there = call(stream=side)
        assert all(s == side for s in made)
        side.synchronize()
        assert torch.equal(here, there)
    assert made


def test_a_captured_step_follows_its_lengths():
    """Tables, append, attention and the single-token recurrence in one graph, replayed as the requests grow; eager work in between."""
    n, heads, group, dim, page, width = 5, 2, 4, 64, 16, 8
    cached = [0, 15, 16, 40, 100]
    pages = n * width
    ids = list(range(pages))
    random.Random(1).shuffle(ids)
    table = [(ids[r * width:r * width + -(-c // page)] + [-1] * width)[:width] for r, c in enumerate(cached)]
    free = [i for i in ids if not any(i in row for row in table)]
    cache, kc, vc = cache_pair(31, pages, heads, page, dim, BF16)
    q, k, v = normal(41, 3, n, heads * group, dim), normal(42, 3, n, heads, dim), normal(43, 3, n, heads, dim)
    state, ld = torch.zeros(n, heads * group, dim, dim, device="cuda"), decays(heads * group)
    d = dict(cached=ints(cached), new=ints([1] * n), free=ints(free), table=ints(table), q=q[0].cuda(), k=k[0].cuda(), v=v[0].cuda(), ld=ld.cuda())
    ws = B.workspace(max(B.mmv_page_tables_workspace_bytes(n), B.mmv_paged_attention_workspace_bytes(n, heads * group, heads, dim, width * page)))
    out, mixed = torch.empty_like(d["q"]), torch.empty_like(d["q"])
    tables = B.mmv_page_tables(d["cached"], d["new"], d["free"], d["table"].clone(), page, n)

    def step():
        B.mmv_page_tables(d["cached"], d["new"], d["free"], d["table"], page, n, out=tables, ws=ws)
        B.mmv_cache_append(d["k"], d["v"], tables.slots, cache)
        B.mmv_paged_attention(d["q"], cache, d["table"], tables.context, out=out, ws=ws)
        B.mmv_decay_step(d["q"], d["k"], d["v"], d["ld"], state, state, out=mixed)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    S = torch.zeros(n, heads * group, dim, dim, dtype=torch.float64)
    for i in range(3):
        for name, x in (("q", q), ("k", k), ("v", v)):
            d[name].copy_(x[i])
        graph.replay()
        torch.cuda.synchronize()
        plain = plain_tables(cached, [1] * n, free, table, page, n)
        assert tables.slots.tolist() == plain["slots"] and d["table"].tolist() == plain["table"]
        for r, s in enumerate(plain["slots"]):
            kc[s // page, :, s % page], vc[s // page, :, s % page] = k[i, r], v[i, r]
        table, cached, free = plain["table"], plain["context"], free[plain["used"][0]:]
        want, _, by, _ = plain_attention(q[i], kc, vc, table, cached, dim ** -0.5, 0)
        check(out, want, by, "attention, replay %d" % i)
        want, S, by, by_state = plain_decay(q[i], k[i], v[i], list(range(n + 1)), ld, dim ** -0.5, S)
        check(mixed, want, by * (i + 1), "recurrence, replay %d" % i)
        S = state.cpu().double()
        d["cached"].copy_(ints(cached))
        d["free"][:len(free)] = ints(free)
        run_attention(cache, kc, vc, table, q[i], cached)   # eager work between the replays
        torch.cuda.synchronize()


@pytest.mark.parametrize("native", [True, False])
def test_the_calls_give_the_same_through_either_marshalling(native, monkeypatch):
    """With every argument given, so that the extension takes the calls; and without it.  What it does not take raises in Python."""
    B.load()
    assert B._marshal is not None
    if not native:
        monkeypatch.setattr(B, "_marshal", None)
    n, heads, dim, page = 3, 2, 64, 16
    contexts = [20, 0, 33]
    cache, kc, vc, table, q = attention_case(51, contexts, heads, 2, dim, page, F16, F16)
    tables = B.PageTables(torch.empty(4, dtype=torch.int32, device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda"), torch.empty(5, dtype=torch.int64, device="cuda"),
                          torch.empty(5, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int64, device="cuda"))
    ws = B.workspace(1 << 20)
    rows = ints(table)
    got = B.mmv_page_tables(ints(contexts), ints([1, 1, 0]), ints([1, 0]), rows, page, 5, out=tables, ws=ws)
    want = plain_tables(contexts, [1, 1, 0], [1, 0], table, page, 5)
    assert got is tables and rows.tolist() == want["table"]
    for name in ("offsets", "context", "slots", "positions", "used"):
        assert getattr(got, name).tolist() == want[name], name
    out, lse = torch.empty(n, 4, dim, dtype=F16, device="cuda"), torch.empty(n, 4, device="cuda")
    assert B.mmv_paged_attention(q.cuda(), cache, ints(table), ints(contexts), scale=0.1, window=0, out=out, lse=lse, ws=ws) is out
    want, want_lse, by, lse_by = plain_attention(q, kc, vc, table, contexts, 0.1, 0)
    check(out, want, by, "out")
    check(lse, want_lse, lse_by, "lse")
    with pytest.raises(B.MmvError):
        B.mmv_paged_attention(q.cuda(), cache, ints(table), ints(contexts), scale=0.1, out=out[:2], lse=lse, ws=ws)
    with pytest.raises(B.MmvError):
        B.mmv_paged_attention(q.cuda(), cache, ints(table), ints(contexts), scale=0.1, out=out, lse=lse, ws=ws[:256])
    with pytest.raises(B.MmvError):
        B.mmv_cache_append(q.cuda(), q.cuda(), ints([0, 1, 2], torch.int64), cache)   # (twice the heads)
    with pytest.raises(B.MmvError):
        B.mmv_page_tables(ints(contexts), ints([1, 1, 0]), ints([1, 0]), rows, page, 6, out=tables, ws=ws)


@pytest.mark.parametrize("columns", [0, 3000])   # a narrow table: a workgroup for a segment; a wide one: the list of tiles
@pytest.mark.parametrize("heads,group,dim,page,dtype,cache_type", [(2, 4, 128, 16, BF16, BF16), (1, 3, 72, 8, F16, F16), (2, 2, 64, 32, BF16, E4M3), (1, 8, 256, 8, BF16, BF16), (2, 1, 160, 24, F16, E4M3)])
def test_attention_does_not_use_what_is_left_out_in_either_form(columns, heads, group, dim, page, dtype, cache_type):
    """NaN in all that is not to be seen: behind the context, before the window, in pages of nobody and of rows that are not there."""
    contexts, window = [37, 5, 0, 129, 64, 200, 32, 1], 90
    cache, kc, vc, table, q = attention_case(8, contexts, heads, group, dim, page, dtype, cache_type)
    seen = {(table[r][p // page], p % page) for r, c in enumerate(contexts) for p in range(max(0, c - window), c)}
    for x, on_gpu in ((kc, cache.k), (vc, cache.v)):
        raw = x.view(torch.uint8) if cache_type == E4M3 else x
        for i in range(x.shape[0]):
            for s in range(page):
                if (i, s) not in seen:
                    raw[i, :, s] = 0x7F if cache_type == E4M3 else (NAN, math.inf, -math.inf)[(i + s) % 3]
        (on_gpu.view(torch.uint8) if cache_type == E4M3 else on_gpu).copy_(raw)
    table = [row + [-1] * columns for row in table]
    run_attention(cache, kc, vc, table, q, contexts, window=window, what="window")
    run_attention(cache, kc, vc, table, q, contexts, window=29, what="a narrower window")
    table[3][2], table[5][-1 - columns], table[4] = 10 ** 9, -7, [-1] * len(table[4])
    run_attention(cache, kc, vc, table, q, contexts, window=window, what="pages that are not there")
    contexts = [-1] * 8
    out = run_attention(cache, kc, vc, table, q, contexts)
    assert bool((out == 0).all())


def test_attention_over_a_cache_without_pages():
    k = torch.empty(0, 2, 16, 64, dtype=BF16, device="cuda")
    lse = torch.zeros(3, 4, device="cuda")
    out = B.mmv_paged_attention(torch.ones(3, 4, 64, dtype=BF16, device="cuda"), B.PagedCache(k, k.clone()), ints([[-1, 0], [1, 2], [5, -1]]), ints([5, 30, 0]), lse=lse)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
