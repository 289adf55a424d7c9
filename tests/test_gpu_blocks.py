"""A cache of 8-bit values with a scale for each block of slots and head: written, read back, and attended to, against the plain forms (tests/block_util.py)."""
import math
import random

import pytest
import torch

from block_util import MOST, plain_append, plain_read, values_of
from paper_2506_23906_amd import binding as B
from serving_util import EPS, U, check, plain_attention, plain_tables

pytestmark = pytest.mark.gpu
BF16, F16, E4M3, INT8 = torch.bfloat16, torch.float16, torch.float8_e4m3fn, torch.int8
NAN = float("nan")
TYPES = [(BF16, INT8), (F16, INT8), (BF16, E4M3), (F16, E4M3)]


def ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


def normal(seed, *shape, dtype=BF16, by=1.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * by).to(dtype)


def raw(x):
    return x.view(torch.uint8)


class Both:
    """A cache on the GPU and the same on the CPU (codes and scales of keys and of values)."""

    def __init__(self, seed, pages, heads, page, dim, block, kind, order="heads", scales=0.02):
        g = torch.Generator().manual_seed(seed)
        self.codes, self.scales, on_gpu = [], [], []
        for _ in "kv":
            x = torch.randint(0, 255, (pages, heads, page, dim), generator=g, dtype=torch.uint8)
            x = (x.int() - 127).to(torch.int8) if kind == INT8 else torch.where((x & 0x7F) == 0x7F, 0x11, x).to(torch.uint8).view(E4M3)
            self.codes.append(x)
            self.scales.append(scales * (0.25 + torch.rand(pages, heads, page // block, generator=g)))
            t = raw(x).cuda()
            if order == "slots":   # a page's slots lie before its heads
                t = t.transpose(1, 2).contiguous().transpose(1, 2)
            on_gpu.append(t.view(kind))
        self.cache = B.BlockCache(*on_gpu, *(s.cuda() for s in self.scales))
        self.block = block

    def append(self, k, v, slots, what=""):
        """On both; the same afterwards, bit for bit."""
        B.mmv_block_append(k.cuda() if not k.is_cuda else k, v.cuda() if not v.is_cuda else v, ints(slots, torch.int64), self.cache)
        for x, codes, scales, got, got_scales in zip((k, v), self.codes, self.scales, (self.cache.k, self.cache.v), (self.cache.k_scales, self.cache.v_scales)):
            plain_append(codes, scales, x.cpu(), slots, self.block)
            gs = got_scales.cpu()
            assert torch.equal(gs.view(torch.int32)[~scales.isnan()], scales.view(torch.int32)[~scales.isnan()]) and torch.equal(gs.isnan(), scales.isnan()), what + " scales"
            same = (raw(got.cpu().contiguous()) == raw(codes)) | (got.cpu().float().isnan() & codes.float().isnan())
            assert bool(same.all()), "%s: %d codes differ" % (what, int((~same).sum()))

    def values(self):
        return [values_of(c, s) for c, s in zip(self.codes, self.scales)]


# ---- writing and reading --------------------------------------------------------------------------------------------

SHAPES = [(1, 8, 8, 8, "heads"), (2, 72, 16, 8, "slots"), (8, 128, 16, 16, "heads"), (3, 160, 48, 24, "slots"), (2, 256, 64, 64, "heads"), (1, 64, 256, 128, "heads"), (5, 40, 32, 16, "heads")]


@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("heads,dim,page,block,order", SHAPES)
def test_append_in_steps(heads, dim, page, block, order, dtype, kind):
    """Requests that grow by one token, by a few and by many: blocks that begin, that go on, whose scale grows and does not."""
    print(heads, dim, page, block, order, dtype, kind, flush=True)
    n, width = 5, 2 + 150 // page
    both = Both(dim, n * width, heads, page, dim, block, kind, order)
    ids = list(range(n * width))
    random.Random(page).shuffle(ids)
    table, cached, free = [[-1] * width for _ in range(n)], [0] * n, ids
    for step, new in enumerate(([1, 0, 2, 17, 33], [1, 1, 1, 1, 1], [1, 1, 1, 1, 1], [3, 70, 1, 0, 9], [1, 1, 1, 1, 1])):
        plain = plain_tables(cached, new, free, table, page, sum(new) + 2)
        t = sum(new) + 2
        fused = normal(step, t, 3 * heads * dim, dtype=dtype, by=2.0 ** (step - 2))
        k, v = (fused[:, i * heads * dim:(i + 1) * heads * dim].unflatten(1, (heads, dim)) for i in (1, 2))
        on_gpu = fused.cuda()
        kg, vg = (on_gpu[:, i * heads * dim:(i + 1) * heads * dim].unflatten(1, (heads, dim)) for i in (1, 2))
        both.append(kg, vg, plain["slots"], "step %d" % step)
        table, cached, free = plain["table"], plain["context"], free[plain["used"][0]:]
    # everything read back, and the middle of every request
    for first, lengths in (([0] * n, cached), ([c // 3 for c in cached], [c - c // 3 for c in cached])):
        offsets = [2]
        for x in lengths:
            offsets.append(offsets[-1] + x)
        tokens = offsets[-1] + 3
        wide = torch.full((tokens, 2 * heads * dim + 16), 9.0, dtype=dtype, device="cuda")
        out = (wide[:, 8:8 + heads * dim].unflatten(1, (heads, dim)), wide[:, 16 + heads * dim - 8:16 + 2 * heads * dim - 8].unflatten(1, (heads, dim)))
        B.mmv_block_read(both.cache, ints(table), ints(offsets), first=ints(first), out=out)
        for got, values in zip(out, both.values()):
            assert torch.equal(got.cpu(), plain_read(values, table, offsets, first, tokens, dtype, 9.0))
        assert bool((wide[:, :8] == 9).all() and (wide[:, -8:] == 9).all())


@pytest.mark.parametrize("kind", [INT8, E4M3])
def test_what_is_held_is_within_half_a_step(kind):
    """Against the values themselves, without the definition's roundings: half a step of 8 bits (e4m3: 2^-4 of the value, or half of its least step of 2^-9).  What is rounded to 8 bits has been
    rounded to 32 three times (the scale, its reciprocal, the product), 2^-24 of up to Q steps each, and so has the scale that the code is multiplied with: 4 Q 2^-24 steps."""
    both = Both(1, 4, 2, 32, 64, 16, kind)
    k, v = normal(1, 128, 2, 64), normal(2, 128, 2, 64, by=1e-3)
    both.append(k, v, list(range(128)))
    for x, values, scales in zip((k, v), both.values(), both.scales):
        x = x.double().unflatten(0, (4, 32)).transpose(1, 2)
        step = scales.double().repeat_interleave(16, 2)[..., None]
        by = step / 2 if kind == INT8 else torch.maximum(2.0 ** -4 * x.abs(), 2.0 ** -10 * step)
        assert bool(((values - x).abs() <= by + 4 * MOST[kind] * EPS * step).all())


@pytest.mark.parametrize("dtype,kind", TYPES)
def test_append_of_runs_of_any_length_and_order(dtype, kind):
    """Slots out of order inside a block, the same slot twice with one value, runs longer than registers hold, slots that are none, and many tokens for the long windows."""
    page, block, heads, dim = 256, 256, 2, 128
    both = Both(3, 6, heads, page, dim, block, kind)
    slots = random.Random(2).sample(range(256, 512), 200) + [-1, 6 * 256, 2 ** 40, -2 ** 62] + list(range(512, 768)) + [1024 + 7]
    both.append(normal(4, len(slots), heads, dim, dtype=dtype), normal(5, len(slots), heads, dim, dtype=dtype), slots, "order")
    x = normal(6, 3, heads, dim, dtype=dtype)
    x = torch.cat([x, x[1:2], x[1:2]])
    both.append(x, x, [1030, 1031, 1040, 1031, 1031], "twice")
    tokens = 9000
    many = Both(4, tokens // 16 + 2, heads, 16, 32, 16, kind)
    slots = list(range(5, tokens + 5))
    for i in range(100, 200):
        slots[i] = -1
    many.append(normal(7, tokens, heads, 32, dtype=dtype), normal(8, tokens, heads, 32, dtype=dtype), slots, "many")
    out = B.mmv_block_read(many.cache, ints([list(range(tokens // 16 + 2))]), ints([0, tokens]), tokens, dtype)
    for got, values in zip(out, many.values()):
        assert torch.equal(got.cpu(), plain_read(values, [list(range(tokens // 16 + 2))], [0, tokens], [0], tokens, dtype, 0.0))


@pytest.mark.parametrize("dtype,kind", TYPES)
def test_append_of_values_that_are_not_ordinary(dtype, kind):
    """Zeros, the type's largest and least values, infinities, NaN; a block that begins anew forgets them."""
    both = Both(5, 3, 2, 16, 64, 8, kind)
    x = normal(9, 40, 2, 64, dtype=dtype)
    x[0:8] = 0.0
    x[8:16, 0] = torch.finfo(dtype).max
    x[8:16, 1] = torch.finfo(dtype).tiny
    x[17, 0, 3], x[20, 1, 5], x[25, 0, 0], x[26, 1, 63] = math.inf, -math.inf, NAN, -0.0
    x[33, 0, 7] = NAN
    both.append(x, x, list(range(40)), "first")
    if kind == INT8:
        assert bool(both.scales[0][1, 0, 1].isnan()) and not bool(both.scales[0][1, 1].isnan().any())
    else:
        assert bool(both.codes[0].float().isnan().any()) and not bool(both.scales[0].isnan().any())
    y = normal(10, 4, 2, 64, dtype=dtype)
    both.append(y, y, [41, 42, 28, 29], "goes on")
    both.append(y, y, [32, 33, 24, 25], "begins anew")
    assert not bool(both.scales[0].isnan().any())
    both.append(x[:0], x[:0], [], "nothing")


def test_scales_of_blocks_that_never_began():
    """Zeros, negative and infinite numbers, NaN in scales that a run in the middle of a block finds: no code is read as anything else than a code."""
    both = Both(6, 2, 1, 16, 64, 16, INT8)
    for s, gpu in zip(both.scales, (both.cache.k_scales, both.cache.v_scales)):
        s[0], s[1] = 0.0, NAN
        gpu.copy_(s)
    x = normal(11, 2, 1, 64)
    both.append(x, x, [3, 16 + 4], "middle")
    assert float(both.scales[0][0, 0, 0]) > 0 and bool(both.scales[0][1].isnan().all())


def test_read_leaves_out_what_has_no_place():
    both = Both(7, 4, 2, 16, 64, 8, INT8)
    table, offsets, first = [[2, -1, 9, 1], [-5, 0, 3, 2 ** 30], [1, 1, 1, 1]], [3, 70, 70, 135], [-3, 5, 60]
    out = tuple(torch.full((140, 2, 64), 5.0, dtype=BF16, device="cuda") for _ in "kv")
    B.mmv_block_read(both.cache, ints(table), ints(offsets), first=ints(first), out=out)
    for got, values in zip(out, both.values()):
        assert torch.equal(got.cpu(), plain_read(values, table, offsets, first, 140, BF16, 5.0))
    # offsets beyond the tokens, positions beyond 2^31
    out = B.mmv_block_read(both.cache, ints(table), ints([0, 50, 50, 2 ** 31 - 1]), 60, F16, first=ints([0, 0, 2 ** 31 - 1]))
    for got, values in zip(out, both.values()):
        assert torch.equal(got.cpu(), plain_read(values, table[:1], [0, 50], [0], 60, F16, 0.0))
    empty = B.BlockCache(*(torch.empty(0, 2, 16, 64, dtype=INT8, device="cuda") for _ in "kv"), *(torch.empty(0, 2, 2, device="cuda") for _ in "kv"))
    out = B.mmv_block_read(empty, ints([[0, 1]]), ints([0, 20]), 20)
    assert not bool(out[0].any()) and not bool(out[1].any())
    B.mmv_block_append(out[0], out[1], torch.arange(20, device="cuda"), empty)


# ---- attention ------------------------------------------------------------------------------------------------------


def attention_case(seed, contexts, heads, group, dim, page, block, dtype, kind, order="heads", columns=0):
    rng, width = random.Random(seed), max(-(-max(contexts + [0]) // page) + 1 + columns, 1)
    counts = [-(-max(c, 0) // page) for c in contexts]
    ids = list(range(sum(counts) + 2))
    rng.shuffle(ids)
    table, at = [], 0
    for c in counts:
        table.append((ids[at:at + c] + [-1] * width)[:width])
        at += c
    return Both(seed, len(ids), heads, page, dim, block, kind, order, 0.02), table, normal(seed + 1, len(contexts), heads * group, dim, dtype=dtype, by=1.5)


def run_attention(both, table, q, contexts, window=0, scale=None, what="", values=None):
    scale = q.shape[2] ** -0.5 if scale is None else scale
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    out = B.mmv_block_attention(q.cuda(), both.cache, ints(table), ints(contexts), scale=scale, window=window, lse=lse)
    k, v = both.values() if values is None else values
    want, want_lse, by, lse_by = plain_attention(q, k, v, table, contexts, scale, window)
    check(out, want, by, what + " out")
    check(lse, want_lse, lse_by, what + " lse")
    return out


@pytest.mark.parametrize("dtype,kind", TYPES)
@pytest.mark.parametrize("heads,group,dim,page,block,order", [(1, 1, 8, 8, 8, "heads"), (2, 1, 64, 16, 8, "heads"), (3, 5, 72, 8, 8, "slots"), (1, 16, 80, 24, 24, "heads"), (2, 4, 112, 32, 16, "slots"),
                                                              (8, 4, 128, 16, 16, "heads"), (1, 7, 136, 128, 64, "heads"), (2, 8, 160, 64, 64, "slots"), (1, 2, 192, 40, 8, "heads"),
                                                              (2, 3, 256, 48, 24, "heads"), (2, 2, 32, 64, 8, "heads"), (1, 3, 96, 72, 24, "heads")])
def test_attention_at_ragged_lengths(heads, group, dim, page, block, order, dtype, kind):
    contexts = [0, 1, 2, 7, 8, 9, 31, 32, 33, 63, 64, 65, 100, 257, 700]
    random.Random(dim).shuffle(contexts)
    print(heads, group, dim, page, block, order, dtype, kind, flush=True)
    run_attention(*attention_case(dim, contexts, heads, group, dim, page, block, dtype, kind, order), contexts)


@pytest.mark.parametrize("window", [1, 5, 32, 33, 100, 5000])
@pytest.mark.parametrize("dtype,kind", TYPES)
def test_attention_in_a_window(window, dtype, kind):
    contexts = [1, 33, 0, 100, 101, 640, 1500]
    run_attention(*attention_case(window, contexts, 2, 4, 128, 16, 8, dtype, kind), contexts, window=window)
    run_attention(*attention_case(window, contexts, 3, 1, 64, 64, 32, dtype, kind), contexts, window=window)


@pytest.mark.parametrize("n,hi,columns", [(1, 1, 0), (1, 20_000, 0), (3, 9000, 0), (70, 300, 0), (300, 40, 900), (1500, 9, 0)])
def test_attention_of_few_and_many_rows(n, hi, columns):
    rng = random.Random(n)
    contexts = [rng.randint(0, hi) if i else hi for i in range(n)]
    for dtype, kind in ((BF16, INT8), (F16, E4M3)):
        run_attention(*attention_case(n, contexts, 2, 2, 64, 16, 16, dtype, kind, columns=columns), contexts, what=str(n))


@pytest.mark.parametrize("columns", [0, 3000])   # a workgroup for a segment; the list of tiles
@pytest.mark.parametrize("heads,group,dim,page,block,dtype,kind", [(2, 4, 128, 16, 16, BF16, INT8), (1, 3, 72, 8, 8, F16, INT8), (2, 2, 64, 32, 8, BF16, E4M3), (1, 8, 256, 64, 8, F16, E4M3)])
def test_attention_does_not_use_what_is_left_out(columns, heads, group, dim, page, block, dtype, kind):
    """NaN codes and scales (and infinite ones) behind the context, before the window and in pages of nobody; pages that are not there."""
    contexts, window = [37, 5, 0, 129, 64, 200, 32, 1], 90
    both, table, q = attention_case(8, contexts, heads, group, dim, page, block, dtype, kind, columns=columns)
    want = [x.clone() for x in both.values()]
    seen = {(table[r][p // page], p % page) for r, c in enumerate(contexts) for p in range(max(0, c - window), c)}
    blocks = {(i, s // block) for i, s in seen}
    for codes, scales, gpu, gpu_scales in zip(both.codes, both.scales, (both.cache.k, both.cache.v), (both.cache.k_scales, both.cache.v_scales)):
        for i in range(codes.shape[0]):
            for s in range(page):
                if kind == E4M3 and (i, s) not in seen:
                    raw(codes)[i, :, s] = 0x7F
            for b in range(page // block):
                if (i, b) not in blocks:
                    scales[i, :, b] = (NAN, math.inf)[(i + b) % 2]
        raw(gpu).copy_(raw(codes))
        gpu_scales.copy_(scales)
    run_attention(both, table, q, contexts, window=window, what="window", values=want)
    run_attention(both, table, q, contexts, window=29, what="a narrower window", values=want)
    table[3][2], table[5][-1 - columns], table[4] = 10 ** 9, -7, [-1] * len(table[4])
    run_attention(both, table, q, contexts, window=window, what="pages that are not there", values=want)
    assert bool((run_attention(both, table, q, [-1] * 8, values=want) == 0).all())


@pytest.mark.parametrize("columns", [0, 900])
@pytest.mark.parametrize("dtype,kind", TYPES)
def test_scales_that_are_not_numbers_reach_their_rows_and_heads(columns, dtype, kind):
    contexts = [200, 190]
    both, table, q = attention_case(12, contexts, 2, 4, 64, 16, 8, dtype, kind, columns=columns)
    want, want_lse, by, lse_by = plain_attention(q, *both.values(), table, contexts, 0.125, 0)
    both.cache.k_scales[table[0][3], 1, 1] = NAN
    both.cache.v_scales[table[1][2], 0, 0] = NAN
    lse = torch.empty(2, 8, device="cuda")
    out = B.mmv_block_attention(q.cuda(), both.cache, ints(table), ints(contexts), scale=0.125, lse=lse).cpu()
    bad, bad_lse = torch.zeros(2, 8, dtype=torch.bool), torch.zeros(2, 8, dtype=torch.bool)
    bad[0, 4:] = bad[1, :4] = bad_lse[0, 4:] = True
    assert bool(out[bad].isnan().all()) and bool(lse.cpu()[bad_lse].isnan().all())
    check(out[~bad], want[~bad], by[~bad], "the other heads")
    check(lse.cpu()[~bad_lse], want_lse[~bad_lse], lse_by[~bad_lse], "their lse")


@pytest.mark.parametrize("columns", [4, 900])
@pytest.mark.parametrize("dtype,kind", TYPES)
def test_probabilities_of_24_bits_whatever_the_scales(columns, dtype, kind):
    """Seven positions whose weights times values cancel to 3e-6 of what they add up: a block of one position of value 193/64 and blocks of -1, each as a code and a scale of its own, large and
    small ones.  Without the third term of a probability, or with scales in the result's type, what is left would be 2^-17 of the sum off."""
    p = 0.5 * (1.0 + (171 / 128 - 0.95 * 2.0 ** -8) * 2.0 ** -8)
    for size in (1.0, 2.0 ** -40, 2.0 ** 60):
        if dtype == F16 and size == 2.0 ** 60:
            continue
        q, k, v = torch.zeros(1, 1, 64), torch.zeros(7, 1, 8, 64), torch.zeros(7, 1, 8, 64)
        ks, vs = torch.ones(7, 1, 1), torch.ones(7, 1, 1)
        q[..., 0], k[1:7, 0, 0, 0] = 1.0, -1.0
        # values: the first 193/64 = 96.5 / 32, as the code 96 or 88 and a scale; the others -1 = -64 / 64
        first = 96.0 if kind == INT8 else 88.0
        v[0, 0, 0], vs[0] = first, 193 / 64 / first * size
        v[1:7, 0, 0], vs[1:7] = -64.0, size / 64
        scale = float(torch.tensor(-math.log(p), dtype=torch.float32))
        cache = B.BlockCache(k.to(kind).cuda(), v.to(kind).cuda(), ks.cuda(), vs.cuda())
        # one position of each page: a page's first slot alone counts, as rows of one position each would; here contexts end in every page, so weights of the other slots must be none
        k[:, 0, 1:, 0], ks = -127.0 if kind == INT8 else -448.0, ks
        cache.k.copy_(k.to(kind))
        lse = torch.empty(1, 1, device="cuda")
        out = B.mmv_block_attention(q.to(dtype).cuda(), cache, ints([[0, 1, 2, 3, 4, 5, 6] + [-1] * (columns - 4)]), ints([56]), scale=scale, lse=lse).cpu()
        weights = torch.exp(-scale * torch.cat([-k.double()[:, 0, :, 0].flatten()]))
        values = (v.to(kind).double() * vs.double()[..., None])[:, 0, :, 0].flatten()
        want, total = float(weights @ values / weights.sum()), float(weights @ values.abs() / weights.sum())
        by = (2.0 ** -24 + 2.0 ** -29 + (56 + 12) * EPS) * total + U[dtype] * abs(want) + (2.0 ** -25 if dtype == F16 else 0.0)
        assert float((out.double() - want).abs().max()) <= by, (size, float(out[0, 0, 0]), want, by)


def test_far_pages_and_far_slots():
    """Codes beyond 2^32, scales beyond 2^31 of them are not needed: pages at the end of a cache of 5 GB; slots that lie far apart."""
    heads, page, dim, pages = 2, 64, 128, 320_000
    k, v = (torch.zeros(pages, heads, page, dim, dtype=INT8, device="cuda") for _ in "kv")
    ks, vs = (torch.zeros(pages, heads, 8, device="cuda") for _ in "kv")
    cache, contexts = B.BlockCache(k, v, ks, vs), [100, 64]
    table = [[pages - 1, pages - 3], [pages - 2, -1]]
    new_k, new_v = normal(1, 164, heads, dim), normal(2, 164, heads, dim)
    slots = [table[0][i // page] * page + i % page for i in range(100)] + [table[1][0] * page + i for i in range(64)]
    B.mmv_block_append(new_k.cuda(), new_v.cuda(), ints(slots, torch.int64), cache)
    small = [torch.zeros(4, heads, page, dim, dtype=INT8) for _ in "kv"]
    scales = [torch.zeros(4, heads, 8) for _ in "kv"]
    for x, c, s, got, got_s in zip((new_k, new_v), small, scales, (k, v), (ks, vs)):
        plain_append(c, s, x, [slot - (pages - 4) * page for slot in slots], 8)
        assert torch.equal(got[-4:].cpu(), c) and torch.equal(got_s[-4:].cpu(), s) and not bool(got_s[:-4].any())
    q = normal(3, 2, 2 * heads, dim)
    out = B.mmv_block_attention(q.cuda(), cache, ints(table), ints(contexts))
    values = [values_of(c, s) for c, s in zip(small, scales)]
    want, _, by, _ = plain_attention(q, *values, [[3, 1], [2, -1]], contexts, dim ** -0.5, 0)
    check(out, want, by, "far pages")
    got = B.mmv_block_read(cache, ints(table), ints([0, 100, 164]), 164)
    for g, x in zip(got, values):
        assert torch.equal(g.cpu(), plain_read(x, [[3, 1], [2, -1]], [0, 100, 164], [0, 0], 164, BF16, 0.0))
    del k, v, cache
    page, pages = 32, 2_900_000
    k, v = (torch.empty(page, pages, 1, 64, dtype=INT8, device="cuda").permute(1, 2, 0, 3) for _ in "kv")
    ks, vs = (torch.zeros(pages, 1, 1, device="cuda") for _ in "kv")
    cache, table = B.BlockCache(k, v, ks, vs), [[pages - 1, 7, pages - 2]]
    new_k, new_v = normal(4, 75, 1, 64), normal(5, 75, 1, 64)
    B.mmv_block_append(new_k.cuda(), new_v.cuda(), ints([table[0][i // page] * page + i % page for i in range(75)], torch.int64), cache)
    small, scales = [torch.zeros(3, 1, page, 64, dtype=INT8) for _ in "kv"], [torch.zeros(3, 1, 1) for _ in "kv"]
    for x, c, s in zip((new_k, new_v), small, scales):
        plain_append(c, s, x, list(range(75)), 32)
    values = [values_of(c, s) for c, s in zip(small, scales)]
    q = normal(6, 1, 4, 64)
    want, _, by, _ = plain_attention(q, *values, [[0, 1, 2]], [75], 0.125, 0)
    check(B.mmv_block_attention(q.cuda(), cache, ints(table), ints([75])), want, by, "far slots")


def test_streams_views_and_marshalling(monkeypatch):
    """Calls on another stream allocate there and give the same; queries and outputs that are views; with and without the extension."""
    contexts, n = [300, 17, 64], 3
    both, table, q = attention_case(21, contexts, 2, 4, 80, 16, 8, F16, INT8)
    made, own = [], B.workspace
    monkeypatch.setattr(B, "workspace", lambda *a: made.append(torch.cuda.current_stream()) or own(*a))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    fused = torch.full((3, 8 * 80 + 96), NAN, dtype=F16, device="cuda")
    fused[:, 48:48 + 640] = q.flatten(1).cuda()
    view = fused[:, 48:688].unflatten(1, (8, 80))
    wide = torch.full((5, len(table[0]) + 9), 10 ** 9, dtype=torch.int32, device="cuda")
    wide[:3, :len(table[0])] = ints(table)
    context, offsets = ints(contexts), ints([0, 300, 317, 381])
    torch.cuda.synchronize()
    for call in (lambda **s: B.mmv_block_attention(view, both.cache, wide, context, **s), lambda **s: B.mmv_block_read(both.cache, wide, offsets, 381, F16, **s)[1]):
        here = call()
        torch.cuda.synchronize()
        made.clear()
        there = call(stream=side)
        assert all(s == side for s in made)
        side.synchronize()
        assert torch.equal(here, there)
    want, want_lse, by, lse_by = plain_attention(q, *both.values(), table, contexts, 0.1, 0)
    x = normal(30, 4, 2, 80, dtype=F16)
    for native in (True, False):
        if not native:
            monkeypatch.setattr(B, "_marshal", None)
        out, lse, ws = torch.empty(n, 8, 80, dtype=F16, device="cuda"), torch.empty(n, 8, device="cuda"), own(1 << 20)
        assert B.mmv_block_attention(view, both.cache, wide, context, scale=0.1, window=0, out=out, lse=lse, ws=ws) is out
        check(out, want, by, "out")
        check(lse, want_lse, lse_by, "lse")
        out = (torch.empty(381, 2, 80, dtype=F16, device="cuda"), torch.empty(381, 2, 80, dtype=F16, device="cuda"))
        assert B.mmv_block_read(both.cache, wide, offsets, first=None, out=out) is out
        for got, values in zip(out, both.values()):
            assert torch.equal(got.cpu(), plain_read(values, table, [0, 300, 317, 381], [0] * 3, 381, F16, 0.0))
        both.append(x, x, [3, 4, 5, 6], "native" if native else "python")
        want, want_lse, by, lse_by = plain_attention(q, *both.values(), table, contexts, 0.1, 0)
        for wrong in (lambda: B.mmv_block_attention(view, both.cache, wide, context, scale=0.1, out=torch.empty(2, 8, 80, dtype=F16, device="cuda"), ws=ws),
                      lambda: B.mmv_block_attention(view, both.cache, wide, context, scale=0.1, lse=lse, ws=ws[:256]),
                      lambda: B.mmv_block_attention(view, B.PagedCache(both.cache.k.view(E4M3), both.cache.v.view(E4M3)), wide, context),
                      lambda: B.mmv_block_append(view, view, ints([0, 1, 2], torch.int64), both.cache), lambda: B.mmv_block_read(both.cache, wide, offsets),
                      lambda: B.mmv_block_read(both.cache, wide, offsets, out=(out[0], out[1][:300]))):
            with pytest.raises(B.MmvError):
                wrong()
