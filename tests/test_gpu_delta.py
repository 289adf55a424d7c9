"""The gated delta rule over prompts and for single tokens, against its plain form (tests/block_util.py)."""
import math

import pytest
import torch

from block_util import plain_delta
from paper_2506_23906_amd import binding as B
from serving_util import EPS, U, check

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16
NAN = float("nan")


def ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


def normal(seed, *shape, dtype=BF16, by=1.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * by).to(dtype)


def unit(x, dtype):
    return (x.float() / x.float().norm(dim=-1, keepdim=True).clamp(min=1e-6)).to(dtype)


def gates(seed, tokens, heads, kind="spread"):
    """log_decay and beta of every token and head."""
    g = torch.Generator().manual_seed(seed)
    if kind == "none":
        return torch.zeros(tokens, heads), torch.full((tokens, heads), 0.5)
    if kind == "hard":   # decays that end a state, next to none; what is written whole, not at all, twice
        some = torch.tensor([-40.0, -math.inf, -3.0, 0.0, -1e-3, -250.0])[torch.randint(6, (tokens, heads), generator=g)]
        return torch.where(torch.rand(tokens, heads, generator=g) < 0.2, some, -1e-2 * torch.rand(tokens, heads, generator=g)), torch.tensor([1.0, 0.0, 1.9, 0.3])[
            torch.randint(4, (tokens, heads), generator=g)]
    return -torch.exp(torch.randn(tokens, heads, generator=g) - 3.0), torch.rand(tokens, heads, generator=g)


def inputs(seed, tokens, heads, group, dk, dv, dtype, alike=0.0):
    """Keys of length 1; alike: so much of one direction that they have in common."""
    shared = heads // group
    common = normal(seed + 7, 1, shared, dk, dtype=torch.float32)
    q, k = (unit(normal(seed + i, tokens, shared, dk, dtype=torch.float32) + alike * common, dtype) for i in (0, 1))
    return q, k, normal(seed + 2, tokens, heads, dv, dtype=dtype)


def run_delta(lengths, heads, group, dk, dv, dtype, kind="spread", states="both", step=False, seed=0, before=0, after=0, alike=0.0):
    print(lengths[:20], heads, group, dk, dv, dtype, kind, states, step, flush=True)
    n, tokens = len(lengths), sum(lengths) + before + after
    q, k, v = inputs(seed, tokens, heads, group, dk, dv, dtype, alike)
    ld, beta = gates(seed + 3, tokens, heads, kind)
    ends = [before]
    for x in lengths:
        ends.append(ends[-1] + x)
    scale = dk ** -0.5
    first = normal(seed + 4, n + 2, heads, dk, dv, dtype=torch.float32)
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
        B.mmv_delta_step(q.cuda(), k.cuda(), v.cuda(), ld.cuda(), beta.cuda(), **args)
    else:
        B.mmv_delta_attention(q.cuda(), k.cuda(), v.cuda(), ints(ends), ld.cuda(), beta.cuda(), **args)
    want, final, by, final_by = plain_delta(q, k, v, ends, ld, beta, scale, None if given is None else first[index])
    check(out[before:tokens - after], want[before:tokens - after], by[before:tokens - after], "out")
    assert bool((out[:before] == 9).all() and (out[tokens - after:] == 9).all())
    if given is not None:
        check(kept.cpu()[index], final, final_by, "states")
        rest = torch.ones(n + 2, dtype=torch.bool)
        rest[index] = False
        assert torch.equal(kept.cpu()[rest], first[rest] if states == "in place" else torch.full_like(first[rest], 5.0))


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("heads,group,dk,dv", [(1, 1, 8, 8), (2, 1, 64, 64), (4, 2, 80, 112), (2, 2, 128, 128), (4, 4, 24, 160), (2, 1, 128, 256), (3, 1, 96, 40), (2, 1, 112, 192)])
def test_ragged_prompts(heads, group, dk, dv, dtype):
    run_delta([0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300], heads, group, dk, dv, dtype)


@pytest.mark.parametrize("kind", ["none", "hard"])
@pytest.mark.parametrize("states", ["none", "in place", "by number"])
def test_with_and_without_states(kind, states):
    run_delta([70, 0, 1, 130], 4, 2, 64, 64, BF16, kind, states)
    run_delta([70, 0, 1, 130], 4, 1, 128, 128, F16, kind, states, before=3, after=2)


@pytest.mark.parametrize("lengths", [[2500], [1025, 3, 1023], [1] * 300, [0, 0, 700, 0], []])
def test_long_and_many_prompts(lengths):
    run_delta(lengths, 2, 1, 64, 64, BF16, seed=9)
    run_delta(lengths, 4, 1, 16, 16, BF16, "hard", "in place", seed=10)
    run_delta(lengths, 2, 2, 128, 96, BF16, "none", seed=11)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("alike", [0.3, 30.0])
def test_keys_that_are_alike(alike, dtype):
    """What tokens write then depends on each other the most: the triangular systems are far from the identity."""
    run_delta([64, 200, 33], 2, 1, 64, 64, dtype, "none", alike=alike)
    run_delta([64, 200, 33], 4, 2, 128, 128, dtype, "hard", "in place", alike=alike)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n,heads,group,dk,dv", [(1, 1, 1, 8, 8), (4, 8, 1, 64, 64), (33, 4, 4, 80, 112), (5, 2, 1, 128, 256), (130, 2, 2, 128, 128), (3, 1, 1, 120, 72), (2, 3, 3, 72, 160), (3, 2, 1, 128, 136)])
def test_step(n, heads, group, dk, dv, dtype):
    for states in ("both", "in place", "by number", "none"):
        run_delta([1] * n, heads, group, dk, dv, dtype, states=states, step=True)
    run_delta([1] * n, heads, group, dk, dv, dtype, "hard", step=True)


def one_hot(tokens, dk, dv, dtype, seed):
    """Every token's key is one component; its value is written there, over what was there before."""
    at = torch.randint(dk, (tokens,), generator=torch.Generator().manual_seed(seed))
    k = torch.zeros(tokens, 1, dk)
    k[torch.arange(tokens), 0, at] = 1.0
    return at, k.to(dtype), normal(seed + 1, tokens, 1, dv, dtype=dtype)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("tokens", [1, 40, 64, 300, 1500])
def test_states_hold_32_bits(tokens, dtype):
    """With keys of one component a row of the state is (1 - beta) times what was there plus beta times a value, decayed: a few roundings of 32 bits for each token that wrote there and for each
    chunk, and none of 16 or fewer.  (Per token that wrote: beta times a value and its difference to what was there, terms of 24 bits of both, 16 roundings of 2^-24; the decay since, at most
    e^-30 in all, in 40 chunks or blocks at most, whose exponents are rounded to 2^-24 of 30: 30 + 40 * 8.)"""
    dk, dv = 32, 32
    at, k, v = one_hot(tokens, dk, dv, dtype, 5)
    g, beta = -torch.rand(tokens, 1, generator=torch.Generator().manual_seed(6)) * (20.0 / max(tokens, 20)), 0.25 + 0.7 * torch.rand(tokens, 1, generator=torch.Generator().manual_seed(7))
    first = normal(8, 1, 1, dk, dv, dtype=torch.float32)
    state = first.cuda()
    B.mmv_delta_attention(k.cuda(), k.cuda(), v.cuda(), ints([0, tokens]), g.cuda(), beta.cuda(), scale=1.0, state_in=state, state_out=state)
    S, A = first[0, 0].double(), first[0, 0].double().abs()
    writes = torch.zeros(dk, 1, dtype=torch.float64)
    for t in range(tokens):
        by, b = math.exp(float(g[t])), float(beta[t])
        S, A = S * by, A * by
        S[at[t]] += b * (v[t, 0].double() - S[at[t]])
        A[at[t]] = (1 - b) * A[at[t]] + b * v[t, 0].double().abs()   # (what is added up)
        writes[at[t]] += 1
    off = (state.cpu()[0, 0].double() - S).abs()
    by = EPS * (16 * (writes + 1) + 30 + 8 * 40) * A
    assert bool((off <= by).all()), float((off / by).max())
    # (what a missing third term would be: 2^-17 of a value that was written, against at most 2^-24 * 400 = 2^-15.4 of all that a row has seen: so the mean has to be small, too)
    assert float(off.norm() / S.norm()) <= 8 * EPS * math.sqrt(float(writes.max()) + 2)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("tokens", [64, 640])
def test_decay_over_everything_is_exact_to_32_bits(tokens, dtype):
    """One key at the first token; the state is its value times the whole decay: also where decays are far from each other in size."""
    dk, dv = 16, 32
    k, v = torch.zeros(tokens, 1, dk), torch.zeros(tokens, 1, dv)
    k[0, 0, 5], v[0, 0] = 1.0, torch.linspace(1.0, 1.99, dv)
    k, v = k.to(dtype), v.to(dtype)
    g = torch.full((tokens, 1), -1e-3)
    g[3::7] = -2e-6
    g[20] = -9.0
    state = torch.zeros(1, 1, dk, dv, device="cuda")
    B.mmv_delta_attention(k.cuda(), k.cuda(), v.cuda(), ints([0, tokens]), g.cuda(), torch.ones(tokens, 1, device="cuda"), scale=1.0, state_out=state)
    want = v[0, 0].double() * math.exp(float(g[1:].double().sum()))
    # a token's decay is an exponential, off by at most its last bit (2 * 2^-24), and a product with it (2^-24): with the same decay for many tokens they all go one way
    assert bool(((state.cpu()[0, 0, 5].double() - want).abs() <= (3 * tokens + 64) * EPS * want).all())


def test_leaves_out_what_has_no_place():
    """Indices outside the states, offsets beyond the tokens or backwards."""
    heads, dk, dv = 2, 64, 64
    q, k, v = inputs(1, 100, heads, 1, dk, dv, BF16)
    ld, beta = gates(2, 100, heads)
    first = normal(4, 2, heads, dk, dv, dtype=torch.float32)
    want, final, by, final_by = plain_delta(q, k, v, [0, 30, 100], ld, beta, 1.0, [torch.zeros(heads, dk, dv), first[1]])
    state = first.cuda()
    out = B.mmv_delta_attention(q.cuda(), k.cuda(), v.cuda(), ints([-4, 30, 2 ** 31 - 1, 50]), ld.cuda(), beta.cuda(), scale=1.0, state_in=state, state_out=state, state_index=ints([-1, 1, 2]))
    check(out, want, by, "out")
    check(state[1], final[1], final_by[1], "state")
    assert torch.equal(state[0].cpu(), first[0])
    out = B.mmv_delta_step(q[:3].cuda(), k[:3].cuda(), v[:3].cuda(), ld[:3].cuda(), beta[:3].cuda(), state, state, scale=1.0, state_index=ints([7, -1, 2 ** 30]))
    want, _, by, _ = plain_delta(q[:3], k[:3], v[:3], [0, 1, 2, 3], ld, beta, 1.0)
    check(out, want, by, "step")
    assert torch.equal(state[0].cpu(), first[0])


@pytest.mark.parametrize("which", ["v", "k", "q", "log_decay", "beta", "state", "infinite v", "infinite k"])
@pytest.mark.parametrize("lengths,where", [([40, 90, 5], 73), ([10, 900, 300], 10 + 333), ([1, 1, 1, 1], 1)])
def test_what_is_not_finite_stays_in_its_request_and_head_and_behind_its_token(lengths, where, which):
    step = max(lengths) == 1
    heads, dk, dv, tokens, n = 2, 64, 64, sum(lengths), len(lengths)
    q, k, v = inputs(3, tokens, heads, 1, dk, dv, BF16)
    ld, beta = gates(4, tokens, heads)
    state = normal(5, n, heads, dk, dv, dtype=torch.float32)
    ends = [sum(lengths[:i]) for i in range(n + 1)]
    {"v": lambda: v.__setitem__((where, 1, 7), NAN), "k": lambda: k.__setitem__((where, 1, 9), NAN), "q": lambda: q.__setitem__((where, 1, 9), NAN),
     "log_decay": lambda: ld.__setitem__((where, 1), NAN), "beta": lambda: beta.__setitem__((where, 1), NAN), "state": lambda: state.__setitem__((1, 1, 3, 7), math.inf),
     "infinite v": lambda: v.__setitem__((where, 1, 7), -math.inf), "infinite k": lambda: k.__setitem__((where, 1, 9), math.inf)}[which]()
    on_gpu = state.cuda()
    args = (ld.cuda(), beta.cuda())
    if step:
        out = B.mmv_delta_step(q.cuda(), k.cuda(), v.cuda(), *args, on_gpu, on_gpu, scale=1.0)
    else:
        out = B.mmv_delta_attention(q.cuda(), k.cuda(), v.cuda(), ints(ends), *args, scale=1.0, state_in=on_gpu, state_out=on_gpu)
    out, on_gpu = out.cpu().double(), on_gpu.cpu().double()
    want, final, by, final_by = plain_delta(q, k, v, ends, ld, beta, 1.0, state)
    # where the recurrence in 64 bits is finite the result is, and within its bound; where it is not finite nothing finite comes out
    for got, ref, off in ((out, want, by), (on_gpu, final, final_by)):
        fine = ref.isfinite()
        assert torch.equal(fine, got.isfinite())
        keep = fine & off.isfinite()
        check(got[keep], ref[keep], off[keep], which)
    other = out.clone()
    other[ends[1]:ends[2], 1] = 0
    assert bool(other.isfinite().all()) and bool(out[:where if which != "state" else ends[1]].isfinite().all()) and not bool(on_gpu[1, 1].isfinite().all()) or which == "q"


def test_streams_views_and_marshalling(monkeypatch):
    heads, dk, dv, lengths = 4, 64, 64, [300, 0, 77]
    q, k, v = inputs(11, 377, heads, 2, dk, dv, BF16)
    ld, beta = gates(12, 377, heads)
    fused = torch.cat([q.flatten(1), k.flatten(1), v.flatten(1)], 1).cuda()
    views = (fused[:, :128].unflatten(1, (2, 64)), fused[:, 128:256].unflatten(1, (2, 64)), fused[:, 256:].unflatten(1, (4, 64)))
    ends, index = ints([0, 300, 300, 377]), ints([2, 0, 1])
    ldg, bg = ld.cuda(), beta.cuda()
    first = normal(13, 3, heads, dk, dv, dtype=torch.float32)
    want, final, by, final_by = plain_delta(q, k, v, [0, 300, 300, 377], ld, beta, 0.1, first[[2, 0, 1]])
    made, own = [], B.workspace
    monkeypatch.setattr(B, "workspace", lambda *a: made.append(torch.cuda.current_stream()) or own(*a))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    for call in (lambda **s: B.mmv_delta_attention(*views, ends, ldg, bg, scale=0.1, **s), lambda **s: B.mmv_delta_step(*(x[:3] for x in views), ldg[:3], bg[:3], scale=0.1, **s)):
        here = call()
        torch.cuda.synchronize()
        made.clear()
        there = call(stream=side)
        assert all(s == side for s in made)
        side.synchronize()
        assert torch.equal(here, there)
    for native in (True, False):
        if not native:
            monkeypatch.setattr(B, "_marshal", None)
        out, state, ws = torch.empty(377, heads, dv, dtype=BF16, device="cuda"), first.cuda(), own(B.mmv_delta_attention_workspace_bytes(3, 377, heads, dk, dv))
        assert B.mmv_delta_attention(*views, ends, ldg, bg, scale=0.1, state_in=state, state_out=state, state_index=index, out=out, ws=ws) is out
        check(out, want, by, "out")
        check(state[[2, 0, 1]], final, final_by, "states")
        few = torch.empty(3, heads, dv, dtype=BF16, device="cuda")
        kept = first.cuda()
        assert B.mmv_delta_step(*(x[:3] for x in views), ldg[:3], bg[:3], kept, kept, scale=0.1, state_index=index, out=few) is few
        ref, last, off, last_off = plain_delta(q[:3], k[:3], v[:3], [0, 1, 2, 3], ld, beta, 0.1, first[[2, 0, 1]])
        check(few, ref, off, "step")
        check(kept[[2, 0, 1]], last, last_off, "its states")
        for wrong in (lambda: B.mmv_delta_step(*views, ldg[:3], bg, kept, kept, scale=0.1), lambda: B.mmv_delta_step(*views, ldg, bg, kept[:, :2], None, scale=0.1),
                      lambda: B.mmv_delta_attention(views[0], views[2], views[2], ends, ldg, bg), lambda: B.mmv_delta_attention(*views, ends, ldg.bfloat16(), bg),
                      lambda: B.mmv_delta_attention(*views, ends, ldg, bg, state_in=state, state_out=state, out=out[:5])):
            with pytest.raises(B.MmvError):
                wrong()


LENGTHS = [(37 * i * i + 11 * i) % 110 for i in range(64)]


@pytest.mark.parametrize("heads,group,dk,dv,dtype", [(8, 2, 64, 128, BF16), (8, 1, 128, 128, BF16), (8, 4, 96, 256, F16), (8, 2, 128, 128, F16), (8, 8, 80, 112, BF16)])
def test_requests_that_fill_the_device(heads, group, dk, dv, dtype):
    """Workgroups of 128 columns; and with one request that is taken apart among them."""
    run_delta(LENGTHS, heads, group, dk, dv, dtype, seed=21, states="in place")
    run_delta(LENGTHS[:40] + [2600] + LENGTHS[40:], heads, group, dk, dv, dtype, seed=22, before=5)


@pytest.mark.parametrize("n", [24, 64, 65, 255, 256, 257])
def test_the_longest_requests_come_first(n):
    """In every order of lengths: all of them are done, and none twice (states that are updated in place)."""
    for lengths in ([i % 71 for i in range(n)], [70 - i % 71 for i in range(n)], [7] * n, [0] * (n - 1) + [200], [65, 64] * (n // 2) + [0] * (n % 2)):
        run_delta(lengths, 12, 2, 16, 24, BF16, seed=23, states="in place")


@pytest.mark.parametrize("dk,dtype", [(64, BF16), (128, BF16), (128, F16)])
def test_what_is_not_finite_where_requests_fill_the_device(dk, dtype):
    heads, dv, n = 8, 128, 64
    lengths, tokens = [150] * n, 150 * n
    q, k, v = inputs(31, tokens, heads, 2, dk, dv, dtype)
    ld, beta = gates(32, tokens, heads, "spread")
    ends = ints([150 * i for i in range(n + 1)])
    args = (q.cuda(), k.cuda()), (ends, ld.cuda(), beta.cuda())
    whole = B.mmv_delta_attention(*args[0], v.cuda(), *args[1]).cpu()
    at, head, column = 150 * 20 + 70, 3, 77
    v[at, head, column] = math.inf
    got = B.mmv_delta_attention(*args[0], v.cuda(), *args[1]).cpu()
    rest = torch.ones(got.shape, dtype=torch.bool)
    rest[150 * 20:150 * 21, head] = False
    assert torch.equal(got[rest], whole[rest])
    own = slice(150 * 20, 150 * 21)
    want, _, by, _ = plain_delta(q[own], k[own], v[own], [0, 150], ld[own], beta[own], dk ** -0.5)
    fine = want.isfinite()
    assert torch.equal(fine, got[own].isfinite()) and not bool(fine[70:, head, column].any())
    keep = fine & by.isfinite()
    check(got[own][keep], want[keep], by[keep], "out")
