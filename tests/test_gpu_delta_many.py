"""The gated delta rule over thousands of requests in one call: each of them as in a call of few, and a call's time in proportion to their number."""
import pytest
import torch

from paper_2506_23906_amd import binding as B
from test_gpu_delta import BF16, F16, gates, inputs, ints, normal, run_delta

pytestmark = pytest.mark.gpu


def many(lengths, heads, dk, dv, dtype, seed):
    tokens = sum(lengths)
    q, k, v = (x.cuda() for x in inputs(seed, tokens, heads, 1, dk, dv, dtype))
    ld, beta = (x.cuda() for x in gates(seed + 3, tokens, heads))
    ends = torch.zeros(len(lengths) + 1, dtype=torch.int32)
    ends[1:] = torch.tensor(lengths).cumsum(0)
    return q, k, v, ld, beta, ends, normal(seed + 4, len(lengths), heads, dk, dv, dtype=torch.float32).cuda()


@pytest.mark.parametrize("n", [768, 769, 4097, 30000])
@pytest.mark.parametrize("kind", ["some empty", "alone at the ends", "whole chunks"])
def test_each_as_in_a_call_of_few(n, kind):
    print(n, kind, flush=True)
    g = torch.Generator().manual_seed(n)
    some = {"some empty": [0, 0, 1, 2, 8, 63, 65, 130], "alone at the ends": [0], "whole chunks": [64, 128, 0]}[kind]
    lengths = [some[i] for i in torch.randint(len(some), (n,), generator=g).tolist()]
    if kind == "alone at the ends":
        lengths[0], lengths[n // 2], lengths[-1] = 3, 70, 200
    q, k, v, ld, beta, ends, first = many(lengths, 2, 16, 24, BF16, 7)
    state = torch.full_like(first, 5.0)
    out = B.mmv_delta_attention(q, k, v, ends.cuda(), ld, beta, state_in=first, state_out=state)
    for a in range(0, n, 1000):
        b = min(n, a + 1000)
        t0, t1 = int(ends[a]), int(ends[b])
        own = torch.full_like(first[a:b], 5.0)
        if t1 > t0:
            few = B.mmv_delta_attention(q[t0:t1], k[t0:t1], v[t0:t1], (ends[a:b + 1] - t0).cuda(), ld[t0:t1], beta[t0:t1], state_in=first[a:b].clone(), state_out=own)
            assert torch.equal(out[t0:t1], few), (a, b)
        else:
            own = first[a:b]
        assert torch.equal(state[a:b], own), (a, b)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("at", [0, 1200, 1999])
def test_one_that_is_taken_apart_among_many(at, dtype):
    lengths = [i % 4 for i in range(2000)]
    lengths[at], lengths[700] = 4000, 3500
    chunks = [(x + 63) // 64 for x in lengths]
    assert max(chunks) >= 16 and (max(chunks) - 12) * 256 > 3 * sum(chunks)   # (one head of up to 64 columns: 256 blocks at once)
    run_delta(lengths, 1, 1, 16, 16, dtype, seed=41, states="in place", before=3, after=2)


def test_offsets_that_go_backwards():
    """What is left out is not defined; nothing outside the requests' own is written, and what comes before the first such offset is right."""
    n, heads = 1500, 2
    q, k, v, ld, beta, ends, first = many([2] * n, heads, 16, 24, BF16, 11)
    want_state = torch.zeros_like(first)
    want = B.mmv_delta_attention(q, k, v, ends.cuda(), ld, beta, state_in=first, state_out=want_state)
    bad = ends.clone()
    bad[1101:1500:50], bad[1120], bad[1130] = 7, 2 ** 31 - 1, -2 ** 31
    big = torch.full((n + 2, heads, 16, 24), 5.0, device="cuda")
    out = B.mmv_delta_attention(q, k, v, bad.cuda(), ld, beta, state_in=torch.cat([first, first[:2]]), state_out=big)
    assert torch.equal(big[:1100], want_state[:1100]) and bool((big[n:] == 5).all())
    assert out.shape == want.shape


@pytest.mark.parametrize("tokens", [0, 1, 70])
def test_requests_without_tokens(tokens):
    """A batch's free places, very many of them."""
    n = 200_000
    q, k, v, ld, beta, ends, _ = many([0] * (n - 1) + [tokens], 1, 8, 8, BF16, 13)
    first = torch.randn(n, 1, 8, 8, device="cuda")
    state = torch.zeros_like(first)
    out = B.mmv_delta_attention(q, k, v, ends.cuda(), ld, beta, state_in=first, state_out=state)
    assert torch.equal(state[:-1], first[:-1])
    own = torch.zeros_like(first[-1:])
    few = B.mmv_delta_attention(q, k, v, ints([0, tokens]), ld, beta, state_in=first[-1:].clone(), state_out=own)
    assert torch.equal(out, few) and torch.equal(state[-1:], own)


def test_a_graph_follows_its_offsets():
    n, heads, dk, dv = 1300, 2, 16, 24
    q, k, v, ld, beta, ends, first = many([2] * n, heads, dk, dv, BF16, 17)
    tokens, offsets, state, out = 2 * n, ends.cuda(), torch.empty_like(first), torch.empty_like(v)
    ws = B.workspace(B.mmv_delta_attention_workspace_bytes(n, tokens, heads, dk, dv))
    call = lambda: B.mmv_delta_attention(q, k, v, offsets, ld, beta, state_in=first, state_out=state, out=out, ws=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i, lengths in enumerate(([2] * n, [0, 4] * (n // 2), [1] * (n - 1) + [n + 1], [1301] + [1] * (n - 1), [2] * n)):
        new = torch.zeros(n + 1, dtype=torch.int32)
        new[1:] = torch.tensor(lengths).cumsum(0)
        offsets.copy_(new)
        out.fill_(3.0)
        state.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), state.clone()
        out.fill_(3.0)
        state.fill_(7.0)
        call()
        torch.cuda.synchronize()
        assert torch.equal(got[0], out) and torch.equal(got[1], state) and not bool((out == 3).all()), i


def test_time_is_in_proportion():
    """16 times the requests in at most twice 16 times the time (where every workgroup counted all the requests before its own it would be about 10 times that)."""
    def microseconds(n):
        q, k, v, ld, beta, ends, _ = many([8] * n, 1, 16, 16, BF16, 19)
        offsets, out = ends.cuda(), torch.empty_like(v)
        ws = B.workspace(B.mmv_delta_attention_workspace_bytes(n, 8 * n, 1, 16, 16))
        took = []
        for _ in range(6):
            start, end = (torch.cuda.Event(enable_timing=True) for _ in "ab")
            start.record()
            B.mmv_delta_attention(q, k, v, offsets, ld, beta, out=out, ws=ws)
            end.record()
            torch.cuda.synchronize()
            took.append(1000 * start.elapsed_time(end))
        print(n, min(took), flush=True)
        return min(took)
    assert microseconds(65536) <= 32 * microseconds(4096)
