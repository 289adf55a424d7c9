"""How exact the gated delta rule's outputs and states are, apart from the outputs' own rounding: queries that take the difference of two rows of the state that are nearly alike, so that
what is left is small beside what was added up."""
import pytest
import torch

from paper_2506_23906_amd import binding as B
from serving_util import EPS, U

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16
GAP = 2.0 ** -14   # of the rows of a pair, relative: with 16 bits or fewer on the way nothing right is left of their difference


def pairs(seed, n, tokens, heads, dk, dv, dtype):
    """Tokens 2 i and 2 i + 1 write the same value over rows 2 m and 2 m + 1 (keys of one component), nearly equal shares of it; every token reads the difference of such a pair of rows."""
    g = torch.Generator().manual_seed(seed)
    m = torch.randint(dk // 2, (n, tokens), generator=g)
    odd = torch.arange(tokens) % 2
    at = 2 * torch.where(odd == 1, m.roll(1, 1), m) + odd
    asked = 2 * torch.randint(dk // 2, (n, tokens), generator=g)
    k, q = torch.zeros(n, tokens, 1, dk), torch.zeros(n, tokens, 1, dk)
    size = (1 + torch.rand(n, tokens, 1, generator=g)).to(dtype).float()
    k.scatter_(3, at[:, :, None, None], 1.0)
    q.scatter_(3, asked[:, :, None, None], size[..., None])
    q.scatter_(3, asked[:, :, None, None] + 1, -size[..., None])
    v = torch.randn(n, tokens, heads, dv, generator=g)
    v = torch.where(odd[None, :, None, None] == 1, v.roll(1, 1), v).to(dtype)
    beta = 0.3 + 0.6 * torch.rand(n, tokens, heads, generator=g)
    beta = torch.where(odd[None, :, None] == 1, beta.roll(1, 1) * (1 + GAP), beta)
    g_of = -torch.rand(n, tokens, heads, generator=g) / tokens   # (a request decays by e^-1 at most)
    first = torch.randn(n, heads, dk, dv, generator=g)
    first[:, :, 1::2] = first[:, :, ::2] * (1 + GAP)
    return q.to(dtype), k.to(dtype), v, g_of, beta, first, at, asked, size


def followed(q_size, v, g, beta, first, at, asked, shape):
    """Token by token in 64 bits: outputs, the state, and what is added up for each of them."""
    n, tokens = at.shape
    S, A = first.double(), first.double().abs()
    M = A.clone()
    want, most = torch.zeros(shape, dtype=torch.float64), torch.zeros(shape, dtype=torch.float64)
    r = torch.arange(n)
    for t in range(tokens):
        by, b = torch.exp(g[:, t].double())[..., None, None], beta[:, t].double()[..., None]
        S, A, x = S * by, A * by, v[:, t].double()
        own = at[:, t]
        M[r, :, own] = torch.maximum(M[r, :, own], x.abs() + S[r, :, own].abs())
        A[r, :, own] += b * M[r, :, own]
        S[r, :, own] += b * (x - S[r, :, own])
        one, two = asked[:, t], asked[:, t] + 1
        by_q = q_size[:, t].double()[..., None]
        want[:, t] = by_q * (S[r, :, one] - S[r, :, two])
        most[:, t] = by_q * (A[r, :, one] + A[r, :, two])
    return want, most, S, A


@pytest.mark.parametrize("n,tokens,heads,dk,dv,dtype", [
    (1, 1, 1, 32, 32, BF16), (1, 200, 2, 64, 64, BF16), (1, 200, 2, 64, 64, F16), (2, 130, 2, 96, 48, BF16), (2, 130, 2, 96, 48, F16), (1, 300, 2, 128, 128, BF16), (1, 300, 2, 128, 128, F16),
    (8, 100, 32, 32, 256, BF16), (8, 100, 32, 64, 256, F16), (8, 100, 32, 96, 256, BF16), (8, 100, 32, 128, 256, BF16), (8, 100, 32, 128, 256, F16),   # eight waves that compute
    (1, 2000, 1, 64, 32, BF16), (1, 2000, 1, 96, 32, BF16), (1, 2000, 1, 128, 32, BF16), (1, 2000, 1, 128, 32, F16), (1, 2000, 1, 64, 32, F16),        # taken apart
])
def test_differences_of_rows(n, tokens, heads, dk, dv, dtype):
    """Bounds, in units of 2^-24 of what is added up in a row (A): its state at the beginning, and for each token that wrote there what that one's share can be, beta M, M the largest |value| + |row| so
    far.  (Not of what is left in the row, (1 - beta) |row| + beta |value|: u = beta (value - row) is rounded where it is beta (|value| + |row|) large, also where the row is small afterwards; and of
    the inverse's entries for tokens j before it, beta_i beta_j times factors 1 - beta of those between, the sum over j is at most beta_i, so that the products add up at most beta_i M.)  16 units for
    each part of A: the difference, the products of three bf16 terms and their sums; 4 for each chunk of 64 tokens: the decay, its exponential and the product; an output, which adds up the products of
    three terms with two rows, each sum rounded, 16 more, and 4 for its own decay.  What two terms in place of three leave out is up to 128 units (2^-17), of the state as of the scores."""
    print(n, tokens, heads, dk, dv, dtype, flush=True)
    q, k, v, g, beta, first, at, asked, size = pairs(5, n, tokens, heads, dk, dv, dtype)
    state = first.cuda()
    ends = torch.arange(n + 1, dtype=torch.int32, device="cuda") * tokens
    out = B.mmv_delta_attention(*(x.flatten(0, 1).cuda() for x in (q, k, v)), ends, g.flatten(0, 1).cuda(), beta.flatten(0, 1).cuda(), scale=1.0, state_in=state, state_out=state)
    out = out.cpu().double().unflatten(0, (n, tokens))
    want, most, S, A = followed(size, v, g, beta, first, at, asked, out.shape)
    chunks = tokens // 64 + 1
    off = ((out - want).abs() - U[dtype] * want.abs() * (1 + 2 * U[dtype]) - 2.0 ** -25).clamp(min=0)   # (2^-25: half of fp16's smallest step)
    by = EPS * (16 + 4 * (chunks + 1) + 16) * most
    print("outputs: of the bound", float((off / by).max()), "rms", float(off.norm() / most.norm() / EPS), flush=True)
    assert bool((off <= by).all())
    off = (state.cpu().double() - S).abs()
    by = EPS * (16 + 4 * (chunks + 1)) * A
    print("states: of the bound", float((off / by).max()), "rms", float(off.norm() / A.norm() / EPS), flush=True)
    assert bool((off <= by).all())


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("heads,dk,dv", [(1, 64, 32), (1, 96, 32), (2, 128, 72), (1, 128, 256)])
def test_states_from_block_to_block(heads, dk, dv, dtype):
    """Few tokens that write and no decay (its factors are exactly 1), so that what is rounded from block to block is not lost in the rest: for each block a state is a matrix, diagonal here, times the one
    before, in products of three bf16 terms, and a summand: 10 units, six products and the sum each rounded, and the three products that are left out.  A lost third term would be up to 128 for each block."""
    tokens = 2000
    chunks, at_once = (tokens + 63) // 64, 256 // (heads * ((dv + 63) // 64))
    assert (chunks - 12) * at_once > 3 * chunks   # (taken apart)
    blocks = -(-chunks // max(4, -(-chunks // at_once)))
    q, k, v, g, beta, first, at, asked, size = pairs(6, 1, tokens, heads, dk, dv, dtype)
    beta[:, torch.arange(tokens) % 40 >= 2] = 0
    g = torch.zeros_like(g)
    state = first.cuda()
    out = B.mmv_delta_attention(*(x[0].cuda() for x in (q, k, v)), torch.tensor([0, tokens], dtype=torch.int32, device="cuda"), g[0].cuda(), beta[0].cuda(), scale=1.0, state_in=state, state_out=state)
    out = out.cpu().double()[None]
    want, most, S, A = followed(size, v, g, beta, first, at, asked, out.shape)
    off = ((out - want).abs() - U[dtype] * want.abs() * (1 + 2 * U[dtype]) - 2.0 ** -25).clamp(min=0)
    by = EPS * (16 + 10 * blocks + 16) * most
    print(blocks, "blocks; outputs: of the bound", float((off / by).max()), "rms", float(off.norm() / most.norm() / EPS), flush=True)
    assert bool((off <= by).all())
    off = (state.cpu().double() - S).abs()
    by = EPS * (16 + 10 * blocks) * A
    print("states: of the bound", float((off / by).max()), "rms", float(off.norm() / A.norm() / EPS), flush=True)
    assert bool((off <= by).all())
