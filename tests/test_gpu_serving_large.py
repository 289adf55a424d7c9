"""Calls of a serving step that take more threads than one launch can have."""
import math

import pytest
import torch

from paper_2506_23906_amd import binding as B

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def test_attention_rows_beyond_one_joining_launch():
    """2^20 + 3 rows of 32 query heads with a position each, or none: what the list's waves and the joining launches write."""
    n, heads, group, dim, page, width = (1 << 20) + 3, 2, 16, 8, 8, 40
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn(1000, heads, page, dim, generator=g, device="cuda").to(BF16) for _ in "kv")
    q = torch.randn(n, heads * group, dim, generator=g, device="cuda").to(BF16)
    row = torch.arange(n, device="cuda")
    table = (row % 1000).int()[:, None].expand(n, width).contiguous()
    context = (row % 5 != 0).int()
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    B.mmv_paged_attention(q, B.PagedCache(k, v), table, context, scale=1.0, out=out, lse=lse)
    want = v[row % 1000, :, 0].repeat_interleave(group, 1)
    score = (q.float() * k[row % 1000, :, 0].repeat_interleave(group, 1).float()).sum(2)
    empty = context == 0
    assert bool((out[empty] == 0).all()) and bool((lse[empty] == -math.inf).all())
    assert torch.equal(out[~empty], want[~empty])
    # (a score of 8 products of normal values, a logarithm of 1)
    assert bool(((lse - score)[~empty].abs() <= 16 * 2.0 ** -24 * (1 + (q.float().abs() * k[row % 1000, :, 0].repeat_interleave(group, 1).float().abs()).sum(2)[~empty])).all())


def test_steps_beyond_one_launch():
    n, heads, dim = (1 << 21) + 5, 8, 8
    g = torch.Generator(device="cuda").manual_seed(2)
    q, k, v = (torch.randn(n, heads, dim, generator=g, device="cuda").to(BF16) for _ in range(3))
    state = torch.full((n, heads, dim, dim), 7.0, device="cuda")
    out = B.mmv_decay_step(q, k, v, torch.zeros(heads, device="cuda"), None, state, scale=1.0)
    want = (q.float() * k.float()).sum(2, keepdim=True) * v.float()
    by = 2.0 ** -8 * want.abs() + 16 * 2.0 ** -24 * (q.float().abs() * k.float().abs()).sum(2, keepdim=True) * v.float().abs() + 2.0 ** -126
    assert bool(((out.float() - want).abs() <= by).all())
    for part in (slice(0, 1000), slice((1 << 21) - 1000, n)):
        assert torch.equal(state[part], k[part].float()[..., :, None] * v[part].float()[..., None, :])
    assert not bool((state.view(n, -1)[:, 0] == 7.0).any())
