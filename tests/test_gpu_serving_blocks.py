"""Prompts' recurrence where some requests have several blocks and others one: states are kept for the former alone."""
import pytest
import torch

from paper_2506_23906_amd import binding as B
from serving_util import check, plain_decay

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


def case(lengths, heads, dk, dv, dtype, seed=3):
    g = torch.Generator().manual_seed(seed)
    t = sum(lengths)
    q, k, v = (torch.randn(t, heads, d, generator=g).to(dtype) for d in (dk, dk, dv))
    ends = [0]
    for x in lengths:
        ends.append(ends[-1] + x)
    ld = torch.tensor([-(2.0 ** -(3 + 2 * h)) for h in range(heads)])
    return q, k, v, ends, ld, torch.randn(len(lengths), heads, dk, dv, generator=g)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("lengths", [[3, 700, 0, 64, 65, 260, 1], [5] * 30 + [900] + [5] * 20 + [300, 0, 129], [2, 0, 3] * 25 + [800] + [7] * 40 + [257, 1] + [1] * 30 + [513]])
@pytest.mark.parametrize("heads,dk,dv", [(2, 16, 24), (3, 128, 128)])
def test_blocks_of_some_requests(heads, dk, dv, lengths, dtype):
    print(heads, dk, dv, len(lengths), dtype, flush=True)
    q, k, v, ends, ld, first = case(lengths, heads, dk, dv, dtype)
    n, t = len(lengths), sum(lengths)
    need = B.mmv_decay_attention_workspace_bytes(n, t, heads, dk, dv)
    ws = torch.full((need + 4096,), 0xFF, dtype=torch.uint8, device="cuda")
    state = first.cuda()
    out = B.mmv_decay_attention(q.cuda(), k.cuda(), v.cuda(), torch.tensor(ends, dtype=torch.int32, device="cuda"), ld.cuda(), state_in=state, state_out=state, ws=ws[:need])
    want, final, by, final_by = plain_decay(q, k, v, ends, ld, dk ** -0.5, first)
    check(out, want, by, "out")
    check(state, final, final_by, "states")
    assert bool((ws[need:] == 0xFF).all())


@pytest.mark.parametrize("n", [5, 70])
def test_offsets_that_go_backwards_stay_inside_the_scratch(n):
    """Every other offset goes back to 0, so that the spans' lengths add up to far more than the tokens."""
    heads, dk, dv, t = 2, 64, 64, 3000
    q, k, v, _, ld, _ = case([t], heads, dk, dv, BF16)
    ends = [0 if i % 2 == 0 else t for i in range(n + 1)]
    need = B.mmv_decay_attention_workspace_bytes(n, t, heads, dk, dv)
    ws = torch.full((need + (1 << 24),), 0xFF, dtype=torch.uint8, device="cuda")
    B.mmv_decay_attention(q.cuda(), k.cuda(), v.cuda(), torch.tensor(ends, dtype=torch.int32, device="cuda"), ld.cuda(), ws=ws[:need])
    assert bool((ws[need:] == 0xFF).all())
