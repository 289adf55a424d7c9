"""Requests of the gated delta rule that are taken apart into blocks of chunks: what is not finite in any of their blocks, and their outputs by the kernels of eight waves that compute.  Every test asserts
that its lengths are such that the rule takes them apart."""
import math

import pytest
import torch

from block_util import plain_delta
from paper_2506_23906_amd import binding as B
from serving_util import check
from test_gpu_delta import BF16, F16, NAN, gates, inputs, ints, normal, run_delta

pytestmark = pytest.mark.gpu


def taken_apart(lengths, heads, dv):
    """The rule: the longest request has more than three times an even share of the chunks and twelve more, 16 at least (256 compute units, a workgroup of 64 columns on each)."""
    chunks, at_once = [(x + 63) // 64 for x in lengths], 256 // (heads * ((dv + 63) // 64))
    return max(chunks) >= 16 and (max(chunks) - 12) * at_once > 3 * sum(chunks)


def block_of(lengths, heads, dv):
    """Tokens of a block."""
    chunks, at_once = sum((x + 63) // 64 for x in lengths), 256 // (heads * ((dv + 63) // 64))
    return 64 * max(4, -(-chunks // at_once))


@pytest.mark.parametrize("which", ["v", "k", "q", "log_decay", "beta", "state", "infinite v", "infinite k", "infinite q"])
@pytest.mark.parametrize("where", ["first block", "middle", "a block's last token", "last block"])
@pytest.mark.parametrize("dk,dv,dtype", [(64, 64, BF16), (128, 96, BF16), (128, 64, F16), (40, 24, F16)])
def test_what_is_not_finite(dk, dv, dtype, where, which):
    lengths, heads = [10, 1500, 200], 2
    assert taken_apart(lengths, heads, dv)
    block = block_of(lengths, heads, dv)
    assert 5 <= 1500 // block
    at = 10 + {"first block": 100, "middle": 4 * block + 37, "a block's last token": 2 * block - 1, "last block": 1490}[where]
    tokens, ends = sum(lengths), [0, 10, 1510, 1710]
    q, k, v = inputs(51, tokens, heads, 1, dk, dv, dtype)
    ld, beta = gates(52, tokens, heads)
    ld = ld * 0.05   # (what comes in the first block is still there in the last)
    state = normal(53, 3, heads, dk, dv, dtype=torch.float32)
    {"v": lambda: v.__setitem__((at, 1, 7), NAN), "k": lambda: k.__setitem__((at, 1, 9), NAN), "q": lambda: q.__setitem__((at, 1, 9), NAN), "log_decay": lambda: ld.__setitem__((at, 1), NAN),
     "beta": lambda: beta.__setitem__((at, 1), NAN), "state": lambda: state.__setitem__((1, 1, 3, 7), math.inf), "infinite v": lambda: v.__setitem__((at, 1, 7), -math.inf),
     "infinite k": lambda: k.__setitem__((at, 1, 9), math.inf), "infinite q": lambda: q.__setitem__((at, 1, 9), -math.inf)}[which]()
    on_gpu = state.cuda()
    out = B.mmv_delta_attention(q.cuda(), k.cuda(), v.cuda(), ints(ends), ld.cuda(), beta.cuda(), scale=1.0, state_in=on_gpu, state_out=on_gpu)
    out, on_gpu = out.cpu().double(), on_gpu.cpu().double()
    want, final, by, final_by = plain_delta(q, k, v, ends, ld, beta, 1.0, state)
    for got, ref, off in ((out, want, by), (on_gpu, final, final_by)):
        fine = ref.isfinite()
        assert torch.equal(fine, got.isfinite())
        keep = fine & off.isfinite()
        check(got[keep], ref[keep], off[keep], which)
    # no other request, no other head, no earlier token
    other = out.clone()
    other[10:1510, 1] = 0
    assert bool(other.isfinite().all())
    assert bool(out[:10 if which == "state" else at].isfinite().all())
    assert bool(on_gpu[[0, 2]].isfinite().all()) and bool(on_gpu[1, 0].isfinite().all())
    column = which in ("v", "infinite v", "state")
    if column:   # nor another column
        rest = [c for c in range(dv) if c != 7]
        assert bool(out[:, :, rest].isfinite().all()) and bool(on_gpu[..., rest].isfinite().all())
    if which in ("q", "infinite q"):   # a query is its own token's alone
        assert not bool(out[at, 1].isfinite().any()) and bool(on_gpu.isfinite().all())
        assert bool(out[at + 1:].isfinite().all())
    else:
        assert not bool(on_gpu[1, 1, :, 7].isfinite().any()) and not bool(out[10 if which == "state" else at:1510, 1, 7].isfinite().any())


LENGTHS = [0] * 30 + [1 + 7 * i % 64 for i in range(14)] + [0, 64, 3000, 63] + [0] * 22


@pytest.mark.parametrize("heads,group,dk,dv,dtype", [(8, 2, 64, 128, BF16), (8, 1, 128, 128, BF16), (8, 4, 96, 256, F16), (8, 2, 128, 128, F16), (8, 8, 80, 112, BF16), (8, 2, 48, 256, F16)])
@pytest.mark.parametrize("states", ["both", "in place", "none"])
def test_outputs_of_eight_waves(heads, group, dk, dv, dtype, states):
    assert taken_apart(LENGTHS, heads, dv) and len(LENGTHS) * heads * ((dv + 127) // 128) >= 512
    run_delta(LENGTHS, heads, group, dk, dv, dtype, seed=61, states=states, before=2, after=1)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("kind", ["none", "hard"])
def test_blocks_of_any_gates(kind, dtype):
    lengths = [1030, 0, 5]
    assert taken_apart(lengths, 2, 72)
    run_delta(lengths, 2, 1, 120, 72, dtype, kind, seed=62, states="in place")
