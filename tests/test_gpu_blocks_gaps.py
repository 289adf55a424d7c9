"""Reading a cache in blocks where most of a batch's places are free: the requests of a wave's tokens may lie far from each other."""
import pytest
import torch

from block_util import plain_read, values_of
from paper_2506_23906_amd import binding as B
from test_gpu_blocks import BF16, F16, INT8, Both, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,dim", [(1, 8), (1, 64), (4, 64), (8, 128)])   # 64, 8, 2 tokens and one to a wave
@pytest.mark.parametrize("gap", [0, 1, 2, 3, 62, 63, 64, 65, 700, 5000])
def test_requests_far_from_each_other(heads, dim, gap):
    print(heads, dim, gap, flush=True)
    both = Both(3, 6, heads, 16, dim, 8, INT8)
    rows = [[0, 1], [2, 3], [4, 5]]
    lengths = [5] + [0] * gap + [3, 1] + [0] * gap + [20, 0, 2]
    table = [rows[r % 3] for r in range(len(lengths))]
    offsets = [0]
    for x in lengths:
        offsets.append(offsets[-1] + x)
    first = [r % 5 for r in range(len(lengths))]
    out = tuple(torch.full((offsets[-1] + 3, heads, dim), 9.0, dtype=BF16, device="cuda") for _ in "kv")
    B.mmv_block_read(both.cache, ints(table), ints(offsets), first=ints(first), out=out)
    for got, values in zip(out, both.values()):
        assert torch.equal(got.cpu(), plain_read(values, table, offsets, first, offsets[-1] + 3, BF16, 9.0))


def test_time_does_not_grow_with_the_free_places_between():
    """100000 of them: 20 times the time of none at most (one after the other, each a read of memory, they would take thousands of times as long)."""
    both = Both(4, 2, 1, 16, 64, 8, INT8)

    def microseconds(gap):
        offsets = ints([0, 3] + [3] * gap + [6])
        table = torch.zeros(len(offsets) - 1, 1, dtype=torch.int32, device="cuda")
        out = tuple(torch.empty(6, 1, 64, dtype=F16, device="cuda") for _ in "kv")
        took = []
        for _ in range(8):
            start, end = (torch.cuda.Event(enable_timing=True) for _ in "ab")
            start.record()
            B.mmv_block_read(both.cache, table, offsets, out=out)
            end.record()
            torch.cuda.synchronize()
            took.append(1000 * start.elapsed_time(end))
        print(gap, min(took), flush=True)
        return min(took)
    assert microseconds(100_000) <= 20 * max(microseconds(0), 3.0)
