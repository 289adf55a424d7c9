"""Attention where a workgroup has a whole segment, at the largest parts that it joins."""
import pytest
import torch

from test_gpu_serving import BF16, E4M3, F16, attention_case, run_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,cache_type", [(BF16, BF16), (F16, F16), (BF16, E4M3)])
@pytest.mark.parametrize("group,dim", [(16, 128), (15, 136), (8, 256), (16, 64), (16, 120), (12, 160)])
def test_the_largest_groups_in_a_workgroup(group, dim, dtype, cache_type):
    """Eight waves' parts of 16 queries of 128 components are 64 KB of LDS, and more stands beside them."""
    contexts = [255, 256, 0, 33, 129]
    print(group, dim, dtype, cache_type, flush=True)
    run_attention(*attention_case(dim, contexts, 2, group, dim, 16, dtype, cache_type), contexts)
    run_attention(*attention_case(dim, [240, 97], 2, group, dim, 16, dtype, cache_type), [240, 97])
