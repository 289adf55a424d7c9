"""Launches of a serving step's largest calls: HIP takes fewer than 2^32 threads a launch, so they are split.  The run-time is replaced by one that writes launches down; no GPU."""
import pytest

from test_serving_launches import BLOCKS, JOIN, LIST, PROMPT, record  # noqa: F401


@pytest.mark.parametrize("call,want", [
    ("attention((1 << 20) + 3, 20, heads=2, group=16)", {LIST: None, JOIN: ((1 << 20) + 3) * 32}),
    ("attention((1 << 22) - 1, 60, heads=2, group=16)", {LIST: None, JOIN: ((1 << 22) - 1) * 32}),
    ("step((1 << 21) + 5)", {"decay_step_kernel": ((1 << 21) + 5) * 8}),
    ("step((1 << 22) - 1, heads=511)", {"decay_step_kernel": ((1 << 22) - 1) * 511}),
    ("decay((1 << 21) + 5, 100)", {PROMPT: ((1 << 21) + 5) * 8}),
    ("decay(1 << 14, 256, 256, 8, 256)", {PROMPT: 1 << 22}),
    ("decay((1 << 21) + 5, (1 << 21) + 5)", {PROMPT: None, BLOCKS: ((1 << 21) + 5) * 8 * 4}),
    ("decay(2100000, 2100000, 1020, 8, 8)", {PROMPT: None, BLOCKS: 2100000 * 1020}),
])
def test_no_launch_has_2_to_32_threads(record, call, want):   # noqa: F811
    launches = record(call)
    assert all(blocks * threads < 1 << 32 for _, blocks, threads in launches), launches
    assert {name for name, _, _ in launches} == set(want)
    for name, blocks in want.items():
        if blocks is not None:
            assert sum(b for n, b, _ in launches if n == name) == blocks
