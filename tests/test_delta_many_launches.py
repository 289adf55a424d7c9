"""What a call of the gated delta rule with many requests launches and needs, on the CPU: beyond 768 requests one launch counts their chunks for all workgroups."""
import pytest

from test_more_serving_launches import CHUNKS, PROMPT, STATES, record  # noqa: F401  (record: a fixture)

COUNT = "delta_count_kernel"


@pytest.mark.parametrize("call,want", [
    ("delta(768, 900)", [(CHUNKS, 6256, 256), (PROMPT, 6144, 512)]), ("delta(769, 900)", [(COUNT, 1, 1024), (CHUNKS, 6264, 256), (PROMPT, 6152, 512)]), ("delta(769, 0)", [(PROMPT, 6152, 512)]),
    ("delta(2000, 9000, heads=1, type=1)", [(COUNT, 1, 1024), (CHUNKS, 2140, 256), (PROMPT, 1024, 512), (STATES, 1024, 128), (PROMPT, 2000, 512)]),
    ("delta(1 << 20, 1 << 20, heads=1)", [(COUNT, 1, 1024), (CHUNKS, 1064960, 256), (PROMPT, 1024, 512), (STATES, 1024, 128), (PROMPT, 1 << 20, 512)]),
])
def test_launches(record, call, want):  # noqa: F811
    assert record(call) == want


def test_workspace(libmmvseg_path):
    """A number for each request, and two more where requests may be taken apart."""
    from paper_2506_23906_amd import binding as B
    per_chunk, round256 = 31232, lambda b: -(-b // 256) * 256
    for n, tokens, heads, slots in ((768, 900, 1, 0), (769, 900, 1, 0), (769, 0, 1, 0), (3000, 900, 2, 0), (3000, 9000, 1, 512), (3000, 9000, 64, 8)):
        chunks = tokens // 64 + min(n, tokens)
        states = min(slots, 2 * chunks // 4) * heads * 32 * 48 * 4
        counts = 0 if n <= 768 or not tokens else round256(4 * (3 * n + 2 if slots else n))
        assert B.mmv_delta_attention_workspace_bytes(n, tokens, heads, 32, 16) == chunks * heads * per_chunk + round256(states) + counts, (n, tokens, heads)
