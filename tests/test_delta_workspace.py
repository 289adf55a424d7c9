"""The workspace of the gated delta rule: its size, and that a smaller or badly aligned one is refused.  No GPU."""
import pytest

from paper_2506_23906_amd import binding as B
from test_more_serving_abi import A, INVALID, NULL, OK, WORKSPACE, delta, lib  # noqa: F401  (lib: a fixture)


@pytest.mark.parametrize("n,tokens,heads,dk,dv", [(3, 9, 4, 64, 32), (3, 5000, 4, 64, 32), (800, 100, 2, 64, 32)])
def test_refused(lib, n, tokens, heads, dk, dv):  # noqa: F811
    chunks, counts = tokens // 64 + min(n, tokens), 4 * n if n > 768 else 0
    states = heads * dk * (dk + dv) * 4 * min(2 * chunks // 4, 2 * 256 // heads) if tokens > 960 else 0   # (of up to 64 columns: 256 / heads blocks of a head at once)
    need = chunks * heads * 31232 + -(-states // 256) * 256 + -(-counts // 256) * 256
    assert B.mmv_delta_attention_workspace_bytes(n, tokens, heads, dk, dv) == need
    sizes = dict(n=n, tokens=tokens, heads=heads, dk=dk, dv=dv, states=n, index=A)
    assert delta(lib, **sizes, ws=(None, 1 << 40, None)) == NULL
    assert delta(lib, **sizes, ws=(A << 8, need - 1, None)) == WORKSPACE and delta(lib, **sizes, ws=((A << 8) + 16, need, None)) == WORKSPACE
    assert delta(lib, **sizes, ws=(A << 8, 0, None)) == WORKSPACE


def test_sizes_that_are_refused_need_none(lib):  # noqa: F811
    for sizes in ((3, 9, 4, 60, 32), (3, 9, 4, 136, 32), (3, 9, 4, 64, 264), (3, 9, 0, 64, 32), (1 << 22, 9, 4, 64, 32), (3, 1 << 31, 4, 64, 32)):
        assert B.mmv_delta_attention_workspace_bytes(*sizes) == 0, sizes
    assert B.mmv_delta_attention_workspace_bytes(3, 0, 4, 64, 32) == 0 and B.mmv_delta_attention_workspace_bytes(0, 9, 4, 64, 32) == 0
    assert OK == 0 and INVALID != WORKSPACE
