"""Refusals of the calls of a serving step: found on the host, before anything is launched; and their workspaces.  No GPU."""
import ctypes

import pytest
import torch

from paper_2506_23906_amd import binding as B

OK, INVALID, NULL, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3, 4
A = 0x10000   # aligned, never dereferenced
WS = (A << 8, 1 << 40, None)


@pytest.fixture(scope="module")
def lib(libmmvseg_path):
    return B.load()


def tables(lib, n=4, cached=A, new=A, free=A, free_count=9, table=A, width=8, stride=8, page=16, most=64, offsets=A, context=A, slots=A, positions=A, used=A, ws=WS):
    return lib.mmv_page_tables(n, cached, new, free, free_count, table, width, stride, page, most, offsets, context, slots, positions, used, *ws)


def test_page_tables_refusals(lib):
    for name in ("cached", "new", "free", "table", "offsets", "context", "slots", "positions", "used"):
        assert tables(lib, **{name: None}) == NULL, name
        assert tables(lib, **{name: A + 2}) == INVALID, name
    assert tables(lib, slots=A + 4) == INVALID and tables(lib, used=A + 4) == INVALID
    for bad in (dict(n=1 << 22), dict(page=0), dict(page=65537), dict(most=1 << 31), dict(free_count=1 << 31), dict(width=1 << 31), dict(stride=7)):
        assert tables(lib, **bad) == INVALID, bad
    n = 5000
    assert B.mmv_page_tables_workspace_bytes(4) == 0 and B.mmv_page_tables_workspace_bytes(1 << 22) == 0
    need = B.mmv_page_tables_workspace_bytes(n)
    assert need >= 8 * n and need % 256 == 0
    assert tables(lib, n=n, ws=(None, 1 << 40, None)) == NULL and tables(lib, n=n, ws=(A << 8, need - 1, None)) == WORKSPACE and tables(lib, n=n, ws=(A + 16, need, None)) == WORKSPACE


def cache(k=A, v=A, type=B.MMV_TYPE_BF16, page=16, heads=2, dim=64, pages=10, strides=(2048, 1024, 64), scales=(1.0, 1.0)):
    return B._CacheStruct(k, v, type, page, heads, dim, pages, *strides, *scales)


BAD_CACHES = [dict(page=0), dict(page=65544), dict(heads=0), dict(heads=1025), dict(dim=4), dict(dim=68), dict(dim=264), dict(pages=1 << 31), dict(pages=1 << 28), dict(strides=(2047, 1024, 64)),
              dict(strides=(2048, 1023, 64)), dict(strides=(2048, 1024, 65)), dict(strides=(1 << 41, 1024, 64)), dict(strides=(2048, 1024, 1 << 28)), dict(k=A + 8), dict(v=A + 8), dict(scales=(0.5, 1.0)),
              dict(type=B.MMV_TYPE_F16), dict(type=0), dict(type=7), dict(type=B.MMV_TYPE_E4M3, scales=(0.0, 1.0)), dict(type=B.MMV_TYPE_E4M3, scales=(1.0, float("inf"))),
              dict(type=B.MMV_TYPE_E4M3, scales=(1.0, float("nan")))]


def append(lib, c, tokens=3, k=A, ks=128, v=A, vs=128, type=B.MMV_TYPE_BF16, slots=A):
    return lib.mmv_cache_append(tokens, k, ks, v, vs, type, slots, ctypes.addressof(c) if c else None, None)


def attention(lib, c, n=3, q_heads=4, q=A, qs=256, type=B.MMV_TYPE_BF16, table=A, width=8, stride=8, context=A, scale=1.0, window=0, out=A, lse=A, ws=WS):
    return lib.mmv_paged_attention(n, q_heads, q, qs, type, ctypes.addressof(c) if c else None, table, width, stride, context, scale, window, out, lse, *ws)


def test_cache_append_refusals(lib):
    assert append(lib, None) == NULL and append(lib, cache(), tokens=0) == OK and append(lib, cache(pages=0, k=None, v=None)) == OK
    for bad in BAD_CACHES:
        assert append(lib, cache(**bad)) == INVALID, bad
    assert append(lib, cache(k=None)) == NULL
    for name in ("k", "v", "slots"):
        assert append(lib, cache(), **{name: None}) == NULL and append(lib, cache(), **{name: A + 4}) == INVALID
    for bad in (dict(ks=132), dict(vs=120), dict(ks=120), dict(tokens=1 << 31), dict(type=B.MMV_TYPE_E4M3), dict(type=B.MMV_TYPE_F16)):
        assert append(lib, cache(), **bad) == INVALID, bad


def test_paged_attention_refusals(lib):
    assert attention(lib, None) == NULL and attention(lib, cache(), n=0) == OK
    for bad in BAD_CACHES:
        assert attention(lib, cache(**bad)) == INVALID, bad
    assert attention(lib, cache(page=12)) == UNSUPPORTED
    for name in ("q", "table", "context", "out"):
        assert attention(lib, cache(), **{name: None}) == NULL and attention(lib, cache(), **{name: A + 2}) == INVALID, name
    for bad in (dict(q=A + 8), dict(out=A + 8), dict(lse=A + 2), dict(q_heads=3), dict(q_heads=0), dict(q_heads=34), dict(qs=248), dict(qs=260), dict(width=1 << 31), dict(width=1 << 27, stride=1 << 27),
                dict(stride=7), dict(n=1 << 22), dict(type=B.MMV_TYPE_F16), dict(type=9)):
        assert attention(lib, cache(), **bad) == INVALID, bad
    need = B.mmv_paged_attention_workspace_bytes(3, 4, 2, 64, 128)
    if need:
        assert need % 256 == 0 and attention(lib, cache(), ws=(None, 1 << 40, None)) == NULL
        assert attention(lib, cache(), ws=(A << 8, need - 1, None)) == WORKSPACE and attention(lib, cache(), ws=((A << 8) + 16, need, None)) == WORKSPACE
    assert B.mmv_paged_attention_workspace_bytes(3, 5, 2, 64, 128) == 0


def decay(lib, n=3, tokens=9, heads=4, kv=2, dk=64, dv=32, q=A, qs=256, k=A, ks=128, v=A, vs=64, type=B.MMV_TYPE_BF16, offsets=A, ld=A, sin=A, sout=A, states=5, index=A, out=A, ws=WS):
    return lib.mmv_decay_attention(n, tokens, heads, kv, dk, dv, q, qs, k, ks, v, vs, type, offsets, ld, 1.0, sin, sout, states, index, out, *ws)


def step(lib, n=3, heads=4, kv=2, dk=64, dv=32, q=A, qs=256, k=A, ks=128, v=A, vs=64, type=B.MMV_TYPE_BF16, ld=A, sin=A, sout=A, states=5, index=A, out=A):
    return lib.mmv_decay_step(n, heads, kv, dk, dv, q, qs, k, ks, v, vs, type, ld, 1.0, sin, sout, states, index, out, None)


def test_decay_refusals(lib):
    assert decay(lib, n=0) == OK and step(lib, n=0) == OK
    for call in (decay, step):
        for name in ("q", "k", "v", "ld", "out"):
            assert call(lib, **{name: None}) == NULL, name
        for name in ("q", "k", "v", "sin", "sout", "out"):
            assert call(lib, **{name: A + 8}) == INVALID, name
        for bad in (dict(ld=A + 2), dict(index=A + 2), dict(heads=0), dict(heads=3), dict(kv=0), dict(kv=8), dict(heads=2048, kv=2), dict(dk=0), dict(dk=136), dict(dk=60), dict(dv=264), dict(dv=4),
                    dict(qs=248), dict(qs=257), dict(ks=120), dict(vs=56), dict(type=0), dict(type=B.MMV_TYPE_E4M3), dict(states=1 << 31), dict(n=1 << 22),
                    dict(index=None, states=2), dict(sout=A + 4 * 64 * 32 * 4)):   # (states that overlap in part)
            assert call(lib, **bad) == INVALID, bad
    assert decay(lib, offsets=None) == NULL and decay(lib, offsets=A + 2) == INVALID and decay(lib, tokens=1 << 31) == INVALID
    need = B.mmv_decay_attention_workspace_bytes(3, 9, 4, 64, 32)
    if need:
        assert need % 256 == 0 and decay(lib, ws=(None, 1 << 40, None)) == NULL
        assert decay(lib, ws=(A << 8, need - 1, None)) == WORKSPACE and decay(lib, ws=((A << 8) + 16, need, None)) == WORKSPACE
    assert B.mmv_decay_attention_workspace_bytes(3, 9, 4, 136, 32) == 0


def test_the_binding_refuses_what_does_not_fit(lib):
    """CPU tensors, wrong types and shapes: before the library is called."""
    i, x = torch.zeros(4, dtype=torch.int32), torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(B.MmvError):
        B.mmv_page_tables(i, i, i, torch.zeros(4, 4, dtype=torch.int32), 16, 4)
    for k, v in ((x, x), (torch.zeros(2, 2, 8, 64), torch.zeros(2, 2, 8, 32)), (torch.zeros(2, 2, 8, 64, dtype=torch.bfloat16),) * 2, (torch.zeros(2, 2, 8, 64),) * 2):
        with pytest.raises(B.MmvError):
            B.PagedCache(k, v)
    cache = B.PagedCache.__new__(B.PagedCache)
    cache.k = cache.v = torch.zeros(2, 2, 8, 64, dtype=torch.bfloat16)
    cache.k_scale = cache.v_scale = 1.0
    cache._struct = B._CacheStruct()
    cache._ref = ctypes.addressof(cache._struct)
    with pytest.raises(B.MmvError):
        B.mmv_cache_append(x, x, torch.zeros(4, dtype=torch.int64), cache)
    with pytest.raises(B.MmvError):
        B.mmv_cache_append(x.float(), x.float(), torch.zeros(4, dtype=torch.int64), cache)
    with pytest.raises(B.MmvError):
        B.mmv_paged_attention(x, cache, torch.zeros(4, 4, dtype=torch.int32), i)
    for q in (x, x.float(), x[0]):
        with pytest.raises(B.MmvError):
            B.mmv_decay_step(q, x, x, torch.zeros(2))
        with pytest.raises(B.MmvError):
            B.mmv_decay_attention(q, x, x, i, torch.zeros(2))
