"""Refusals of the calls on a cache in blocks and of the gated delta rule: found on the host, before anything is launched.  No GPU."""
import ctypes

import pytest
import torch

from block_util import codes_of, plain_append, plain_delta, values_of
from paper_2506_23906_amd import binding as B

OK, INVALID, NULL, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3, 4
A = 0x10000   # aligned, never dereferenced
WS = (A << 8, 1 << 40, None)


@pytest.fixture(scope="module")
def lib(libmmvseg_path):
    return B.load()


def cache(k=A, v=A, ks=A, vs=A, type=B.MMV_TYPE_I8, page=32, heads=2, dim=64, block=16, pages=10, strides=(4096, 2048, 64)):
    return B._BlockCacheStruct(k, v, ks, vs, type, page, heads, dim, block, pages, *strides)


BAD_CACHES = [dict(page=0), dict(page=65544, block=8), dict(page=40), dict(heads=0), dict(heads=1025), dict(dim=4), dict(dim=68), dict(dim=264), dict(pages=1 << 31), dict(pages=1 << 27),
              dict(block=0), dict(block=4), dict(block=12, page=24), dict(block=64), dict(block=24), dict(strides=(4095, 2048, 64)), dict(strides=(4096, 2047, 64)), dict(strides=(4096, 2048, 65)),
              dict(strides=(1 << 41, 2048, 64)), dict(strides=(4096, 2048, 1 << 28)), dict(k=A + 8), dict(v=A + 8), dict(ks=A + 2), dict(vs=A + 2), dict(type=B.MMV_TYPE_BF16), dict(type=0), dict(type=7)]


def ref(c):
    return ctypes.addressof(c) if c else None


def append(lib, c, tokens=3, k=A, ks=128, v=A, vs=128, type=B.MMV_TYPE_BF16, slots=A):
    return lib.mmv_block_append(tokens, k, ks, v, vs, type, slots, ref(c), None)


def read(lib, c, n=3, tokens=9, offsets=A, first=A, table=A, width=8, stride=8, type=B.MMV_TYPE_F16, k=A, ks=128, v=A, vs=128):
    return lib.mmv_block_read(n, tokens, offsets, first, table, width, stride, ref(c), type, k, ks, v, vs, None)


def attention(lib, c, n=3, q_heads=4, q=A, qs=256, type=B.MMV_TYPE_BF16, table=A, width=8, stride=8, context=A, window=0, out=A, lse=A, ws=WS):
    return lib.mmv_block_attention(n, q_heads, q, qs, type, ref(c), table, width, stride, context, 1.0, window, out, lse, *ws)


def test_caches(lib):
    for call, empty in ((append, dict(tokens=0)), (read, dict(tokens=0)), (attention, dict(n=0))):
        assert call(lib, None) == NULL and call(lib, cache(), **empty) == OK
        for bad in BAD_CACHES:
            assert call(lib, cache(**bad), **empty) == INVALID, bad
        for name in ("k", "v", "ks", "vs"):
            assert call(lib, cache(**{name: None}), **empty) == NULL, name
            assert call(lib, cache(pages=0, **{name: None}), **empty) == OK, name
    assert append(lib, cache(pages=0)) == OK


def test_append(lib):
    for name in ("k", "v", "slots"):
        assert append(lib, cache(), **{name: None}) == NULL and append(lib, cache(), **{name: A + 4}) == INVALID
    for bad in (dict(ks=132), dict(vs=120), dict(ks=120), dict(vs=132), dict(tokens=1 << 26), dict(type=B.MMV_TYPE_E4M3), dict(type=B.MMV_TYPE_I8), dict(type=0)):
        assert append(lib, cache(), **bad) == INVALID, bad


def test_read(lib):
    for name in ("offsets", "table", "k", "v"):
        assert read(lib, cache(), **{name: None}) == NULL and read(lib, cache(), **{name: A + 2}) == INVALID, name
    for bad in (dict(first=A + 2), dict(k=A + 8), dict(v=A + 8), dict(n=1 << 22), dict(tokens=1 << 31), dict(width=1 << 31), dict(stride=7), dict(type=B.MMV_TYPE_I8), dict(ks=120), dict(vs=132)):
        assert read(lib, cache(), **bad) == INVALID, bad
    assert read(lib, cache(), n=0) == OK


def test_attention(lib):
    for name in ("q", "table", "context", "out"):
        assert attention(lib, cache(), **{name: None}) == NULL and attention(lib, cache(), **{name: A + 2}) == INVALID, name
    for bad in (dict(q=A + 8), dict(out=A + 8), dict(lse=A + 2), dict(q_heads=3), dict(q_heads=0), dict(q_heads=34), dict(qs=248), dict(qs=260), dict(width=1 << 31), dict(width=1 << 26, stride=1 << 26),
                dict(stride=7), dict(n=1 << 22), dict(type=B.MMV_TYPE_E4M3), dict(type=9)):
        assert attention(lib, cache(), **bad) == INVALID, bad
    need = B.mmv_paged_attention_workspace_bytes(3, 4, 2, 64, 256)
    assert need and attention(lib, cache(), ws=(None, 1 << 40, None)) == NULL
    assert attention(lib, cache(), ws=(A << 8, need - 1, None)) == WORKSPACE and attention(lib, cache(), ws=((A << 8) + 16, need, None)) == WORKSPACE


def delta(lib, n=3, tokens=9, heads=4, kh=2, dk=64, dv=32, q=A, qs=128, k=A, ks=128, v=A, vs=128, type=B.MMV_TYPE_BF16, offsets=A, ld=A, beta=A, sin=A, sout=A, states=5, index=A, out=A, ws=WS):
    return lib.mmv_delta_attention(n, tokens, heads, kh, dk, dv, q, qs, k, ks, v, vs, type, offsets, ld, beta, 1.0, sin, sout, states, index, out, *ws)


def step(lib, n=3, heads=4, kh=2, dk=64, dv=32, q=A, qs=128, k=A, ks=128, v=A, vs=128, type=B.MMV_TYPE_BF16, ld=A, beta=A, sin=A, sout=A, states=5, index=A, out=A):
    return lib.mmv_delta_step(n, heads, kh, dk, dv, q, qs, k, ks, v, vs, type, ld, beta, 1.0, sin, sout, states, index, out, None)


def test_delta(lib):
    assert delta(lib, n=0) == OK and step(lib, n=0) == OK
    for call in (delta, step):
        for name in ("q", "k", "v", "ld", "beta", "out"):
            assert call(lib, **{name: None}) == NULL, name
        for name in ("q", "k", "v", "sin", "sout", "out"):
            assert call(lib, **{name: A + 8}) == INVALID, name
        for bad in (dict(ld=A + 2), dict(beta=A + 2), dict(index=A + 2), dict(heads=0), dict(heads=3), dict(kh=0), dict(kh=8), dict(heads=2048, kh=2), dict(dk=0), dict(dk=136), dict(dk=60), dict(dv=264),
                    dict(dv=4), dict(qs=120), dict(qs=129), dict(ks=120), dict(vs=120), dict(qs=(1 << 24) + 8), dict(type=0), dict(type=B.MMV_TYPE_E4M3), dict(states=1 << 31), dict(n=1 << 22),
                    dict(index=None, states=2), dict(sout=A + 4 * 64 * 32 * 4)):   # (states that overlap in part)
            assert call(lib, **bad) == INVALID, bad
    assert delta(lib, offsets=None) == NULL and delta(lib, offsets=A + 2) == INVALID and delta(lib, tokens=1 << 31) == INVALID
    need = B.mmv_delta_attention_workspace_bytes(3, 9, 4, 64, 32)
    if need:
        assert need % 256 == 0 and delta(lib, ws=(None, 1 << 40, None)) == NULL
        assert delta(lib, ws=(A << 8, need - 1, None)) == WORKSPACE and delta(lib, ws=((A << 8) + 16, need, None)) == WORKSPACE
    assert B.mmv_delta_attention_workspace_bytes(3, 9, 4, 60, 32) == 0


def test_python_refuses_what_is_no_cache(libmmvseg_path):
    k = torch.zeros(2, 1, 16, 64, dtype=torch.int8)
    s = torch.zeros(2, 1, 2)
    for bad in ((k, k, s, s), (k.half(), k.half(), s, s), (k, k[:1], s, s)):   # (not in GPU memory)
        with pytest.raises(B.MmvError):
            B.BlockCache(*bad)
    for call in (lambda: B.mmv_block_append(k, k, k, object()), lambda: B.mmv_block_read(object(), k, k), lambda: B.mmv_block_attention(k, object(), k, k)):
        with pytest.raises(B.MmvError):
            call()


# ---- the plain forms themselves ---------------------------------------------------------------------------------------


def test_codes():
    x = torch.tensor([0.5, 1.5, 2.5, -0.5, 126.5, 127.5, 1e9, -1e9], dtype=torch.float64)
    assert codes_of(x, torch.tensor(1.0, dtype=torch.float64), torch.int8).tolist() == [0, 2, 2, 0, 126, 127, 127, -127]
    x = torch.tensor([17.0, 19.0, 449.0, 2.0 ** -10, 3 * 2.0 ** -10], dtype=torch.float64)   # (ties go to even)
    assert codes_of(x, torch.tensor(1.0, dtype=torch.float64), torch.float8_e4m3fn).tolist() == [16, 20, 448, 0, 2.0 ** -8]


def test_a_block_whose_scale_grows():
    codes, scales = torch.zeros(1, 1, 16, 8, dtype=torch.int8), torch.zeros(1, 1, 2)
    one = torch.full((1, 1, 8), 1.0).half()
    plain_append(codes, scales, one, [0], 8)
    plain_append(codes, scales, 0.5 * one, [1], 8)
    plain_append(codes, scales, 4 * one, [2], 8)
    assert codes[0, 0, :3, 0].tolist() == [32, 16, 127] and scales[0, 0, 1] == 0     # (127 / 4 = 31.75, 64 / 4: what held 63.5 was rounded to 64 first)
    assert abs(float(values_of(codes, scales)[0, 0, 2, 0]) - 4) < 1e-6
    plain_append(codes, scales, one, [0], 8)
    assert codes[0, 0, :3, 0].tolist() == [127, 16, 127] and abs(float(scales[0, 0, 0]) - 1 / 127) < 1e-9


def test_the_delta_rule_writes_what_was_asked_for():
    """With beta 1, a key of length 1 reads what it has just written; the state before it is otherwise left."""
    q = torch.zeros(3, 1, 8)
    q[0, 0, 0] = q[1, 0, 1] = q[2, 0, 0] = 1
    v = torch.randn(3, 1, 8)
    out, states, by, _ = plain_delta(q.half(), q.half(), v.half(), [0, 3], torch.zeros(3, 1), torch.ones(3, 1), 1.0)
    assert torch.equal(out, v.half().double()) and torch.equal(states[0, 0, 0], v[2, 0].half().double()) and torch.equal(states[0, 0, 1], v[1, 0].half().double())
    assert bool((by < 0.02).all())
