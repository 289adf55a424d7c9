"""Which kernels the calls of a serving step launch, with the HIP run-time replaced by one that only writes them down (hip_recorder.c): no GPU."""
import re
import subprocess
import sys
import textwrap

import pytest

from conftest import ROOT

A, WS = 0x10_0000_0000, 0x40_0000_0000


@pytest.fixture(scope="module")
def record(tmp_path_factory, libmmvseg_path):
    """record(call): the kernels of a call (an expression on `lib` and the helpers below), with their workgroups."""
    so = str(tmp_path_factory.mktemp("hip") / "libhip_recorder.so")
    subprocess.run(["gcc", "-shared", "-fPIC", "-O1", "-Wall", "-o", so, "tests/hip_recorder.c"], cwd=ROOT, check=True, timeout=120)
    child = textwrap.dedent("""
        import ctypes, sys
        rec = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
        rec.recorder_log.restype = ctypes.c_char_p
        lib = ctypes.CDLL(sys.argv[2])
        u64, vp, size, f32 = ctypes.c_uint64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float
        class Cache(ctypes.Structure):
            _fields_ = [("k", vp), ("v", vp), ("type", ctypes.c_int), ("page", ctypes.c_uint32), ("heads", ctypes.c_uint32), ("dim", ctypes.c_uint32), ("pages", u64),
                        ("a", u64), ("b", u64), ("c", u64), ("ks", f32), ("vs", f32)]
        a, ws = vp(%d), (vp(%d), size(1 << 40), None)
        def tables(n, tokens):
            return lib.mmv_page_tables(u64(n), a, a, a, u64(9), a, u64(8), u64(8), 16, u64(tokens), a, a, a, a, a, *ws)
        def cache(heads=8, dim=128, page=16, pages=1000, type=2):
            return ctypes.byref(Cache(a, a, type, page, heads, dim, pages, heads * page * dim, page * dim, dim, 1.0, 1.0))
        def append(tokens, heads=8):
            return lib.mmv_cache_append(u64(tokens), a, u64(heads * 128), a, u64(heads * 128), 2, a, cache(heads), None)
        def attention(n, width, heads=8, group=4, window=0):
            return lib.mmv_paged_attention(u64(n), heads * group, a, u64(heads * group * 128), 2, cache(heads), a, u64(width), u64(width), a, f32(1), window, a, a, *ws)
        def decay(n, tokens, heads=8, dk=64, dv=64):
            return lib.mmv_decay_attention(u64(n), u64(tokens), heads, heads, dk, dv, a, u64(heads * dk), a, u64(heads * dk), a, u64(heads * dv), 2, a, a, f32(1), a, a, u64(n), None, a, *ws)
        def step(n, heads=8, dk=64, dv=64):
            return lib.mmv_decay_step(u64(n), heads, heads, dk, dv, a, u64(heads * dk), a, u64(heads * dk), a, u64(heads * dv), 2, a, f32(1), a, a, u64(n), None, a, None)
        for call in sys.stdin.read().split(";"):
            rec.recorder_clear()
            print("status", eval(call))
            print(rec.recorder_log().decode(), end="")
            print("--", flush=True)
        """ % (A, WS))

    def run(call):
        res = subprocess.run([sys.executable, "-c", child, so, libmmvseg_path], input=call, capture_output=True, text=True, timeout=120)
        assert res.returncode == 0, res.stderr[-2000:]
        lines = res.stdout.split("--\n")[0].strip().split("\n")
        assert lines[0] == "status 0", res.stdout
        return [(re.search(r"\d+([a-z_]+_kernel)", line).group(1), *map(int, line.split()[2:])) for line in lines[1:]]
    return run


WHOLE, LIST, JOIN, PROMPT, BLOCKS = "whole_attention_kernel", "paged_attention_kernel", "join_attention_kernel", "decay_prompt_kernel", "decay_blocks_kernel"


@pytest.mark.parametrize("call,want", [
    ("tables(0, 0)", [("page_tables_kernel", 1, 256)]), ("tables(2048, 1000)", [("page_tables_kernel", 4, 256)]),
    ("tables(2049, 257)", [("sum_requests_kernel", 1, 1024), ("page_tables_kernel", 2, 256)]),
    ("append(0)", []), ("append(3)", [("cache_append_kernel", 2, 256)]),
    ("append(1 << 25)", [("cache_append_kernel", 8388607, 256)] * 2 + [("cache_append_kernel", 2, 256)]),   # (numbers of pieces below 2^31 in every launch)
    # segments of one tile (one wave writes them), of eight, of sixteen for each of which there is a table; longer ones in a list, which is joined
    ("attention(3, 2)", [(WHOLE, 24, 64)]), ("attention(3, 16)", [(WHOLE, 24, 512)]), ("attention(3, 32)", [(WHOLE, 24, 512)]),
    ("attention(3, 33)", [(LIST, 102, 256), (JOIN, 96, 256)]), ("attention(3, 1000)", [(LIST, 256, 256), (JOIN, 96, 256)]),
    # a window bounds them too; enough segments keep the device busy with longer ones; too many would come in rounds
    ("attention(3, 1000, window=225)", [(WHOLE, 24, 512)]), ("attention(40, 80)", [(WHOLE, 320, 512)]), ("attention(400, 80)", [(LIST, 256, 256), (JOIN, 12800, 128)]),
    ("attention(3, 2, heads=1, group=16)", [(WHOLE, 3, 64)]),
    ("decay(3, 256)", [(PROMPT, 24, 256)]), ("decay(3, 257)", [(PROMPT, 8 * 96, 256), (BLOCKS, 96, 256), (PROMPT, 8 * 96, 256)]),
    ("decay(3, 9000, 16, 128, 128)", [(PROMPT, 512, 512), (BLOCKS, 768, 256), (PROMPT, 512, 512)]), ("decay(3, 0)", [(PROMPT, 24, 256)]),
    ("decay(11, 9000, 16, 128, 128)", [(PROMPT, 1024, 512), (BLOCKS, 2816, 256), (PROMPT, 1024, 512)]),
    ("step(5)", [("decay_step_kernel", 40, 256)]),
])
def test_launches(record, call, want):
    assert record(call) == want
