"""Which kernels the calls on a cache in blocks and of the gated delta rule launch, with the HIP run-time replaced by one that only writes them down (hip_recorder.c): no GPU."""
import re
import subprocess
import sys
import textwrap

import pytest

from conftest import ROOT

A, WS = 0x10_0000_0000, 0x40_0000_0000


@pytest.fixture(scope="module")
def record(tmp_path_factory, libmmvseg_path):
    """record(call): the kernels of a call (an expression on the helpers below), with their workgroups."""
    so = str(tmp_path_factory.mktemp("hip") / "libhip_recorder.so")
    subprocess.run(["gcc", "-shared", "-fPIC", "-O1", "-Wall", "-o", so, "tests/hip_recorder.c"], cwd=ROOT, check=True, timeout=120)
    child = textwrap.dedent("""
        import ctypes, sys
        rec = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
        rec.recorder_log.restype = ctypes.c_char_p
        lib = ctypes.CDLL(sys.argv[2])
        u64, vp, size, f32, u32 = ctypes.c_uint64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_float, ctypes.c_uint32
        class Cache(ctypes.Structure):
            _fields_ = [("k", vp), ("v", vp), ("ks", vp), ("vs", vp), ("type", ctypes.c_int), ("page", u32), ("heads", u32), ("dim", u32), ("block", u32), ("pages", u64), ("a", u64), ("b", u64), ("c", u64)]
        a, ws = vp(%d), (vp(%d), size(1 << 40), None)
        def cache(heads=8, dim=128, page=32, block=16, pages=1000, type=6):
            return ctypes.byref(Cache(a, a, a, a, type, page, heads, dim, block, pages, heads * page * dim, page * dim, dim))
        def append(tokens, heads=8, block=16, type=6):
            return lib.mmv_block_append(u64(tokens), a, u64(heads * 128), a, u64(heads * 128), 2, a, cache(heads, block=block, type=type), None)
        def read(tokens, n=3, heads=8, dim=128):
            return lib.mmv_block_read(u64(n), u64(tokens), a, a, a, u64(8), u64(8), cache(heads, dim), 1, a, u64(heads * dim), a, u64(heads * dim), None)
        def attention(n, width, heads=8, group=4, window=0):
            return lib.mmv_block_attention(u64(n), heads * group, a, u64(heads * group * 128), 2, cache(heads), a, u64(width), u64(width), a, f32(1), window, a, a, *ws)
        def delta(n, tokens, heads=8, dk=64, dv=64, type=2):
            return lib.mmv_delta_attention(u64(n), u64(tokens), heads, heads, dk, dv, a, u64(heads * dk), a, u64(heads * dk), a, u64(heads * dv), type, a, a, a, f32(1), a, a, u64(n), None, a, *ws)
        def step(n, heads=8, dk=64, dv=64):
            return lib.mmv_delta_step(u64(n), heads, heads, dk, dv, a, u64(heads * dk), a, u64(heads * dk), a, u64(heads * dv), 2, a, a, f32(1), a, a, u64(n), None, a, None)
        rec.recorder_clear()
        print("status", eval(sys.stdin.read()))
        print(rec.recorder_log().decode(), end="", flush=True)
        """ % (A, WS))

    def run(call):
        res = subprocess.run([sys.executable, "-c", child, so, libmmvseg_path], input=call, capture_output=True, text=True, timeout=120)
        assert res.returncode == 0, res.stderr[-2000:]
        lines = res.stdout.strip().split("\n")
        assert lines[0] == "status 0", res.stdout
        return [(re.search(r"\d+([a-z_]+_kernel)", line).group(1), *map(int, line.split()[2:])) for line in lines[1:]]
    return run


APPEND, READ, CHUNKS, PROMPT, STATES, STEP = "block_append_kernel", "block_read_kernel", "delta_chunks_kernel", "delta_prompt_kernel", "delta_states_kernel", "delta_step_kernel"
WHOLE, LIST, JOIN = "whole_attention_kernel", "paged_attention_kernel", "join_attention_kernel"


@pytest.mark.parametrize("call,want", [
    # few tokens: a wave for each, head and kind; more: for as many as a block holds, 32 at most
    ("append(0)", []), ("append(1)", [(APPEND, 4, 256)]), ("append(1024)", [(APPEND, 4096, 256)]), ("append(1025)", [(APPEND, 260, 256)]), ("append(3200, block=32)", [(APPEND, 400, 256)]),
    ("append(3200, block=8, type=5)", [(APPEND, 1600, 256)]), ("append((1 << 26) - 1, heads=1024)", [(APPEND, 16776704, 256)] * 128 + [(APPEND, 65536, 256)]),
    # a wave for a token, or for several where a token is less than a wave's pieces
    ("read(0)", []), ("read(1)", [(READ, 1, 256)]), ("read(9)", [(READ, 3, 256)]), ("read(100, heads=1, dim=64)", [(READ, 4, 256)]), ("read(100, heads=1, dim=8)", [(READ, 1, 256)]),
    ("read((1 << 31) - 1)", [(READ, (1 << 24) - 1, 256)] * 32 + [(READ, 32, 256)]),
    ("attention(3, 1)", [(WHOLE, 24, 64)]), ("attention(3, 16)", [(WHOLE, 24, 512)]), ("attention(3, 17)", [(LIST, 102, 256), (JOIN, 96, 256)]), ("attention(0, 1)", []),
    # chunks, then requests; where long ones may be taken apart, two launches for that, and as many workgroups as the device holds
    ("delta(3, 900)", [(CHUNKS, 136, 256), (PROMPT, 24, 512)]), ("delta(3, 0)", [(PROMPT, 24, 512)]), ("delta(0, 100)", []), ("delta(3, 960)", [(CHUNKS, 144, 256), (PROMPT, 24, 512)]),
    ("delta(3, 961)", [(CHUNKS, 144, 256), (PROMPT, 1024, 512), (STATES, 1024, 128), (PROMPT, 1024, 512)]),
    ("delta(700, 9000, dk=128, dv=256, type=1)", [(CHUNKS, 6720, 256), (PROMPT, 1024, 512), (STATES, 1024, 256), (PROMPT, 11200, 512)]),   # (128 columns to a workgroup)
    ("delta(3, 9000, heads=32, dk=96, dv=128)", [(CHUNKS, 4576, 256), (PROMPT, 1024, 512), (STATES, 1024, 192), (PROMPT, 1024, 512)]),
    ("delta(3, 9000, heads=64, dk=96, dv=128)", [(CHUNKS, 9152, 256), (PROMPT, 384, 512)]),   # (two of a head at once: nothing to gain)
    ("delta(63, 100, heads=8, dv=128)", [(CHUNKS, 512, 256), (PROMPT, 1008, 512)]), ("delta(64, 100, heads=8, dv=128)", [(CHUNKS, 520, 256), (PROMPT, 512, 512)]),   # the device filled twice
    ("step(5)", [(STEP, 40, 256)]), ("step(5, dv=256)", [(STEP, 40, 512)]),
])
def test_launches(record, call, want):
    assert record(call) == want


def test_workspaces_of_the_delta_rule(libmmvseg_path):
    """Bounded by the tokens: 31 KB for each chunk of a head that there can be, and the states of blocks."""
    from paper_2506_23906_amd import binding as B
    last = 0
    for tokens in (0, 1, 64, 65, 959, 961, 5000, 100_000, 10 ** 7):
        need = B.mmv_delta_attention_workspace_bytes(3, tokens, 16, 128, 128)
        chunks = tokens // 64 + min(3, tokens)
        assert need % 256 == 0 and need >= last and chunks * 16 * 31232 <= need <= chunks * 16 * 31232 + (32 * 16 * 128 * 256 * 4 if tokens > 960 else 0)
        last = need
