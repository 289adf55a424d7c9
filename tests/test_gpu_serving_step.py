"""The model of paper_2506_23906_amd/serving_step.py: the calls of a step together, against their plain forms in the same places."""
import pytest
import torch

from paper_2506_23906_amd import serving_step as M
from serving_util import e4m3, plain_attention, plain_decay

pytestmark = pytest.mark.gpu


def plain_run(shape, w, sequences):
    """Hidden states of whole sequences: the projections as the model makes them (bf16 products on the GPU), what lies between in 64 bits on the CPU."""
    tokens = torch.tensor(sum(sequences, []), device="cuda")
    ends = [0]
    for s in sequences:
        ends.append(ends[-1] + len(s))
    x = w["embedding"][tokens]
    for i in range(shape.layers):
        kv = shape.kv_heads if i % 2 == 0 else shape.heads
        q, k, v = (t.cpu() for t in M.split(M.normalised(x) @ w["in"][i], shape, kv))
        if i % 2:
            o = plain_decay(q, k, v, ends, w["decay"].cpu(), shape.dim ** -0.5)[0]
        else:
            scale = 1.0
            if shape.cache == torch.float8_e4m3fn:
                k, v, scale = e4m3(k, shape.scale).float(), e4m3(v, shape.scale).float(), shape.scale
            rows = []
            for a, b in zip(ends, ends[1:]):   # every position is a page of its own here
                table = [[a + j if j <= p else -1 for j in range(b - a)] for p in range(b - a)]
                rows.append(plain_attention(q[a:b], k[:, :, None], v[:, :, None], table, [p + 1 for p in range(b - a)], shape.dim ** -0.5, 0, scale, scale)[0])
            o = torch.cat(rows)
        x = x + o.to(torch.bfloat16).cuda().flatten(1) @ w["out"][i]
    return x


@pytest.mark.parametrize("cache", [torch.bfloat16, torch.float8_e4m3fn])
def test_prompts_and_steps(cache):
    """Two layers, three requests: prompts, an eager step and three of a graph.  An operator's result and the plain one's are the same but for roundings to
    bf16, 2^-8 of a value each; a layer passes what its input is off on with a factor below 2 (the projections' entries are 0.5 / sqrt(width) at
    the end), and rounds four times: 2 * 2 * 4 * 2^-8 = 2^-4 of the root of the mean square bounds what the last layer's output is off."""
    shape = M.Shape(layers=2, heads=4, dim=32, vocabulary=50, page=8, cache=cache)
    w = M.weights(shape, seed=3)
    lengths = [1, 9, 23]
    sequences = [torch.randint(50, (n,), generator=torch.Generator().manual_seed(n)).tolist() for n in lengths]
    server = M.Server(shape, w, 3, 40)
    hidden = [list(part) for part in server.prompts(torch.tensor(sum(sequences, []), device="cuda"), torch.tensor(lengths, dtype=torch.int32, device="cuda")).cpu().split(lengths)]
    for i in range(4):
        for s, t in zip(sequences, server.next.tolist()):
            s.append(t)
        if i == 1:
            server.capture()       # (nothing runs while it is recorded)
        x = server.step() if i == 0 else server.replay()
        torch.cuda.synchronize()
        for part, row in zip(hidden, x.cpu()):
            part.append(row.clone())
    got, want = torch.cat([torch.stack(p) for p in hidden]).double(), plain_run(shape, w, sequences).cpu().double()
    off = (got - want).square().mean().sqrt() / want.square().mean().sqrt()
    assert server.cached.tolist() == [5, 13, 27] and float(off) < 2.0 ** -4, float(off)
    assert int((server.table >= 0).sum()) == 1 + 2 + 4


def test_pages_come_from_the_free_ones_alone():
    shape = M.Shape(layers=1, heads=4, dim=32, vocabulary=50, page=8)
    server = M.Server(shape, M.weights(shape), 5, 33)
    server.prompts(torch.zeros(5 * 8, dtype=torch.int64, device="cuda"), torch.full((5,), 8, dtype=torch.int32, device="cuda"))
    for _ in range(9):
        server.step()
    held = server.table[server.table >= 0].tolist()
    assert server.cached.tolist() == [17] * 5 and len(held) == len(set(held)) == 15
