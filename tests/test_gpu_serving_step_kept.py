"""A captured step of paper_2506_23906_amd/serving_step.py as its requests grow, against a second server that runs every step eagerly."""
import pytest
import torch

from paper_2506_23906_amd import serving_step as M

pytestmark = pytest.mark.gpu


def servers(requests, longest, layers=2):
    shape = M.Shape(layers=layers, heads=4, dim=32, vocabulary=50, page=8)
    w = M.weights(shape, seed=5)
    return [M.Server(shape, w, requests, longest) for _ in range(2)]


def give(server, lengths, seed):
    tokens = torch.randint(50, (sum(lengths),), generator=torch.Generator().manual_seed(seed))
    server.prompts(tokens.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda"))


def same(a, b, x, y, what):
    torch.cuda.synchronize()
    assert torch.equal(a.table, b.table) and torch.equal(a.free, b.free) and torch.equal(a.cached, b.cached), what
    off = float((x.double() - y.double()).square().mean().sqrt() / y.double().square().mean().sqrt())
    assert off < 2.0 ** -6, (what, off)   # (the same kernels on the same values; products of the library may round otherwise in a graph)


def test_replays_of_requests_past_the_longest():
    """Pages are taken in five of the replays; eager work stands between them."""
    a, b = servers(4, 24)
    for s in (a, b):
        give(s, [23, 1, 9, 16], 1)
        s.step()
    a.capture()
    for i in range(23):
        x, y = a.replay().clone(), b.step()
        b.next.copy_(a.next)
        same(a, b, x, y, i)
        torch.ones(1000, device="cuda").sum().item()
    held = a.table[a.table >= 0].tolist()
    assert len(held) == len(set(held)) == 12 and a.cached.tolist() == [47, 25, 33, 40]


def test_replays_after_longer_prompts():
    """Prompts of many more tokens than before come in between a captured step and its replays; what they were given is given back to the allocator and written over."""
    a, b = servers(3, 200, layers=4)
    for s in (a, b):
        give(s, [2, 1, 1], 1)
        s.step()
    a.capture()
    for i in range(6):
        if i % 2 == 0:
            for s in (a, b):
                give(s, [10 + 20 * i, 20, 9], 2 + i)
            taken = [torch.full((1 << 20,), 0xFF, dtype=torch.uint8, device="cuda") for _ in range(32)]
            del taken
            b.next.copy_(a.next)
        x, y = a.replay().clone(), b.step()
        b.next.copy_(a.next)
        same(a, b, x, y, i)
