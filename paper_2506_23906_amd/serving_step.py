"""A serving step that runs the calls for ragged batches together, as a small model with random weights.

The model has layers of two kinds, by turns: attention over a paged cache (16-bit, 8-bit with one scale, or 8-bit with a scale for each block of slots and head), and a recurrence, which is
linear attention with a decay for each head or the gated delta rule.  A batch of prompts goes in as one packed token vector, whose segments are the requests; after that every step adds one token to each request.

    python -m paper_2506_23906_amd.serving_step --requests 16 --prompt 300 --steps 64

prints the time of the prompts and of a decoding step, eager and as a HIP graph.
"""
from __future__ import annotations

import argparse
import math
import time
from typing import NamedTuple

import torch

from . import binding as B


class Shape(NamedTuple):
    layers: int = 4          # even ones: attention over the paged cache; odd ones: the recurrence
    heads: int = 8           # of queries; a quarter of them (one at least) of keys and values, in attention layers
    dim: int = 64
    vocabulary: int = 1000
    page: int = 16
    cache: torch.dtype = torch.bfloat16   # or float8_e4m3fn; in blocks int8 or float8_e4m3fn
    scale: float = 0.05      # of an 8-bit cache's keys and values, where it has one for all
    block: int = 0           # slots of a page that share a scale (a multiple of 8): an 8-bit cache in blocks
    recurrence: str = "decay"   # or "delta"

    @property
    def kv_heads(self) -> int:
        return max(1, self.heads // 4)

    @property
    def width(self) -> int:
        return self.heads * self.dim


def weights(shape: Shape, seed: int = 0, device="cuda") -> dict:
    """Random weights in bf16: a fused projection into queries, keys and values and one back for every layer, and the embedding."""
    g = torch.Generator().manual_seed(seed)

    def normal(*size, by):
        return (torch.randn(*size, generator=g) * by).to(torch.bfloat16).to(device)

    w = {"embedding": normal(shape.vocabulary, shape.width, by=1.0), "in": [], "out": []}
    for i in range(shape.layers):
        kv = shape.kv_heads if i % 2 == 0 else shape.heads
        w["in"].append(normal(shape.width, (shape.heads + 2 * kv) * shape.dim, by=shape.width ** -0.5))
        w["out"].append(normal(shape.width, shape.width, by=0.5 * shape.width ** -0.5))
    w["decay"] = torch.tensor([-(2.0 ** (-8.0 * (h + 1) / shape.heads)) for h in range(shape.heads)], device=device)
    if shape.recurrence == "delta":   # every token's decay and how much of its value is written, for each head
        w["gates"] = [normal(shape.width, 2 * shape.heads, by=shape.width ** -0.5) if i % 2 else None for i in range(shape.layers)]
    return w


def normalised(x: torch.Tensor) -> torch.Tensor:
    x = x.float()
    return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)).to(torch.bfloat16)


def unit(x: torch.Tensor) -> torch.Tensor:
    """Vectors of length 1 (the delta rule's keys and queries)."""
    y = x.float()
    return (y * torch.rsqrt(y.square().sum(-1, keepdim=True) + 1e-6)).to(x.dtype)


def gates(x: torch.Tensor, w: torch.Tensor, heads: int):
    """log_decay and beta of the delta rule, [tokens, heads] each, of normalised hidden states."""
    log_decay, beta = (x @ w).float().split(heads, dim=1)
    return -0.1 * torch.nn.functional.softplus(log_decay), torch.sigmoid(beta)


def split(fused: torch.Tensor, shape: Shape, kv: int):
    """Queries, keys and values of a fused projection, as views."""
    q, k, v = fused.split([shape.width, kv * shape.dim, kv * shape.dim], dim=1)
    return q.unflatten(1, (shape.heads, shape.dim)), k.unflatten(1, (kv, shape.dim)), v.unflatten(1, (kv, shape.dim))


class Server:
    """Caches, states, tables and workspaces of up to `requests` requests of up to `longest` positions (in whole pages), and the steps on them.  A request that steps past them keeps
    its pages and takes no others': its further tokens have no place in the cache, and see the positions that have."""

    def __init__(self, shape: Shape, w: dict, requests: int, longest: int, device="cuda"):
        self.shape, self.w, self.n, self.device = shape, w, requests, device
        self.columns = -(-longest // shape.page)
        pages = requests * (self.columns + 1)    # (a full request asks for one more in a step, at the end of a page; it is not given, but those behind it in the list go to the others)
        scale = shape.scale if shape.cache == torch.float8_e4m3fn else 1.0

        def cache():
            size = (pages, shape.kv_heads, shape.page, shape.dim)
            if shape.block:
                scales = (torch.zeros(pages, shape.kv_heads, shape.page // shape.block, device=device) for _ in "kv")
                return B.BlockCache(*(torch.zeros(size, dtype=torch.uint8, device=device).view(shape.cache) for _ in "kv"), *scales)
            return B.PagedCache(*(torch.zeros(size, dtype=torch.uint8 if shape.cache.itemsize == 1 else shape.cache, device=device).view(shape.cache) for _ in "kv"), scale, scale)

        self.caches = [cache() if i % 2 == 0 else None for i in range(shape.layers)]
        self.states = [None if i % 2 == 0 else torch.zeros(requests, shape.heads, shape.dim, shape.dim, device=device) for i in range(shape.layers)]
        self.table = torch.full((requests, self.columns), -1, dtype=torch.int32, device=device)
        self.free = torch.randperm(pages, generator=torch.Generator().manual_seed(1)).int().to(device)
        self.after = torch.empty_like(self.free)
        self.selected = torch.zeros(1, dtype=torch.int64, device=device)
        self.cached = torch.zeros(requests, dtype=torch.int32, device=device)
        self.one_each = torch.ones(requests, dtype=torch.int32, device=device)
        self.next = torch.zeros(requests, dtype=torch.int64, device=device)      # every request's newest token, which has no key and value yet
        self.graph = None
        self._kept = {}

    def _workspace(self, key, nbytes):
        """Scratch by its use; one that a step uses is never asked for in another size, since a captured step goes on using it."""
        if key not in self._kept or self._kept[key].numel() < nbytes:
            self._kept[key] = B.workspace(nbytes, self.device)
        return self._kept[key]

    def _tables(self, new, tokens):
        ws = self._workspace("tables", B.mmv_page_tables_workspace_bytes(self.n))
        return B.mmv_page_tables(self.cached, new, self.free, self.table, self.shape.page, tokens, ws=ws)

    def _took(self, tables):
        """Free pages that are in the table now leave the list, the others move up (-1 behind them: no page); the new tokens are cached ones."""
        pages = self.free.numel()
        gone = torch.zeros(pages + 1, dtype=torch.uint8, device=self.device)
        gone.scatter_(0, torch.where(self.table >= 0, self.table, pages).flatten().long(), 1)
        gone[pages:].fill_(1)
        free = 1 - gone[torch.where(self.free >= 0, self.free, pages).long()]
        if "free" not in self._kept:
            self._kept["free"] = B.new_workspace(B.MMV_OP_COMPRESS, B.MMV_I8_I32, B.MMV_FLAGS_U8, pages, self.device)
        self.after.fill_(-1)
        B.mmv_compress(self.free, free, pages, out=self.after, count=self.selected, ws=self._kept["free"])
        self.free.copy_(self.after)
        self.cached.copy_(tables.context)

    def _layers(self, use, tokens, tables, table, context, recurrence):
        shape, x = self.shape, self.w["embedding"][tokens]
        append, attention = (B.mmv_block_append, B.mmv_block_attention) if shape.block else (B.mmv_cache_append, B.mmv_paged_attention)
        for i in range(shape.layers):
            kv = shape.kv_heads if i % 2 == 0 else shape.heads
            y = normalised(x)
            q, k, v = split(y @ self.w["in"][i], shape, kv)
            if i % 2 == 0:
                append(k, v, tables.slots, self.caches[i])
                nbytes = B.mmv_paged_attention_workspace_bytes(q.shape[0], shape.heads, kv, shape.dim, self.columns * shape.page)
                o = attention(q, self.caches[i], table, context, ws=self._workspace("attention of " + use, nbytes))
            elif shape.recurrence == "delta":
                o = recurrence(unit(q), unit(k), v, self.states[i], *gates(y, self.w["gates"][i], shape.heads))
            else:
                o = recurrence(q, k, v, self.states[i])
            x = x + o.flatten(1) @ self.w["out"][i]
        return x

    def prompts(self, tokens: torch.Tensor, lengths: torch.Tensor) -> torch.Tensor:
        """The packed tokens of all requests' prompts (none of them empty, none that does not fit behind what is cached); returns every token's hidden state.  A token attends to
        those before it as a row of its own."""
        count, shape = tokens.numel(), self.shape
        if int((self.cached + lengths).max()) > self.columns * shape.page:
            raise ValueError("a prompt is longer than the pages of a request")
        tables = self._tables(lengths, count)
        request = torch.searchsorted(tables.offsets[1:].contiguous(), torch.arange(count, dtype=torch.int32, device=self.device), right=True)

        def recurrence(q, k, v, state, *gates):
            if gates:
                ws = self._workspace("recurrence of prompts", B.mmv_delta_attention_workspace_bytes(self.n, count, shape.heads, shape.dim, shape.dim))
                return B.mmv_delta_attention(q, k, v, tables.offsets, *gates, state_in=state, state_out=state, ws=ws)
            ws = self._workspace("recurrence of prompts", B.mmv_decay_attention_workspace_bytes(self.n, count, shape.heads, shape.dim, shape.dim))
            return B.mmv_decay_attention(q, k, v, tables.offsets, self.w["decay"], state_in=state, state_out=state, ws=ws)

        x = self._layers("prompts", tokens, tables, self.table[request], tables.positions + 1, recurrence)
        self.next.copy_((x[tables.offsets[1:].long() - 1] @ self.w["embedding"].T).argmax(-1))
        self._took(tables)
        return x

    def step(self) -> torch.Tensor:
        """One more token for every request; returns the hidden states, and leaves the next tokens in `next`."""
        tables = self._tables(self.one_each, self.n)

        def recurrence(q, k, v, state, *gates):
            return B.mmv_delta_step(q, k, v, *gates, state, state) if gates else B.mmv_decay_step(q, k, v, self.w["decay"], state, state)

        x = self._layers("a step", self.next, tables, self.table, tables.context, recurrence)
        self.next.copy_((x @ self.w["embedding"].T).argmax(-1))
        self._took(tables)
        return x

    def capture(self) -> None:
        """The step as a HIP graph (run one eager step before: it makes the workspaces)."""
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            self._kept["x"] = self.step()

    def replay(self) -> torch.Tensor:
        self.graph.replay()
        return self._kept["x"]


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--requests", type=int, default=16)
    ap.add_argument("--prompt", type=int, default=300, help="longest prompt; lengths are spread from a tenth of it")
    ap.add_argument("--steps", type=int, default=64)
    ap.add_argument("--cache", choices=["bf16", "e4m3", "e4m3-blocks", "int8-blocks"], default="bf16")
    ap.add_argument("--recurrence", choices=["decay", "delta"], default="decay")
    a = ap.parse_args()
    shape = Shape(cache={"bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}[a.cache.split("-")[0]], block=16 if a.cache.endswith("blocks") else 0, recurrence=a.recurrence)
    lengths = [max(1, round(a.prompt * 10 ** (i / max(1, a.requests - 1) - 1))) for i in range(a.requests)]
    server = Server(shape, weights(shape), a.requests, max(lengths) + 2 * a.steps + 3)
    tokens = torch.randint(shape.vocabulary, (sum(lengths),), generator=torch.Generator().manual_seed(3)).cuda()

    def timed(what, run, count):
        torch.cuda.synchronize()
        began = time.perf_counter()
        for _ in range(count):
            run()
        torch.cuda.synchronize()
        print("%-28s %9.1f us" % (what, (time.perf_counter() - began) / count * 1e6))

    timed("%d prompt tokens, first run" % len(tokens), lambda: server.prompts(tokens, torch.tensor(lengths, dtype=torch.int32, device="cuda")), 1)
    server.step()
    timed("a step, eager", server.step, a.steps)
    server.capture()
    timed("a step, as a graph", server.replay, a.steps)
    print("positions per request:", server.cached.tolist())


if __name__ == "__main__":
    main()
