"""The operators of a serving step over a ragged batch of requests, and the work that their performance is measured on.

The requests of a batch are the segments of its packed token vector: request r owns the tokens offsets[r] .. offsets[r + 1] - 1.

  tables        page tables and slot maps from the requests' lengths: which page of the cache, and which slot in it, every new
                token gets (mmv_page_tables)
  append        the new tokens' keys and values written into their slots of the paged cache (mmv_cache_append)
  attention     one new token of every request against its keys and values in the paged cache (mmv_paged_attention)
  decay_prompt  linear attention with a decay for each head over the packed prompts of a batch (mmv_decay_attention)
  decay_step    the same recurrence for one token of every request (mmv_decay_step)

A case is a dict of plain values.  Lengths of requests run from `lo` to `hi` in equal steps of their logarithm, in an order that the
seed draws; with eight requests or more one of them is empty, as the free places of a batch are.
"""
import math
import random

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}
_SIZE = {"bf16": 2, "f16": 2, "e4m3": 1}
_E4M3_MOST = 448.0


def listed():
    def tables(name, n, page, lo, hi, new_lo, new_hi):
        return {"name": name, "op": "tables", "n": n, "page": page, "lo": lo, "hi": hi, "new_lo": new_lo, "new_hi": new_hi}

    def append(name, tokens, heads, dim, page, dtype, cache):
        return {"name": name, "op": "append", "tokens": tokens, "heads": heads, "dim": dim, "page": page, "dtype": dtype, "cache": cache}

    def attention(name, n, lo, hi, heads, group, dim, page, dtype, cache, window=0):
        return {"name": name, "op": "attention", "n": n, "lo": lo, "hi": hi, "heads": heads, "group": group, "dim": dim, "page": page,
                "dtype": dtype, "cache": cache, "window": window}

    def decay(name, op, n, lo, hi, heads, group, dk, dv):
        return {"name": name, "op": op, "n": n, "lo": lo, "hi": hi, "heads": heads, "group": group, "dk": dk, "dv": dv}

    return [
        # every step of a decoding batch: one new token each, a new page now and then; latency counts
        tables("tables_decode", 256, 16, 1, 8000, 1, 1),
        # a batch of prompts that comes in at once, some of them behind a prefix that is cached already
        tables("tables_prompts", 100, 16, 1, 2000, 100, 8000),
        # a decoding batch's keys and values, sliced from the fused projection
        append("append_decode", 256, 8, 128, 16, "bf16", "bf16"),
        # a batch of prompts into a cache of 8-bit values
        append("append_prompts_e4m3", 16385, 8, 128, 64, "bf16", "e4m3"),
        # one user's next token behind a page or two of text
        attention("attention_one_request", 1, 1000, 1000, 8, 4, 128, 16, "bf16", "bf16"),
        # the ordinary batch: ragged lengths, grouped heads
        attention("attention_batch", 48, 64, 8192, 8, 4, 128, 16, "bf16", "bf16"),
        # as many key heads as query heads, short heads, a sliding window
        attention("attention_window_f16", 24, 17, 3001, 16, 1, 64, 32, "f16", "f16", window=1024),
        # long documents in a cache of 8-bit values
        attention("attention_long_e4m3", 16, 4096, 65536, 8, 8, 128, 64, "bf16", "e4m3"),
        # a few short prompts
        decay("decay_prompts_short", "decay_prompt", 3, 100, 700, 8, 1, 64, 64),
        # a batch of prompts from short ones to a whole document, the largest of which has half of all tokens
        decay("decay_prompts_long", "decay_prompt", 12, 64, 32768, 16, 1, 128, 128),
        # the next token of a few requests
        decay("decay_step_few", "decay_step", 4, 1, 1, 8, 1, 64, 64),
        # the next token of a large batch
        decay("decay_step_batch", "decay_step", 128, 1, 1, 32, 1, 128, 128),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["tables", "append", "attention", "attention", "decay_prompt", "decay_step"])
    if op == "tables":
        new_hi = rng.choice([1, log(2, 9000)])
        return {"op": op, "n": log(1, 1000 if new_hi == 1 else 150), "page": rng.choice([8, 16, 32, 64, 128, 256]), "lo": 1, "hi": log(2, 20000),
                "new_lo": 1, "new_hi": new_hi}
    if op == "append":
        dtype = rng.choice(["bf16", "f16"])
        return {"op": op, "tokens": log(1, 16000), "heads": rng.choice([1, 2, 4, 8]), "dim": rng.choice([64, 72, 80, 112, 128, 160, 256]),
                "page": rng.choice([8, 16, 32, 64]), "dtype": dtype, "cache": rng.choice([dtype, "e4m3"])}
    if op == "attention":
        n, heads, dim, dtype = log(1, 128), rng.choice([1, 2, 4, 8]), rng.choice([64, 72, 80, 112, 128, 160, 256]), rng.choice(["bf16", "f16"])
        most = max(40, min(40000, 8_000_000 // (n * heads)))
        hi = log(20, most)
        return {"op": op, "n": n, "lo": max(1, log(1, hi)), "hi": hi, "heads": heads, "group": rng.choice([1, 2, 4, 5, 7, 8, 16]), "dim": dim,
                "page": rng.choice([8, 16, 32, 64, 128]), "dtype": dtype, "cache": rng.choice([dtype, dtype, "e4m3"]),
                "window": rng.choice([0, 0, 0, log(1, hi)])}
    heads = rng.choice([2, 4, 8, 16])
    group = rng.choice([g for g in (1, 1, 2, 4) if g <= heads])
    if op == "decay_prompt":
        n, heads = log(1, 40), heads
        hi = log(2, min(30000, 400_000 // n))
        return {"op": op, "n": n, "lo": max(1, log(1, hi)), "hi": hi, "heads": heads, "group": group, "dk": rng.choice([64, 80, 128]),
                "dv": rng.choice([64, 112, 128, 160, 256])}
    return {"op": op, "n": log(1, 200), "lo": 1, "hi": 1, "heads": heads, "group": group, "dk": rng.choice([64, 80, 128]), "dv": rng.choice([64, 112, 128, 160, 256])}


def _lengths(n, lo, hi, empty=True):
    got = [int(round(lo * (hi / lo) ** ((i + 0.5) / n))) for i in range(n)]
    if empty and n >= 8:
        got[0] = 0
    return got


def _pages(lengths, page):
    return [(x + page - 1) // page for x in lengths]


def work(case):
    c = case
    if c["op"] == "tables":
        # lengths, tables' partial pages and the pages taken read; slots, positions, offsets, contexts and new table entries written
        new, old = _lengths(c["n"], c["new_lo"], c["new_hi"], c["new_hi"] > 1), _lengths(c["n"], c["lo"], c["hi"])
        taken = sum((a + b + c["page"] - 1) // c["page"] for a, b in zip(old, new)) - sum(_pages(old, c["page"]))
        return {"bytes": 24.0 * c["n"] + 8.0 * taken + 12.0 * sum(new), "flops": 10.0 * sum(new)}
    if c["op"] == "append":
        values = 2.0 * c["tokens"] * c["heads"] * c["dim"]
        return {"bytes": values * (_SIZE[c["dtype"]] + _SIZE[c["cache"]]) + 8.0 * c["tokens"], "flops": 2.0 * values}
    if c["op"] == "attention":
        lengths = [min(x, c["window"] or x) for x in _lengths(c["n"], c["lo"], c["hi"])]
        rows = 1.0 * sum(lengths) * c["heads"]
        small = 2.0 * c["n"] * c["heads"] * c["group"] * c["dim"] * _SIZE[c["dtype"]] + 4.0 * sum(_pages(lengths, c["page"]))
        return {"bytes": 2.0 * rows * c["dim"] * _SIZE[c["cache"]] + small, "flops": 4.0 * rows * c["group"] * c["dim"]}
    key_heads = c["heads"] // c["group"]
    tokens = sum(_lengths(c["n"], c["lo"], c["hi"])) if c["op"] == "decay_prompt" else c["n"]
    vectors = 2.0 * tokens * (c["heads"] * (c["dk"] + c["dv"]) + key_heads * (c["dk"] + c["dv"]))
    states = 8.0 * c["n"] * c["heads"] * c["dk"] * c["dv"]
    return {"bytes": vectors + states, "flops": 4.0 * tokens * c["heads"] * c["dk"] * c["dv"]}


# ---- inputs -------------------------------------------------------------------------------------------------------


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def _shuffled(values, seed):
    random.Random(seed).shuffle(values)
    return values


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.bfloat16, by=1.0):
        return (torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32 if dtype == torch.float32 else torch.bfloat16) * by).to(dtype)

    def permuted(n):
        return torch.randperm(n, generator=g, device="cuda").to(torch.int32)

    def cache(pages, scale):
        values = normal(pages, c["heads"], c["page"], c["dim"])
        if c["cache"] != "e4m3":
            return values.to(_DT[c["cache"]])
        return (values * (1.0 / scale)).clamp(-_E4M3_MOST, _E4M3_MOST).to(_DT["e4m3"])

    s = {"case": c}
    if c["op"] == "tables":
        old = _shuffled(_lengths(c["n"], c["lo"], c["hi"]), seed)
        new = _shuffled(_lengths(c["n"], c["new_lo"], c["new_hi"], c["new_hi"] > 1), seed + 1)
        held, need = _pages(old, c["page"]), _pages([a + b for a, b in zip(old, new)], c["page"])
        ids = permuted(sum(need) + 64)  # the pool: pages in use, in no order, and free ones
        table = torch.full((c["n"], (max(old) + max(new)) // c["page"] + 3), -1, dtype=torch.int32, device="cuda")
        width = torch.arange(table.shape[1], device="cuda")[None, :] < _ints(held)[:, None]
        table[width] = ids[:sum(held)]
        # room for a whole batch's new tokens, as a program has that captures its steps
        s |= {"cached": _ints(old), "new": _ints(new), "table": table, "free": ids[sum(held):].contiguous(), "max_tokens": sum(new) + (7 if sum(new) > 64 else 0)}
    elif c["op"] == "append":
        t, heads, d = c["tokens"], c["heads"], c["dim"]
        fused = normal(t, 3 * heads * d, dtype=_DT[c["dtype"]])  # q, k and v side by side
        s["k"], s["v"] = (fused[:, i * heads * d:(i + 1) * heads * d].unflatten(1, (heads, d)) for i in (1, 2))
        s["k_scale"], s["v_scale"] = (0.017, 0.02) if c["cache"] == "e4m3" else (1.0, 1.0)
        pages = t // c["page"] + 5
        s["k_cache"], s["v_cache"] = cache(pages, s["k_scale"]), cache(pages, s["v_scale"])
        slots = torch.arange(t, device="cuda")
        if t <= 1000:  # tokens of as many requests: anywhere
            slots = torch.randperm(pages * c["page"], generator=g, device="cuda")[:t]
        else:  # a prompt's tokens: pages in no order
            slots = permuted(pages).long()[slots // c["page"]] * c["page"] + slots % c["page"]
        if t > 8:  # tokens that pad the batch have no slot
            slots[t - 3:] = -1
        s["slots"] = slots
    elif c["op"] == "attention":
        lengths = _shuffled(_lengths(c["n"], c["lo"], c["hi"]), seed)
        counts = _pages(lengths, c["page"])
        s["k_scale"], s["v_scale"] = (0.017, 0.02) if c["cache"] == "e4m3" else (1.0, 1.0)
        pages = sum(counts) + 3
        s["k_cache"], s["v_cache"] = cache(pages, s["k_scale"]), cache(pages, s["v_scale"])
        table = torch.full((c["n"], max(counts) + 2), -1, dtype=torch.int32, device="cuda")
        table[torch.arange(table.shape[1], device="cuda")[None, :] < _ints(counts)[:, None]] = permuted(pages)[:sum(counts)]
        heads = c["heads"] * c["group"]
        fused = normal(c["n"], (heads + 2 * c["heads"]) * c["dim"], dtype=_DT[c["dtype"]], by=1.5)
        s |= {"table": table, "context": _ints(lengths), "q": fused[:, :heads * c["dim"]].unflatten(1, (heads, c["dim"])), "scale": c["dim"] ** -0.5}
    else:
        n, heads, kv, dk, dv = c["n"], c["heads"], c["heads"] // c["group"], c["dk"], c["dv"]
        lengths = _shuffled(_lengths(n, c["lo"], c["hi"]), seed) if c["op"] == "decay_prompt" else [1] * n
        t = sum(lengths)
        s["q"], s["k"], s["v"] = normal(t, heads, dk), normal(t, kv, dk), normal(t, kv, dv)
        s["log_decay"] = torch.tensor([-2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)], device="cuda")
        s["scale"] = dk ** -0.5
        s["index"] = permuted(n + 2)[:n].contiguous()
        s["state_in"], s["state_out"] = normal(n + 2, heads, dk, dv, dtype=torch.float32), torch.zeros(n + 2, heads, dk, dv, device="cuda")
        if c["op"] == "decay_prompt":
            ends = [0]
            for x in lengths:
                ends.append(ends[-1] + x)
            s |= {"offsets": _ints(ends), "longest": max(lengths)}
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------


def run(state):
    op = state["case"]["op"]
    if own:
        return {"tables": _own_tables, "append": _own_append, "attention": _own_attention, "decay_prompt": _own_decay_prompt, "decay_step": _own_decay_step}[op](state)
    return {"tables": _plain_tables, "append": _plain_append, "attention": _plain_attention, "decay_prompt": _plain_decay_prompt,
            "decay_step": _plain_decay_step}[op](state)


def _binding():
    from paper_2506_23906_amd import binding
    return binding


def _kept(s, key, make):
    """What a program makes once and keeps: workspaces, outputs, the description of its cache."""
    if key not in s:
        s[key] = make()
    return s[key]


def _own_tables(s):
    B, n, t = _binding(), s["case"]["n"], s["max_tokens"]
    out = _kept(s, "out", lambda: B.PageTables(*(torch.empty(k, dtype=d, device="cuda") for k, d in (
        (n + 1, torch.int32), (n, torch.int32), (t, torch.int64), (t, torch.int32), (2, torch.int64)))))
    ws = _kept(s, "ws", lambda: B.workspace(B.mmv_page_tables_workspace_bytes(n)))
    B.mmv_page_tables(s["cached"], s["new"], s["free"], s["table"], s["case"]["page"], t, out=out, ws=ws)
    return {"offsets": out.offsets, "context": out.context, "slots": out.slots, "positions": out.positions, "used": out.used, "table": s["table"]}


def _own_append(s):
    B = _binding()
    cache = _kept(s, "cache", lambda: B.PagedCache(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"]))
    B.mmv_cache_append(s["k"], s["v"], s["slots"], cache)
    return {"k": s["k_cache"], "v": s["v_cache"]}


def _own_attention(s):
    B, c, q = _binding(), s["case"], s["q"]
    cache = _kept(s, "cache", lambda: B.PagedCache(s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"]))
    out = _kept(s, "out", lambda: torch.empty(q.shape, dtype=q.dtype, device="cuda"))
    lse = _kept(s, "lse", lambda: torch.empty(q.shape[:2], dtype=torch.float32, device="cuda"))
    ws = _kept(s, "ws", lambda: B.workspace(B.mmv_paged_attention_workspace_bytes(c["n"], q.shape[1], c["heads"], c["dim"], s["table"].shape[1] * c["page"])))
    B.mmv_paged_attention(q, cache, s["table"], s["context"], scale=s["scale"], window=c["window"], out=out, lse=lse, ws=ws)
    return {"out": out, "lse": lse}


def _own_decay_prompt(s):
    B, c, q, v = _binding(), s["case"], s["q"], s["v"]
    out = _kept(s, "out", lambda: torch.empty(q.shape[0], q.shape[1], v.shape[2], dtype=q.dtype, device="cuda"))
    ws = _kept(s, "ws", lambda: B.workspace(B.mmv_decay_attention_workspace_bytes(c["n"], q.shape[0], c["heads"], c["dk"], c["dv"])))
    B.mmv_decay_attention(q, s["k"], v, s["offsets"], s["log_decay"], scale=s["scale"], state_in=s["state_in"], state_out=s["state_out"],
                          state_index=s["index"], out=out, ws=ws)
    return {"out": out, "state": s["state_out"]}


def _own_decay_step(s):
    B, q, v = _binding(), s["q"], s["v"]
    out = _kept(s, "out", lambda: torch.empty(q.shape[0], q.shape[1], v.shape[2], dtype=q.dtype, device="cuda"))
    B.mmv_decay_step(q, s["k"], v, s["log_decay"], s["state_in"], s["state_out"], scale=s["scale"], state_index=s["index"], out=out)
    return {"out": out, "state": s["state_out"]}


def _plain_tables(s):
    page, t, table = s["case"]["page"], s["max_tokens"], s["table"]
    cached, new = s["cached"].long(), s["new"].long()
    end = torch.cumsum(new, 0)
    held, need = (cached + page - 1) // page, (cached + new + page - 1) // page
    taken = torch.cumsum(need - held, 0)
    token = torch.arange(t, device="cuda")
    live = token < end[-1]
    r = torch.searchsorted(end, token, right=True).clamp(max=len(new) - 1)
    position = cached[r] + token - (end - new)[r]
    where = (position // page).clamp(max=table.shape[1] - 1)
    fresh = where >= held[r]
    first_free = (taken - (need - held))[r] + where - held[r]
    at = torch.where(fresh, s["free"][first_free.clamp(0, len(s["free"]) - 1)], table[r, where]).long()
    opens = live & fresh & (position % page == 0)
    entries = torch.cat([table.reshape(-1), table.new_zeros(1)])
    entries[torch.where(opens, r * table.shape[1] + where, table.numel())] = at.int()
    minus = torch.full_like(position, -1)
    return {"offsets": torch.cat([end.new_zeros(1), end]).int(), "context": (cached + new).int(),
            "slots": torch.where(live, at * page + position % page, minus), "positions": torch.where(live, position, minus).int(),
            "used": torch.stack([taken[-1], end[-1]]), "table": entries[:-1].view_as(table)}


def _plain_append(s):
    c, found, live = s["case"], {}, s["slots"] >= 0
    at = torch.where(live, s["slots"], s["slots"][0])  # (tokens without a slot, which only come last, do what the first one does again)
    page, slot = at // c["page"], at % c["page"]
    for x in "kv":
        cache, values = s[x + "_cache"], torch.where(live[:, None, None], s[x], s[x][:1])
        if c["cache"] == "e4m3":
            values = (values.float() * (1.0 / s[x + "_scale"])).clamp(-_E4M3_MOST, _E4M3_MOST).to(cache.dtype).view(torch.uint8)
        raw = cache.view(torch.uint8) if c["cache"] == "e4m3" else cache
        raw[page, :, slot] = values
        found[x] = cache
    return found


def _gathered(s, x):
    """Keys or values of every request in fp32, [requests, heads, positions, dim]."""
    cache, table = s[x + "_cache"], s["table"].clamp(min=0).long()
    pages = cache.view(torch.uint8)[table].view(cache.dtype) if cache.dtype == _DT["e4m3"] else cache[table]
    return pages.transpose(1, 2).flatten(2, 3).float()


def _plain_attention(s):
    c, q = s["case"], s["q"]
    q = q.float().unflatten(1, (c["heads"], c["group"]))
    scores = (q @ _gathered(s, "k").transpose(2, 3)) * (s["scale"] * s["k_scale"])
    position, context = torch.arange(scores.shape[3], device="cuda"), s["context"][:, None]
    seen = position < context
    if c["window"]:
        seen = seen & (position >= context - c["window"])
    scores = scores.masked_fill(~seen[:, None, None, :], -math.inf)
    most = scores.amax(3, keepdim=True)
    weights = torch.exp(scores - torch.where(most == -math.inf, 0.0, most))
    total = weights.sum(3, keepdim=True)
    out = (weights @ _gathered(s, "v")) * (s["v_scale"] / torch.where(total == 0, 1.0, total))
    return {"out": out.flatten(1, 2).to(s["q"].dtype), "lse": (most + torch.log(total)).flatten(1, 3)}


def _plain_decay_prompt(s):
    c, chunk = s["case"], 128
    n, heads, group = c["n"], c["heads"], c["group"]
    offsets, decay = s["offsets"].long(), s["log_decay"]
    length, chunks = offsets[1:] - offsets[:-1], -(-s["longest"] // chunk)
    position = torch.arange(chunks * chunk, device="cuda")
    live = position < length[:, None]
    at = torch.where(live, offsets[:-1, None] + position, 0)

    def padded(x):  # [requests, heads, chunks, chunk, dim]
        x = torch.where(live[:, :, None, None], x[at].float(), 0.0)
        return x.transpose(1, 2).unflatten(2, (chunks, chunk)).repeat_interleave(heads // x.shape[2], 1)

    q, k, v = padded(s["q"]), padded(s["k"]), padded(s["v"])
    inside = torch.arange(chunk, device="cuda")
    apart = inside[:, None] - inside[None, :]
    local = torch.where(apart >= 0, torch.exp(decay[:, None, None] * apart.clamp(min=0)), 0.0)
    out = ((q @ k.transpose(3, 4)) * local[None, :, None]) @ v
    # every chunk's own state at its end, and what has come in before it
    ends = torch.minimum((torch.arange(chunks, device="cuda") + 1) * chunk, length[:, None])
    left = (ends[:, :, None] - 1 - position.view(chunks, chunk)).clamp(min=0)
    own_state = (k * torch.exp(decay[None, :, None, None] * left[:, None])[..., None]).transpose(3, 4) @ v
    before = torch.arange(chunks, device="cuda")
    between = before[:, None] - before[None, :] - 1
    carry = torch.where(between >= 0, torch.exp(decay[:, None, None] * (between.clamp(min=0) * chunk)), 0.0)
    first = s["state_in"][s["index"].long()]
    came = torch.exp(decay[:, None] * (before * chunk))[None, :, :, None] * first.flatten(2)[:, :, None]
    came = (came + carry @ own_state.flatten(3)).unflatten(3, (c["dk"], c["dv"]))
    out = (out + torch.exp(decay[:, None] * (inside + 1))[None, :, None, :, None] * (q @ came)) * s["scale"]
    final = torch.exp(decay[None, :, None] * (length[:, None] - ends).clamp(min=0)[:, None]) * (before * chunk < length[:, None])[:, None]
    final = (final[:, :, None] @ own_state.flatten(3)).view(n, heads, c["dk"], c["dv"])
    final = final + torch.exp(decay[None, :] * length[:, None])[:, :, None, None] * first
    s["state_out"][s["index"].long()] = final
    token = torch.arange(s["q"].shape[0], device="cuda")
    r = torch.searchsorted(offsets[1:].contiguous(), token, right=True)
    out = out.flatten(2, 3).transpose(1, 2)[r, token - offsets[r]]
    return {"out": out.to(s["q"].dtype), "state": s["state_out"]}


def _plain_decay_step(s):
    group, index = s["case"]["group"], s["index"].long()
    q, k, v = s["q"].float(), s["k"].float().repeat_interleave(group, 1), s["v"].float().repeat_interleave(group, 1)
    state = s["state_in"][index] * torch.exp(s["log_decay"])[:, None, None] + k[..., :, None] * v[..., None, :]
    s["state_out"][index] = state
    out = (q[..., None, :] @ state)[..., 0, :] * s["scale"]
    return {"out": out.to(s["q"].dtype), "state": s["state_out"]}


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    return {"tables": _exact_tables, "append": _exact_append, "attention": _exact_attention, "decay_prompt": _exact_decay, "decay_step": _exact_decay}[case["op"]](s)


def _exact_tables(s):
    """Request by request, as a program on the host does it."""
    page, free, table = s["case"]["page"], s["free"].tolist(), s["table"].tolist()
    cached, new, taken = s["cached"].tolist(), s["new"].tolist(), 0
    offsets, slots, positions = [0], [], []
    for r, (old, more) in enumerate(zip(cached, new)):
        for p in range(old, old + more):
            if p % page == 0:
                table[r][p // page] = free[taken]
                taken += 1
            slots.append(table[r][p // page] * page + p % page)
            positions.append(p)
        offsets.append(offsets[-1] + more)
    blank = [-1] * (s["max_tokens"] - len(slots))
    return {"offsets": _ints(offsets), "context": _ints([a + b for a, b in zip(cached, new)]), "slots": _ints(slots + blank, torch.int64),
            "positions": _ints(positions + blank), "used": _ints([taken, offsets[-1]], torch.int64), "table": _ints(table)}


def _exact_append(s):
    found, keep = {}, (s["slots"] >= 0).nonzero()[:, 0]
    for x in "kv":
        rows = s[x + "_cache"].double().transpose(1, 2).flatten(0, 1)  # slot by slot
        values = s[x][keep].double()
        if s["case"]["cache"] == "e4m3":
            values = (values / s[x + "_scale"]).clamp(-_E4M3_MOST, _E4M3_MOST)
        rows[s["slots"][keep]] = values
        found[x] = rows.unflatten(0, (-1, s["case"]["page"])).transpose(1, 2).contiguous()
    return found


def _exact_attention(s):
    c, q = s["case"], s["q"].double()
    out, lse = torch.zeros_like(q), torch.full(q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for r, length in enumerate(s["context"].tolist()):
        if not length:
            continue
        start = max(0, length - c["window"]) if c["window"] else 0
        at = s["table"][r, :-(-length // c["page"])].long()
        for h in range(c["heads"]):
            k, v = ((s[x + "_cache"].view(torch.uint8)[at, h].view(s[x + "_cache"].dtype) if c["cache"] == "e4m3" else s[x + "_cache"][at, h]).double().flatten(0, 1)[start:length]
                    * s[x + "_scale"] for x in "kv")
            rows = slice(h * c["group"], (h + 1) * c["group"])
            scores = s["scale"] * (q[r, rows] @ k.T)
            lse[r, rows] = torch.logsumexp(scores, 1)
            out[r, rows] = torch.softmax(scores, 1) @ v
    return {"out": out, "lse": lse}


def _exact_decay(s):
    """Every output from all tokens before it, without a state in between."""
    c, q, k, v = s["case"], s["q"].double().transpose(0, 1), s["k"].double().transpose(0, 1), s["v"].double().transpose(0, 1)
    k, v = (x.repeat_interleave(c["group"], 0) for x in (k, v))
    decay, first, final = s["log_decay"].double()[:, None, None], s["state_in"].double(), s["state_out"].double()
    out = torch.empty(q.shape[0], q.shape[1], c["dv"], dtype=torch.float64, device="cuda")
    ends = s["offsets"].tolist() if c["op"] == "decay_prompt" else list(range(c["n"] + 1))
    for r, (a, b) in enumerate(zip(ends, ends[1:])):
        at, step = s["index"][r], 2048
        for i in range(a, b, step):
            e = min(b, i + step)
            row, col = torch.arange(i, e, device="cuda")[:, None], torch.arange(a, e, device="cuda")[None, :]
            weights = torch.exp(decay * (row - col).clamp(min=0)) * (row >= col) * (q[:, i:e] @ k[:, a:e].transpose(1, 2))
            out[:, i:e] = s["scale"] * (weights @ v[:, a:e] + torch.exp(decay * (row - a + 1)) * (q[:, i:e] @ first[at]))
        left = torch.arange(b - a, device="cuda").flip(0)[None, :, None]
        final[at] = torch.exp(decay * (b - a)) * first[at] + (k[:, a:b] * torch.exp(decay * left)).transpose(1, 2) @ v[:, a:b]
    return {"out": out.transpose(0, 1).contiguous(), "state": final}
