"""Plain forms of the calls of a serving step in 64 bits, on the CPU, and how far a result may be from them.

Every bound counts roundings: U[type] is the largest relative error of one rounding to the type, EPS that of one in fp32."""
import math

import torch

EPS = 2.0 ** -24
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
E4M3_MOST = 448.0


def plain_tables(cached, new, free, table, page, max_tokens):
    """Request by request; free pages and rows that are too short leave tokens without a slot."""
    table, free = [row[:] for row in table], list(free)
    offsets, slots, positions, taken = [0], [], [], 0
    for r, (old, more) in enumerate(zip(cached, new)):
        old, more = max(old, 0), max(more, 0)
        held, need = -(-old // page), -(-(old + more) // page)
        for p in range(old, old + more):
            w, slot = p // page, -1
            if w < len(table[r]):
                if w < held:
                    entry = table[r][w]
                else:
                    k = taken + w - held
                    entry = free[k] if k < len(free) else -1
                    if k < len(free) and p % page == 0 and len(slots) < max_tokens:
                        table[r][w] = entry
                slot = entry * page + p % page if entry >= 0 else -1
            slots.append(slot)
            positions.append(p)
        taken += need - held
        offsets.append(offsets[-1] + more)
    total = len(slots)
    slots, positions = (x[:max_tokens] + [-1] * (max_tokens - total) for x in (slots, positions))
    return {"offsets": offsets, "context": [max(a, 0) + max(b, 0) for a, b in zip(cached, new)], "slots": slots, "positions": positions,
            "used": [taken, total], "table": table}


def plain_attention(q, k, v, table, context, scale, window, k_scale=1.0, v_scale=1.0):
    """q [n, query heads, dim], k and v [pages, heads, slots, dim] (anything torch can make double of), table and context lists.  Returns
    out, lse, and the bounds of both: the scores are sums of dim products in fp32 (dim + 8 roundings of the sum of magnitudes), an
    exponential and the sum of L of them add L + 64 roundings and what the scores are off; probabilities are rounded to q's type once,
    and so is the result."""
    n, heads, dim = q.shape
    group, page, u = heads // k.shape[1], k.shape[2], U[q.dtype]
    q, kd, vd = q.double(), k.double() * k_scale, v.double() * v_scale
    out, lse = torch.zeros(n, heads, dim, dtype=torch.float64), torch.full((n, heads), -math.inf, dtype=torch.float64)
    out_by, lse_by = torch.zeros_like(out), torch.zeros_like(lse)
    for r in range(n):
        length = min(max(context[r], 0), len(table[r]) * page)
        begin = max(0, length - window) if window else 0
        at = [(table[r][p // page], p % page) for p in range(begin, length) if 0 <= table[r][p // page] < k.shape[0]]
        if not at:
            continue
        pages, places = torch.tensor([a for a, _ in at]), torch.tensor([b for _, b in at])
        for h in range(heads):
            kk, vv = kd[pages, h // group, places], vd[pages, h // group, places]
            s = scale * (kk @ q[r, h])
            off = float((dim + 8) * EPS * abs(scale) * (kk.abs() @ q[r, h].abs()).max())
            p = torch.softmax(s, 0)
            out[r, h], lse[r, h] = p @ vv, torch.logsumexp(s, 0)
            loose = 2 * off + (len(at) + 64) * EPS
            out_by[r, h] = (1 + 2 * u) * ((u + loose) * (p @ vv.abs()) + u * out[r, h].abs()) + 2.0 ** -24
            lse_by[r, h] = loose + 4 * EPS * abs(lse[r, h])
    return out, lse, out_by, lse_by


def plain_decay(q, k, v, ends, log_decay, scale, first=None):
    """q [tokens, heads, dk], k, v with their heads, ends the offsets; first: one state for each request, or None.  Token by token.  Returns out and
    final states and their bounds: of the terms of an output, each may have been rounded to q's type twice on its way (a score or a
    state that meets a matrix product, a key or value times its decay), the result once; fp32 sums over the tokens add a rounding
    for each, and the decay of each its own."""
    heads, group, u = q.shape[1], q.shape[1] // k.shape[1], U[q.dtype]
    q, k, v = q.double(), k.double().repeat_interleave(group, 1), v.double().repeat_interleave(group, 1)
    by = torch.exp(log_decay.double())[:, None, None]
    out = torch.zeros(q.shape[0], heads, v.shape[2], dtype=torch.float64)
    out_by, states, states_by = torch.zeros_like(out), [], []
    for r, (a, b) in enumerate(zip(ends, ends[1:])):
        S = torch.zeros(heads, q.shape[2], v.shape[2], dtype=torch.float64) if first is None else first[r].double()
        A = S.abs()
        for t in range(a, b):
            S = by * S + k[t][:, :, None] * v[t][:, None, :]
            A = by * A + (k[t][:, :, None] * v[t][:, None, :]).abs()
            out[t] = scale * (q[t][:, None, :] @ S)[:, 0]
            loose = 2 * u + (t - a + q.shape[2] + 64) * 2 * EPS
            out_by[t] = (1 + 2 * u) * (u * out[t].abs() + loose * abs(scale) * (q[t].abs()[:, None, :] @ A)[:, 0]) + 2.0 ** -24
        states.append(S)
        states_by.append((b - a + 64) * 2 * EPS * A)
    none = torch.zeros(0, heads, q.shape[2], v.shape[2], dtype=torch.float64)
    return out, torch.stack(states) if states else none, out_by, torch.stack(states_by) if states else none


def check(got, want, by, what):
    """Every value within its bound; what is infinite there is the same here."""
    got = got.detach().cpu().double()
    fine = torch.isfinite(want)
    assert got.shape == want.shape, what
    assert bool((got[~fine] == want[~fine]).all()), "%s: values that are not finite" % what
    off = (got[fine] - want[fine]).abs()
    bad = ~(off <= by[fine])
    assert not bool(bad.any()), "%s: %d of %d values off, the worst %.3g times its bound" % (what, int(bad.sum()), bad.numel(), float((off / by[fine]).max()))


def e4m3(x, scale):
    """What an 8-bit cache holds for the values x of 16 bits: fp32 product, clamp, rounding to the nearest (NaN stays)."""
    by = torch.tensor(1.0 / float(torch.tensor(scale, dtype=torch.float32)), dtype=torch.float32)
    return (x.float() * by).clamp(-E4M3_MOST, E4M3_MOST).to(torch.float8_e4m3fn)
