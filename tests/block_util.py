"""Plain forms, on the CPU, of the calls on a cache of 8-bit values with block scales and of the gated delta rule, and how far a result may be from them."""
import math

import torch

from serving_util import E4M3_MOST, EPS, U

MOST = {torch.int8: 127.0, torch.float8_e4m3fn: E4M3_MOST}
LEAST = 2.0 ** -100


def f32(x):
    """Rounded to 32 bits, as one operation of the definition is."""
    return x.float().double()


def codes_of(x, by, kind):
    """Codes of x * by: the product rounded to 32 bits, then to 8 (as doubles)."""
    x = f32(x * by)
    if kind == torch.int8:
        return x.clamp(-127, 127).round()
    return x.clamp(-E4M3_MOST, E4M3_MOST).float().to(torch.float8_e4m3fn).double()


def plain_append(codes, scales, x, slots, block):
    """codes [pages, heads, slots, dim] (int8 or e4m3) and scales [pages, heads, blocks], changed in place; x [tokens, heads, dim] of 16 bits; slots a list.  Run by run, in 64 bits
    with every operation of the definition rounded to 32.  Returns the (page, block) pairs that were written."""
    kind, page = codes.dtype, codes.shape[2]
    held = codes.double()
    largest = float(torch.finfo(x.dtype).max)
    values = x.double().clamp(-largest, largest)   # (NaN stays)
    total, t, touched = codes.shape[0] * page, 0, []
    while t < len(slots):
        if not 0 <= slots[t] < total:
            t += 1
            continue
        b, e = slots[t] // block, t
        while e < len(slots) and 0 <= slots[e] < total and slots[e] // block == b:
            e += 1
        p, i = b * block // page, b * block % page // block
        anew = any(s % block == 0 for s in slots[t:e])
        for h in range(codes.shape[1]):
            run = values[t:e, h]
            top = run.abs().nan_to_num(nan=0.0).max().clamp(min=LEAST)
            wanted = f32(top * f32(torch.tensor(1.0 / MOST[kind], dtype=torch.float64)))
            if kind == torch.int8 and bool(run.isnan().any()):
                wanted = torch.tensor(math.nan, dtype=torch.float64)
            before = scales[p, h, i].double()
            scale = wanted if anew or before < wanted else wanted if bool(wanted.isnan()) and not bool(before.isnan()) else before
            by = f32(1.0 / scale)
            rows = held[p, h, i * block:(i + 1) * block]
            if not anew and before < scale:
                rows.copy_(codes_of(rows, f32(before * by), kind))
            for j in range(t, e):
                rows[slots[j] % block] = codes_of(values[j, h], by, kind)
            scales[p, h, i] = scale.float()
        touched.append((p, i))
        t = e
    if kind == torch.int8:
        held = held.nan_to_num(nan=-127.0)   # (of blocks whose scale is none)
    codes.copy_(held.to(kind) if kind == torch.int8 else held.float().to(kind))
    return touched


def values_of(codes, scales):
    """What a cache stands for, in 64 bits."""
    blocks = codes.double().unflatten(2, (scales.shape[2], -1))
    return (blocks * scales.double()[..., None, None]).flatten(2, 3)


def plain_read(values, table, offsets, first, tokens, dtype, fill):
    """values [pages, heads, slots, dim] in 64 bits; table, offsets and first lists.  Code times scale is rounded to 32 bits and then to the type."""
    page, out = values.shape[2], torch.full((tokens, values.shape[1], values.shape[3]), fill, dtype=dtype)
    for r in range(len(offsets) - 1):
        for t in range(max(0, offsets[r]), min(tokens, offsets[r + 1])):
            p = first[r] + t - offsets[r]
            at = table[r][p // page] if 0 <= p // page < len(table[r]) else -1
            out[t] = values[at, :, p % page].float().to(dtype) if 0 <= at < values.shape[0] else 0.0
    return out


def plain_delta(q, k, v, ends, log_decay, beta, scale, first=None):
    """q, k [tokens, key heads, dk], v [tokens, heads, dv], ends the offsets; first: one state for each request, or None.  Token by token.  Returns out and final states and
    their bounds.

    A column s of a state is S' = e^g s, s <- S' + beta k (v - k S'), and I - beta k k^T does not lengthen it while beta |k|^2 <= 2: what a column is off, in 2-norm, decays with it
    and grows by what a token rounds.  That is, in units of fp32's EPS: 8 for the exponential and the product with it; for k S' and k u, sums of dk products, dk + 8 of |k| times what they
    add up; and in chunks of up to 64 tokens, where what a token writes comes from a triangular system, a sum of 64 products at most 2 (|v| + |k| |s|) each, to 24 bits both.  M is the largest
    |v| + |k| |s| of the request so far.  An output rounds the result, and terms of 16 bits (2^-16) of a state and of a score that meet q and what was written."""
    heads, group, u, dk = v.shape[1], v.shape[1] // k.shape[1], U[q.dtype], q.shape[2]
    q, k, v = q.double().repeat_interleave(group, 1), k.double().repeat_interleave(group, 1), v.double()
    out = torch.zeros(v.shape, dtype=torch.float64)
    out_by, states, states_by = torch.zeros_like(out), [], []
    for r, (a, b) in enumerate(zip(ends, ends[1:])):
        S = torch.zeros(heads, dk, v.shape[2], dtype=torch.float64) if first is None else first[r].double().clone()
        off, M = torch.zeros(heads, 1, v.shape[2], dtype=torch.float64), torch.zeros(heads, 1, v.shape[2], dtype=torch.float64)
        for t in range(a, b):
            by, kk, qq = torch.exp(log_decay[t].double().clamp(min=-200))[:, None, None], k[t][:, None, :], q[t][:, None, :]
            S = by * S
            size, length = S.norm(dim=1, keepdim=True), kk.norm(dim=2, keepdim=True)
            M = torch.maximum(M, v[t][:, None, :].abs() + length * size)
            S = S + kk.transpose(1, 2) * (beta[t].double()[:, None, None] * (v[t][:, None, :] - kk @ S))
            off = by * off + EPS * (16 * size + (dk + 8 + 3 * 64) * 2 * length * beta[t].double().abs()[:, None, None] * M)
            size, wide = S.norm(dim=1, keepdim=True), qq.norm(dim=2, keepdim=True)
            out[t] = scale * (qq @ S)[:, 0]
            out_by[t] = ((1 + 2 * u) * (u * out[t].abs() + abs(scale) * (wide * (off + (2.0 ** -15 + (dk + 8 + 64) * EPS) * (size + M)))[:, 0])) + 2.0 ** -24
        states.append(S)
        states_by.append((off + 2.0 ** -126).expand_as(S))
    none = torch.zeros(0, heads, dk, v.shape[2], dtype=torch.float64)
    return out, torch.stack(states) if states else none, out_by, torch.stack(states_by) if states else none
