"""Inputs whose exact results nearly cancel, so that every bit of what lies between shows, with bounds that count the roundings of each term and nothing more.

The matrix cores take 16-bit operands.  What meets them is split into two terms (a probability in fp16, a score, a state) or three (a probability in bf16, a value times its decay); the
bounds here hold for those splits and not if the last term is left out (tests/test_serving_rounding.py tries both on the CPU)."""
import math

import torch

from serving_util import EPS, U

BF16, F16, E4M3 = torch.bfloat16, torch.float16, torch.float8_e4m3fn
# Two terms: what the first leaves, cut off, is below 2^-7 (bf16), 2^-10 (fp16) of the value, and the second rounds that.  What keeps a probability's later
# terms from zero adds less than 2^-20 of it (bf16), or half of fp16's least value, 2^-36 of the largest probability.
TWO = {BF16: 2.0 ** -7 * U[BF16], F16: 2.0 ** -10 * U[F16]}
GUARD, LEAST = {BF16: 2.0 ** -20, F16: 0.0}, {BF16: 0.0, F16: 2.0 ** -36}


def split(x, dtype, terms):
    """What `terms` terms of a type stand for."""
    held = torch.zeros_like(x)
    for _ in range(terms):
        held = held + (x - held).to(dtype).double()
    return held


def cancelling_probabilities(dtype, cache_type, dim=64, page=16):
    """One row: a position of weight 1 and value 30, and 60 of value -1 whose weight is a little above 1/2, all but half a spacing of the type.  Returns q, k, v (on pages 0, 1, 2, ...),
    the scale, the weights and values, and a component's result and bound."""
    p = 0.5 * (1.0 + 0.95 * U[dtype])
    q, k, v = torch.zeros(1, 1, dim), torch.zeros(4, page, dim), torch.zeros(4, page, dim)
    q[..., 0], k.view(-1, dim)[1:61, 0] = 1.0, -1.0
    v.view(-1, dim)[0], v.view(-1, dim)[1:61] = 30.0, -1.0
    scale = float(torch.tensor(-math.log(p), dtype=torch.float32))
    weights, values = torch.tensor([1.0] + [math.exp(-scale)] * 60, dtype=torch.float64), v.view(-1, dim)[:61, 0].double()
    want = float(weights @ values / weights.sum())
    # (a score is one product, rounded twice before an exponential of a rounding or two; 61 weights are added up)
    by = (TWO[dtype] + GUARD[dtype] + (61 + 8) * EPS) * float(weights @ values.abs() / weights.sum()) + U[dtype] * abs(want) + LEAST[dtype] * 61 * 30
    return q.to(dtype), k[:, None].to(cache_type), v[:, None].to(cache_type), scale, weights, values, want, by


def probabilities_of_24_bits(dim=64, page=16):
    """The same for bf16's third term: seven positions whose sum cancels to 3e-6, and whose weights are 0.95 * 2^-17 from what two terms of 8 bits, the first cut off, can say."""
    p = 0.5 * (1.0 + (171 / 128 - 0.95 * 2.0 ** -8) * 2.0 ** -8)
    q, k, v = torch.zeros(1, 1, dim), torch.zeros(4, page, dim), torch.zeros(4, page, dim)
    q[..., 0], k.view(-1, dim)[1:7, 0] = 1.0, -1.0
    v.view(-1, dim)[0], v.view(-1, dim)[1:7] = 193 / 64, -1.0
    scale = float(torch.tensor(-math.log(p), dtype=torch.float32))
    weights, values = torch.tensor([1.0] + [math.exp(-scale)] * 6, dtype=torch.float64), v.view(-1, dim)[:7, 0].double()
    want = float(weights @ values / weights.sum())
    by = (2.0 ** -24 + 2.0 ** -29 + (7 + 8) * EPS) * float(weights @ values.abs() / weights.sum()) + U[BF16] * abs(want)
    return q.to(BF16), k[:, None].to(BF16), v[:, None].to(BF16), scale, weights, values, want, by


def flat_tail(dtype, first_value, dim=8, page=16, positions=1 << 16, below=25.3):
    """One position of weight 1 and 65535 of 2^-25.3 and value 1: the others' weight together is 1.6e-3.  Page 0 has the first 16, page 1 any 16 others.  Returns q, k, v, the scale,
    a component's result and bound, and lse with its bound."""
    q, k, v = torch.zeros(1, 1, dim), torch.zeros(2, 1, page, dim), torch.ones(2, 1, page, dim)
    q[..., 0], k[..., 0], k[0, 0, 0, 0], v[0, 0, 0] = 1.0, -1.0, 0.0, first_value
    scale = float(torch.tensor(below * math.log(2.0), dtype=torch.float32))
    tail = (positions - 1) * math.exp(-scale)
    want, size = (first_value + tail) / (1 + tail), (abs(first_value) + tail) / (1 + tail)
    # outputs: one rounding of what the tiles of 32 have come to for each; weights' sums: of up to 256 positions, and those of 64 such sums; scores of 25 in 32 bits
    by = U[dtype] * want + (TWO[dtype] + GUARD[dtype] + (positions / 32 + 64 + 4 * below) * EPS) * 2 * size + positions * LEAST[dtype]
    return q.to(dtype), k.to(dtype), v.to(dtype), scale, want, by, math.log1p(tail), (256 + 64 + 4 * below) * EPS


def cancelling_state(dtype, tokens, dk=16, dv=32):
    """A state of 1 + 0.95 * 2^-8 in one row and -1 in another, queries that are 1 at both, keys of zero, no decay.  The recurrence splits into bf16 terms, whatever its inputs are."""
    x = 1.0 + 0.95 * U[BF16]
    q, k, v = torch.zeros(tokens, 1, dk), torch.zeros(tokens, 1, dk), torch.ones(tokens, 1, dv)
    q[..., 3] = q[..., 9] = 1.0
    state = torch.zeros(1, 1, dk, dv)
    state[..., 3, :], state[..., 9, :] = x, -1.0
    terms = torch.tensor([float(state[0, 0, 3, 0]), -1.0], dtype=torch.float64)
    want = float(terms.sum())
    return q.to(dtype), k.to(dtype), v.to(dtype), state, terms, want, (TWO[BF16] + 16 * EPS) * 2.1 + U[dtype] * want


def cancelling_scores(dtype, tokens, dk=16, dv=32):
    """Two tokens whose scores with all that follow are 1 + 0.95 * 2^-8 and 1 and whose values are 1 and -1; no decay."""
    q, k, v = torch.zeros(tokens, 1, dk), torch.zeros(tokens, 1, dk), torch.zeros(tokens, 1, dv)
    q[..., 2] = q[..., 11] = 1.0
    k[0, 0, 2], k[0, 0, 11], k[1, 0, 2] = 1.0, 0.95 * U[BF16], 1.0
    v[0], v[1] = 1.0, -1.0
    q, k, v = q.to(dtype), k.to(dtype), v.to(dtype)
    terms = torch.tensor([float(k[0].double().sum()), -1.0], dtype=torch.float64)
    want = float(terms.sum())
    return q, k, v, terms, want, (TWO[BF16] + 16 * EPS) * 2.1 + U[dtype] * want


def decayed_values(dtype, tokens, log_decay=-1e-3, dk=16, dv=32):
    """One key of 1 at the first token: the final state's row is its value times all the decay since, to the bits of 32 (three terms of bf16: 2^-8 * 2^-8 * 2^-8, a few roundings of the
    exponential, whose argument is at most 1.5, and one for each of the blocks' states)."""
    q, k, v = torch.zeros(tokens, 1, dk), torch.zeros(tokens, 1, dk), torch.zeros(tokens, 1, dv)
    k[0, 0, 5] = 1.0
    v[0, 0] = torch.linspace(1.0, 1.99, dv)
    q, k, v = q.to(dtype), k.to(dtype), v.to(dtype)
    ld = float(torch.tensor(log_decay, dtype=torch.float32))
    values, by_decay = v[0, 0].double(), math.exp(ld * (tokens - 1))
    return q, k, v, torch.tensor([ld]), values, by_decay, 2.0 ** -20 * values * by_decay
