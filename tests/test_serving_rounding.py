"""The bounds of tests/serving_rounding.py notice a term that is left out.  No GPU: the mistake is planted in a plain form."""
import pytest
import torch

import serving_rounding as R

TYPES = [(R.BF16, R.BF16), (R.F16, R.F16), (R.BF16, R.E4M3), (R.F16, R.E4M3)]


@pytest.mark.parametrize("dtype,cache_type", TYPES)
def test_probabilities(dtype, cache_type):
    *_, weights, values, want, by = R.cancelling_probabilities(dtype, cache_type)
    off = [abs(float(R.split(weights, dtype, terms) @ values / weights.sum()) - want) for terms in (1, 2)]
    assert off[1] <= by / 4 and off[0] >= 4 * by


def test_probabilities_of_24_bits():
    *_, weights, values, want, by = R.probabilities_of_24_bits()
    off, held = [], torch.zeros_like(weights)
    for _ in range(3):
        left = weights - held
        off.append(abs(float((held + left.to(R.BF16).double()) @ values / weights.sum()) - want))     # this term rounded, the last one
        held = held + (left.float().view(torch.int32) & -65536).view(torch.float32).double()          # cut off, with one to follow
    assert off[2] <= by / 4 and off[1] >= 4 * by


@pytest.mark.parametrize("dtype", [R.BF16, R.F16])
@pytest.mark.parametrize("case", [R.cancelling_state, R.cancelling_scores])
def test_states_and_scores(case, dtype):
    *_, terms, want, by = case(dtype, 70)
    off = [abs(float(R.split(terms, R.BF16, n).sum()) - want) for n in (1, 2)]
    assert off[1] <= by / 4 and off[0] >= 4 * by


@pytest.mark.parametrize("dtype", [R.BF16, R.F16])
@pytest.mark.parametrize("tokens", [40, 700])
def test_decayed_values(tokens, dtype):
    *_, values, by_decay, by = R.decayed_values(dtype, tokens)
    off = [(R.split(values * by_decay, R.BF16, n) - values * by_decay).abs() / by for n in (2, 3)]
    assert float(off[1].max()) < 0.25 and float(off[0].max()) > 2


@pytest.mark.parametrize("first_value", [0.0, 1.0])
def test_flat_tail(first_value):
    """Probabilities as multiples of fp16's least value, with the largest at 1 and at 2^12."""
    *_, scale, want, by, _, _ = R.flat_tail(R.F16, first_value)
    n, p = (1 << 16) - 1, torch.exp(torch.tensor(-scale, dtype=torch.float64))
    got = [(first_value + n * float((p * 2.0 ** up).to(R.F16)) * 2.0 ** -up) / (1 + n * float(p)) for up in (0, 12)]
    assert abs(got[1] - want) <= by / 2 and abs(got[0] - want) > by


def test_flat_tail_sum():
    """Weights that one lane adds up (8 of every 32) in 32 bits: one by one beside the first one, and by 256."""
    *_, scale, _, _, want, by = R.flat_tail(R.BF16, 1.0)
    weights = torch.exp(torch.full((1 << 14,), -scale, dtype=torch.float64)).float()
    weights[0] = 1.0
    rest = 3 * (1 << 14) * float(weights[1])
    one_by_one = torch.zeros(())
    for w in weights:
        one_by_one = one_by_one + w
    by_256 = torch.zeros(())
    for part in weights.view(-1, 256):
        own = torch.zeros(())
        for w in part:
            own = own + w
        by_256 = by_256 + own
    off = [abs(torch.log(torch.tensor(float(x) + rest, dtype=torch.float64)).item() - want) for x in (one_by_one, by_256)]
    assert off[0] > 4 * by and off[1] <= by
