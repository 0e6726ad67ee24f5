"""How far a cached value of the 8-bit cache may be from what was written, by the host's rules (that the GPU's calls
follow them to the bit is tested elsewhere).

A write rounds to the nearest code: 2^-4 of the value at most where the code is normal (2^-6 of the scale s and
up), else half of the code's step 2^-9 s, 2^-10 s.  When the scale grows to s', codes from 2^-6 s' on only change
their exponent; below, they are rounded to multiples of 2^-9 s', by 2^-10 s' at most.  Scales never shrink while a
page keeps its tokens, and at least double where they grow, so that over all growths up to s these sum to less than
2^-9 s: a value x ends up within 2^-4 |x| if |x| >= 2^-6 s (which rounding to nearest leaves at 2^-6 s or above), and
else within 2^-4 |x| + 2^-9 s."""
from __future__ import annotations

import random

import pytest
import torch

from pages8_sim import VALUES, codes


def bound(x, s):
    return torch.where(x.abs() >= 2.0 ** -6 * s, 2.0 ** -4 * x.abs(), 2.0 ** -4 * x.abs() + 2.0 ** -9 * s)


def counted_in(x, exps):
    """x written in 2^exps[0], whose scale then grows to each of the others in turn."""
    y = VALUES[codes(x * 2.0 ** -exps[0]).long()]
    for was, now in zip(exps, exps[1:]):
        y = VALUES[codes(y * 2.0 ** (was - now)).long()]
    return y * 2.0 ** exps[-1]


def every_value():
    """Every bf16 magnitude up to 448, and their negatives."""
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).double()
    return x[torch.isfinite(x) & (x.abs() <= 448)]


@pytest.mark.parametrize("up", list(range(0, 20)) + [60])
def test_one_growth(up):
    x = every_value()
    err = (counted_in(x, [0, up]) - x).abs()
    if up == 0:
        assert (err <= torch.maximum(2.0 ** -4 * x.abs(), torch.tensor(2.0 ** -10).double())).all()
    assert (err <= bound(x, 2.0 ** up)).all()


def test_many_growths():
    x, r = every_value(), random.Random(1)
    chains = [list(range(15)), list(range(0, 15, 2)), list(range(0, 16, 3))]
    for _ in range(150):
        chains.append(sorted(r.sample(range(0, 17), r.randint(2, 9))))
    for exps in chains:
        s = 2.0 ** exps[-1]
        assert ((counted_in(x * 2.0 ** exps[0], exps) - x * 2.0 ** exps[0]).abs() <= bound(x * 2.0 ** exps[0], s)).all(), exps


def test_a_grown_page_passes_the_bound_of_one_write():
    """3.359375 is 3.25 in steps of 1/4, and 3.0 when it comes to count in 2^8, in steps of 1/2."""
    x = torch.tensor([3.359375], dtype=torch.float64)
    got = counted_in(x, [0, 8])
    assert got.item() == 3.0
    assert (got - x).abs().item() > max(2.0 ** -4 * x.item(), 2.0 ** -10 * 2.0 ** 8)
    assert (got - x).abs().item() <= bound(x, 2.0 ** 8).item()
