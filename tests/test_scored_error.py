"""How far a biased score may be off, by the kernels' steps in 32 bits on the host: the score's products start from
the bias of the key's place in its tile, and the bias of the tile's first key joins less the reference.

With s = slope log2 e (2 roundings, the constant's included: (1 + 2^-2) 2^-24 of it), o the key's place in its tile
and D the distance of the tile's first key:
  - the accumulator starts at s o / c, three roundings, and adds d products: each step rounds what the bias
    has there, 63 slopes at most, so (3 + d) 63 2^-24 < 2^-11 + 2^-16 slopes;
  - s D and s D - ref round once each, the exponential's fma once more: 3 2^-24 of |slope D| and of the reference, which
    lies within some 10 of the row's largest score (2^-20 for those);
  - keys past their row, which a prefix shows, take 2 slope distance off: twice 2^-24 of that.
Together under 2^-10 |slope| + 2^-21 (|slope (i - j)| + |row's largest|) + 2^-20, beside the products' own error."""
from __future__ import annotations

import numpy as np
import pytest

F = np.float32


def kernel_score(dots, slope, places, dist0, ref, d):
    """log weights (64 bits, natural) of the keys at `places` of a tile whose first key lies at dist0 (j - i):
    dots [keys, d] fp32 products, ref in base-2 units."""
    log2e, c = F(1.4426950408889634), F(1.4426950408889634 / np.sqrt(d))
    inv_c = F(1) / c
    s = F(slope) * log2e
    acc = F(s * inv_c) * places.astype(F)
    for i in range(d):
        acc = (acc + dots[:, i]).astype(F)
    off = F(s * F(dist0)) - F(ref)
    return (np.float64(c) * acc.astype(np.float64) + np.float64(off)).astype(F).astype(np.float64) + np.float64(F(ref))


def exact_score(dots, slope, places, dist0, d):
    return (dots.astype(np.float64).sum(1) / np.sqrt(d) + np.float64(F(slope)) * (dist0 + places)) / np.log(2)


def errors(slope, dist, d, seed, ref_is):
    r = np.random.default_rng(seed)
    dots = (r.standard_normal((64, d)) * r.standard_normal((64, d))).astype(F)
    places = np.arange(64)
    dist0 = -(dist + 63)  # the tile's last key lies `dist` behind the row
    want = exact_score(dots, slope, places, dist0, d)
    largest = {"here": want.max(), "near": want.max() + 8.0, "own": 0.0}[ref_is]
    got = kernel_score(dots, slope, places, dist0, largest, d)
    products = d * 2.0 ** -24 * np.abs(dots).sum(1).max() / np.sqrt(d) + 2.0 ** -20
    bias = abs(slope) * (dist + 63.0)
    return (np.abs(got - want).max() * np.log(2), products,
            2.0 ** -10 * abs(slope) + 2.0 ** -21 * (bias + abs(largest) * np.log(2)))


SLOPES = [2.0 ** -8, 0.0123, 0.5, 0.84, 1.0, 3.7, 1024.0]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("slope", SLOPES)
@pytest.mark.parametrize("dist", [0, 1, 500, 8192, 131072, 1000003])
def test_the_bound(d, sign, slope, dist):
    for seed in range(3):
        for ref_is in ("here", "near", "own"):
            err, products, bias = errors(sign * slope, dist, d, seed, ref_is)
            assert err <= products + bias


def test_a_share_of_the_slope_alone_does_not_bound_it():
    """Far keys: a bias of 110,000 in 32 bits is not held to 2^-11 of a slope of 0.84."""
    far = [errors(-0.84, 131072 + x, 128, 0, "here") for x in range(0, 640, 64)]
    assert any(err > products + 2.0 ** -11 * 0.84 for err, products, _ in far)
