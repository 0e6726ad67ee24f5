"""Appends to several sequences of the 8-bit cache, some of which begin a page while others go on in one, by the host's
rules: whichever page that is, page 0 among them."""
from __future__ import annotations

import itertools

import pytest
import torch

from pages8_sim import Cache8
from test_gpu_pages8 import i32, put

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("going_on", [0, 5])
@pytest.mark.parametrize("order", list(itertools.permutations(range(3))))
def test_pages_begun_beside_a_page_that_goes_on(d, going_on, order):
    """Slot 0 goes on in page `going_on`, whose scale grows; slots 1 and 2 begin pages."""
    from paper_2505_11254_amd import binding
    c = Cache8(2, 8, 2, d, 3, 2, seed=d)
    put(c, 0, 20, [going_on])
    put(c, 1, 0, [])
    put(c, 2, 64, [3])
    c.ke[:, going_on], c.ve[:, going_on] = -3, 1
    dev = c.gpu8()
    slots, start = list(order), [[20, 0, 64][s] for s in order]
    want = [n + 6 for n in start]
    got = binding.pages8_resize(*dev, i32(slots), i32(want))
    assert got.cpu().tolist() == [list(x) for x in c.resize(slots, want)]
    g = torch.Generator().manual_seed(order[0])
    k, v = ((torch.randn((2, 18, 2, d), generator=g) * 2.0 ** 9).to(torch.bfloat16) for _ in range(2))
    binding.pages8_append(k.cuda(), v.cuda(), *dev[:6], slots=i32(slots), B=3)
    c.append8(slots, [0, 6, 12, 18], k, v)
    assert (c.ke[:, going_on] > -3).all()
    c.equal8(*dev)
