"""The error of values in the 8-bit cache on the GPU, against what was written: pages whose scales grow, by later
tokens and by tokens that move in, and pages that were cut back (the bound: test_pages8_error.py)."""
from __future__ import annotations

import random

import pytest
import torch

from paged_sim import PAGE, pages_of
from test_gpu_pages8 import i32
from test_pages8_error import bound

pytestmark = pytest.mark.gpu


class Slot:
    """A slot that all calls are made on, and the rows that went into it, in 64 bits."""

    def __init__(self, M, Hkv, d):
        P = M + 2
        self.kp, self.vp = (torch.zeros((P, Hkv, PAGE, d), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
                            for _ in range(2))
        self.ks, self.vs = (torch.full((P, Hkv), float("nan"), device="cuda") for _ in range(2))
        self.table, self.lens = torch.full((1, M), -1, dtype=torch.int32, device="cuda"), i32([0])
        self.refs = torch.zeros(P, dtype=torch.int32, device="cuda")
        self.k = self.v = torch.zeros((0, Hkv, d), dtype=torch.float64)

    def cache(self):
        return self.kp, self.vp, self.ks, self.vs, self.table, self.lens

    def resize(self, n):
        from paper_2505_11254_amd import binding
        assert binding.pages8_resize(*self.cache(), self.refs, i32([0]), i32([n])).cpu()[0, 0] == n
        self.k, self.v = self.k[:n], self.v[:n]

    def append(self, k, v):
        from paper_2505_11254_amd import binding
        n = len(self.k) + len(k)
        assert binding.pages8_resize(*self.cache(), self.refs, i32([0]), i32([n])).cpu()[0, 0] == n
        binding.pages8_append(k.cuda(), v.cuda(), *self.cache())
        self.k, self.v = torch.cat([self.k, k.double()]), torch.cat([self.v, v.double()])

    def compact(self, start, keep):
        from paper_2505_11254_amd import binding
        got = binding.pages8_compact(*self.cache(), self.refs, i32([0]), i32([start]), i32(keep), i32([0, len(keep)]))
        assert got.cpu()[0, 0] == len(keep)
        rows = list(range(start)) + [start + j for j in keep]
        self.k, self.v = self.k[rows], self.v[rows]

    def check(self):
        from paper_2505_11254_amd import binding
        n = len(self.k)
        got = binding.pages8_read(*self.cache(), n)
        table = self.table.cpu()[0, :pages_of(n)].long()
        for x, y, s in ((self.k, got[0], self.ks), (self.v, got[1], self.vs)):
            unit = s.cpu().double()[table].repeat_interleave(PAGE, 0)[:n, :, None]
            assert ((y.cpu().double() - x).abs() <= bound(x, unit)).all()


def rows(g, n, Hkv, d, exponent):
    spread = torch.pow(2.0, torch.randint(-16, 1, (n, Hkv, d), generator=g).double())
    return (torch.randn((n, Hkv, d), generator=g).double() * spread * 2.0 ** exponent).to(torch.bfloat16)


@pytest.mark.parametrize("Hkv,d", [(2, 64), (1, 128)])
@pytest.mark.parametrize("step", [1, 4, 9])
def test_scales_that_grow(Hkv, d, step):
    g, r = torch.Generator().manual_seed(step), random.Random(d)
    s = Slot(8, Hkv, d)
    for i in range(12):
        n = r.choice([1, 3, 16, 17, 40])
        s.append(rows(g, n, Hkv, d, i * step - 40), rows(g, n, Hkv, d, (i % 4) * step))
        s.check()
    while len(s.k) > 20:
        start = r.randint(0, len(s.k) - 1)
        rest = len(s.k) - start
        s.compact(start, sorted(r.sample(range(rest), max(1, rest - r.randint(1, 30)))))
        s.check()
        if r.random() < 0.3:
            s.append(rows(g, 5, Hkv, d, 0), rows(g, 5, Hkv, d, 0))
            s.check()
        elif len(s.k) > 40:
            s.resize(len(s.k) - 7)
            s.check()


@pytest.mark.parametrize("Hkv,d", [(2, 64), (1, 128)])
@pytest.mark.parametrize("leave", ["resize", "compact"])
def test_a_scale_stays_when_the_tokens_that_set_it_leave(Hkv, d, leave):
    """A dropped draft of large values leaves its page's scale; a page begun anew gets its own."""
    g = torch.Generator().manual_seed(d)
    s = Slot(3, Hkv, d)
    small, big = rows(g, 10, Hkv, d, 0), torch.full((1, Hkv, d), 448.0 * 2 ** 9, dtype=torch.bfloat16)
    s.append(small, small)
    page = int(s.table[0, 0])
    first = s.ks[page].clone()
    s.append(big, -big)
    assert (s.ks[page] == 512.0).all() and (s.vs[page] == 512.0).all() and (first < 1.0).all()
    if leave == "resize":
        s.resize(10)
    else:
        s.compact(4, [0, 1, 2, 3, 4, 5])
    s.check()
    more = rows(g, 53, Hkv, d, 0)
    s.append(more, more)
    assert (s.ks[page] == 512.0).all() and (s.vs[page] == 512.0).all()
    s.check()
    more = rows(g, 20, Hkv, d, 0)
    s.append(more, more)  # one ends the page, the others begin the next
    assert (s.ks[int(s.table[0, 1])] < 1.0).all()
    s.check()
    s.resize(0)
    s.append(small, small)
    assert torch.equal(s.ks[int(s.table[0, 0])], first)
    s.check()
