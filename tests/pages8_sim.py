"""The 8-bit cache's rules on the host, written out plainly: what the GPU calls are checked against."""
from __future__ import annotations

import math

import torch

from paged_sim import PAGE, Cache, pages_of

LEAST, MOST = -110, 119


def values_of_codes():
    """The 256 values of e4m3 from their bits."""
    out = []
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        x = math.nan if (e, m) == (15, 7) else (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
        out.append(-x if c >> 7 else x)
    return torch.tensor(out, dtype=torch.float64)


VALUES = values_of_codes()
NAN = 0x7F


def codes(y):
    """The codes nearest to y (64 bits, up to 448), ties to the even code; not finite: NaN."""
    grid = VALUES[:127]
    y = y.double()
    a = torch.where(torch.isfinite(y), y.abs(), torch.zeros_like(y)).clamp(max=448.0)
    hi = torch.searchsorted(grid, a).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    dl, dh = a - grid[lo], grid[hi] - a
    pick = torch.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    neg = torch.signbit(y)
    pick = torch.where(neg, pick + 128, pick)
    return torch.where(torch.isfinite(y), pick, torch.full_like(pick, NAN)).to(torch.uint8)


def needed(x):
    """The least exponent whose scale brings the finite values x within 448."""
    x = x.double()
    top = float(torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).max()) if x.numel() else 0.0
    e = LEAST
    while e < MOST and top > 448 * 2.0 ** e:
        e += 1
    return e


class Cache8(Cache):
    """paged_sim.Cache with codes (uint8) and exponents in place of bf16 pages."""

    def __init__(self, layers, P, Hkv, d, S, M, seed=0):
        super().__init__(layers, P, Hkv, d, S, M, seed)
        g = torch.Generator().manual_seed(seed)
        self.k, self.v = (torch.randint(0, 256, (layers, P, Hkv, PAGE, d), generator=g).to(torch.uint8) for _ in range(2))
        self.ke, self.ve = (torch.randint(-3, 4, (layers, P, Hkv), generator=g) for _ in range(2))

    def gpu8(self):
        """(k_pages, v_pages, k_scales, v_scales, table, lens, refs), one layer without its axis."""
        def t(x):
            return torch.from_numpy(x.copy()).cuda()
        one = self.k.shape[0] == 1
        kv = [(x[0] if one else x).cuda().view(torch.float8_e4m3fn) for x in (self.k, self.v)]
        sc = [torch.pow(2.0, (x[0] if one else x).double()).float().cuda() for x in (self.ke, self.ve)]
        return (*kv, *sc, t(self.table), t(self.lens), t(self.refs))

    def equal8(self, k, v, ks, vs, table, lens, refs):
        assert (table.cpu().numpy() == self.table).all()
        assert (lens.cpu().numpy() == self.lens).all()
        assert (refs.cpu().numpy() == self.refs).all()
        for mine, got, e, s in ((self.k, k, self.ke, ks), (self.v, v, self.ve, vs)):
            got = got.view(torch.uint8).cpu().view(mine.shape)
            assert torch.equal(torch.pow(2.0, e.double()).float().view(-1), s.cpu().view(-1))
            nan = (got & 0x7F) == NAN
            assert torch.equal(nan, (mine & 0x7F) == NAN)
            assert torch.equal(torch.where(nan, 0, got), torch.where(nan, 0, mine))

    def values(self, which, layer, page, h, rows):
        x, e = (self.k, self.ke) if which == "k" else (self.v, self.ve)
        return VALUES[x[layer, page, h, rows].long()] * 2.0 ** float(e[layer, page, h])

    def rows(self, which, layer, slot, h, n0, n1):
        """Values [n1 - n0, d] of tokens n0 .. n1 of a slot."""
        return torch.stack([self.values(which, layer, int(self.table[slot, j // PAGE]), h, j % PAGE) for j in range(n0, n1)]
                           or [torch.zeros(0, dtype=torch.float64)])

    def append8(self, slots, cu, k, v):
        for b, s in enumerate(slots):
            m, n = cu[b + 1] - cu[b], int(self.lens[s])
            for c in range((n - m) // PAGE, pages_of(n)):
                a0, a1 = max(n - m, c * PAGE), min(n, (c + 1) * PAGE)
                p, r0 = int(self.table[s, c]), a0 - c * PAGE
                for x, e, new in ((self.k, self.ke, k), (self.v, self.ve, v)):
                    for layer in range(x.shape[0]):
                        for h in range(x.shape[2]):
                            w = new[layer, cu[b] + a0 - (n - m):cu[b] + a1 - (n - m), h].double()
                            was = int(e[layer, p, h]) if r0 else LEAST
                            now = max(was, needed(w))
                            if r0 and now > was:
                                x[layer, p, h, :r0] = codes(VALUES[x[layer, p, h, :r0].long()] * 2.0 ** (was - now))
                            x[layer, p, h, r0:r0 + a1 - a0] = codes(w * 2.0 ** -now)
                            e[layer, p, h] = now

    def resize(self, slots, new):
        was = self.table.copy()
        out = super().resize(slots, new)
        for n, p, q, rows in out:
            if q >= 0:
                self.ke[:, q], self.ve[:, q] = self.ke[:, p], self.ve[:, p]
        del was
        return out

    def compact8(self, slots, start, keep):
        old = [x.clone() for x in (self.k, self.v, self.ke, self.ve)]
        table, lens = self.table.copy(), self.lens.copy()
        out = self.compact(slots, start, keep)  # (rows move as bytes; their scales follow here)
        for got, s, st, kp in zip(out, slots, start, keep):
            moved = [j for j, x in enumerate(kp) if x != j]
            if got < 0 or not moved:
                continue
            for c in range((st + moved[0]) // PAGE, (st + len(kp) - 1) // PAGE + 1):
                p = int(table[s, c])
                js = [j for j in range(moved[0], len(kp)) if (st + j) // PAGE == c]
                r0 = (st + js[0]) % PAGE
                for x, e, ox, oe in ((self.k, self.ke, old[0], old[2]), (self.v, self.ve, old[1], old[3])):
                    for layer in range(x.shape[0]):
                        for h in range(x.shape[2]):
                            src = [(int(table[s, (st + kp[j]) // PAGE]), (st + kp[j]) % PAGE) for j in js]
                            now = max([int(oe[layer, q, h]) for q, _ in src] + ([int(oe[layer, p, h])] if r0 else []))
                            rows = [(r, p, r) for r in range(r0)] + [((st + j) % PAGE, q, r) for j, (q, r) in zip(js, src)]
                            for to, q, r in rows:
                                w = int(oe[layer, q, h])
                                y = ox[layer, q, h, r]
                                x[layer, p, h, to] = y if w == now else codes(VALUES[y.long()] * 2.0 ** (w - now))
                            e[layer, p, h] = now
        del lens
        return out
