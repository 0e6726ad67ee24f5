"""The paged cache's rules, the attention over it and the block selection, written
out plainly on the host: what the GPU calls are checked against.

Integers follow the documented order of service one request at a time; attention is
in 64-bit floats from its definition.
"""
from __future__ import annotations

import numpy as np
import torch

PAGE = 64


def pages_of(n):
    return -(-n // PAGE)


class Cache:
    """A cache on the CPU (bf16 pages as torch tensors, integers as numpy arrays)."""

    def __init__(self, layers, P, Hkv, d, S, M, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.k = torch.randn((layers, P, Hkv, PAGE, d), generator=g).to(torch.bfloat16)
        self.v = torch.randn((layers, P, Hkv, PAGE, d), generator=g).to(torch.bfloat16)
        self.table = np.full((S, M), -1, dtype=np.int32)
        self.lens = np.zeros(S, dtype=np.int32)
        self.refs = np.zeros(P, dtype=np.int32)
        self.S, self.M, self.P = S, M, P

    def put(self, slot, n, pages):
        """A sequence of n tokens in the given pages (shared ones may be named again)."""
        self.table[slot, :pages_of(n)] = pages[:pages_of(n)]
        self.lens[slot] = n
        for p in pages[:pages_of(n)]:
            self.refs[p] += 1

    def gpu(self):
        t = lambda x: torch.from_numpy(x.copy()).cuda()  # noqa: E731
        k, v = self.k.cuda(), self.v.cuda()
        return k, v, t(self.table), t(self.lens), t(self.refs)

    def equal(self, k, v, table, lens, refs):
        np.testing.assert_array_equal(table.cpu().numpy(), self.table)
        np.testing.assert_array_equal(lens.cpu().numpy(), self.lens)
        np.testing.assert_array_equal(refs.cpu().numpy(), self.refs)
        assert torch.equal(k.cpu().view(torch.int16), self.k.view(torch.int16))
        assert torch.equal(v.cpu().view(torch.int16), self.v.view(torch.int16))

    def fork(self, src, dst):
        out = []
        for i, (s, d) in enumerate(zip(src, dst)):
            ok = 0 <= s < self.S and 0 <= d < self.S and s not in dst and d not in dst[:i]
            if not ok or self.lens[d] != 0 or self.table[d, 0] >= 0:
                out.append(-1)
                continue
            n = int(self.lens[s])
            self.table[d, :pages_of(n)] = self.table[s, :pages_of(n)]
            for p in self.table[s, :pages_of(n)]:
                self.refs[p] += 1
            self.lens[d] = n
            out.append(n)
        return out

    def _give_back(self, s, c0):
        for c in range(c0, self.M):
            if self.table[s, c] >= 0:
                self.refs[self.table[s, c]] -= 1
                self.table[s, c] = -1

    def resize(self, slots, new):
        out = [None] * len(slots)
        grow = []
        for i, (s, n) in enumerate(zip(slots, new)):
            if not 0 <= s < self.S or s in slots[:i] or not 0 <= n <= self.M * PAGE:
                out[i] = (-1, -1, -1, 0)
            elif n <= self.lens[s]:
                self._give_back(s, pages_of(n))
                self.lens[s] = n
                out[i] = (n, -1, -1, 0)
            else:
                grow.append(i)
        free = [p for p in range(self.P) if self.refs[p] == 0]
        full = False
        for i in grow:
            s, n, old = slots[i], new[i], int(self.lens[slots[i]])
            c = old // PAGE
            copy = old % PAGE > 0 and self.refs[self.table[s, c]] > 1
            ask = pages_of(n) - pages_of(old) + copy
            if full or ask > len(free):
                full = True
                out[i] = (-1, -1, -1, 0)
                continue
            out[i] = (n, -1, -1, 0)
            if copy:
                p, q = int(self.table[s, c]), free.pop(0)
                self.refs[p] -= 1
                self.refs[q] = 1
                self.table[s, c] = q
                for x in (self.k, self.v):
                    x[:, q, :, :old % PAGE] = x[:, p, :, :old % PAGE]
                out[i] = (n, p, q, old % PAGE)
            for c in range(pages_of(old), pages_of(n)):
                q = free.pop(0)
                self.table[s, c] = q
                self.refs[q] = 1
            self.lens[s] = n
        return out

    def append(self, slots, cu, k, v):
        for b, s in enumerate(slots):
            m = cu[b + 1] - cu[b]
            for i in range(m):
                pos = int(self.lens[s]) - m + i
                p = self.table[s, pos // PAGE]
                self.k[:, p, :, pos % PAGE] = k[:, cu[b] + i]
                self.v[:, p, :, pos % PAGE] = v[:, cu[b] + i]

    def compact(self, slots, start, keep):
        out = []
        for i, (s, st, kp) in enumerate(zip(slots, start, keep)):
            n = int(self.lens[s]) if 0 <= s < self.S else 0
            ok = 0 <= s < self.S and s not in slots[:i] and 0 <= st <= n
            ok = ok and all(0 <= x < n - st for x in kp) and all(a < b for a, b in zip(kp, kp[1:]))
            moved = [j for j, x in enumerate(kp) if x != j]
            if ok and moved:
                for c in range((st + moved[0]) // PAGE, (st + len(kp) - 1) // PAGE + 1):
                    ok = ok and self.refs[self.table[s, c]] == 1
            if not ok:
                out.append(-1)
                continue
            for j, x in enumerate(kp):
                a, b = st + x, st + j
                for y in (self.k, self.v):
                    y[:, self.table[s, b // PAGE], :, b % PAGE] = y[:, self.table[s, a // PAGE], :, a % PAGE].clone()
            self.lens[s] = st + len(kp)
            self._give_back(s, pages_of(st + len(kp)))
            out.append(len(kp))
        return out


def attend(q, k, v, vis):
    """softmax over visible keys in 64 bits: q [rows, d], k, v [keys, d], vis [rows, keys] ->
    (out, log-sum-exp); rows that see nothing: 0 and -inf."""
    q, k, v = (x.double() for x in (q, k, v))
    a = (q @ k.T) / q.shape[1] ** 0.5
    a = torch.where(vis, a, torch.full_like(a, float("-inf")))
    top = torch.where(vis.any(1), a.max(1).values if a.shape[1] else torch.zeros(len(q), dtype=a.dtype),
                      torch.zeros(len(q), dtype=a.dtype))
    p = torch.exp(a - top[:, None])
    z = p.sum(1)
    out = torch.where(z[:, None] > 0, (p @ v) / torch.where(z > 0, z, torch.ones_like(z))[:, None],
                      torch.zeros_like(q))
    return out, torch.where(z > 0, top + torch.log(z), torch.full_like(z, float("-inf")))


def summary(keys):
    """Codes (int64) and scales (fp32) of the mean keys of blocks [n, 64, d]."""
    s = keys.double().sum(1)
    big = s.abs().max(1).values
    unit = torch.where(big > 0, big, torch.ones_like(big))
    code = torch.where(big[:, None] > 0, torch.round(s * 127 / unit[:, None]), torch.zeros_like(s))
    return code.long(), (big / (127 * PAGE)).float()


def choose(rows, codes, scales, top_k, n_sink, n_recent):
    """The blocks that query rows [rows, d] choose among the given ones."""
    n = len(scales)
    if n <= top_k:
        return list(range(n))
    a = rows.double().abs().max()
    q8 = torch.round(rows.double() * 127 / a) if a > 0 else rows.double() * 0
    best = (q8 @ codes.double().T).max(0).values
    score = (best * scales.double()).float().tolist()  # one rounding of an exact product
    forced = set(range(min(n_sink, n))) | set(range(max(0, n - n_recent), n))
    return sorted(sorted(range(n), key=lambda x: (x not in forced, -score[x], x))[:top_k])
