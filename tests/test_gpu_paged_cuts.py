"""Attention over the paged cache where workgroups share a sequence's pages, so that partial results
are merged: draft trees of several row groups, and lists of pages.  Every case asserts that it needs the
partial results' workspace.  Tolerances as in test_gpu_paged_attn."""
from __future__ import annotations

import random

import pytest
import torch

from paged_sim import PAGE
from test_gpu_paged_attn import Case

pytestmark = pytest.mark.gpu


def _masks(news, r, words):
    """Trees with rows that see nothing, rows that see others but not themselves, and bits behind the last
    draft: (bits per sequence, int64 [T, words])."""
    seen, rows = [], []
    for m in news:
        mine = []
        for i in range(m):
            kind = r.random()
            if kind < 0.1:
                x = 0
            elif kind < 0.3:
                x = r.getrandbits(m)
            elif kind < 0.5:
                x = 1 << r.randrange(m)  # (a single draft, often pages away)
            else:
                p = r.randint(max(-1, i - 5), i - 1)
                x = (mine[p] if p >= 0 else 0) | 1 << i
            mine.append(x)
        seen.append(mine)
        for x in mine:
            x |= r.getrandbits(words * 64) >> m << m
            w = [(x >> 64 * j) & (2 ** 64 - 1) for j in range(words)]
            rows.append([y - 2 ** 64 if y >> 63 else y for y in w])
    return seen, torch.tensor(rows, dtype=torch.int64)


@pytest.mark.parametrize("lens,news,Hq,Hkv,d,bound", [
    ([5000, 4000, 3500], [24, 20, 24], 28, 4, 128, 5000),       # one group of four row tiles
    ([9000, 5000], [64, 62], 16, 2, 128, 9000),                 # two groups of eight, side by side
    ([9000, 700, 64, 4000], [64, 0, 63, 61], 16, 2, 128, 9000),
    ([9000, 5000], [64, 20], 16, 2, 128, 9000),                 # (one sequence has one group only)
    ([6000, 6000 - 64], [90, 90], 20, 4, 64, 6000),             # four groups of four
    ([4000, 150], [150, 150], 8, 1, 64, 7000),
    ([700, 690, 64], [700, 690, 64], 4, 1, 128, 9000),          # no context: parts that some rows see nothing of
    ([700, 320, 700], [700, 310, 640], 2, 1, 64, 9000),
])
def test_trees_over_shared_pages(lens, news, Hq, Hkv, d, bound):
    from paper_2505_11254_amd import binding
    r = random.Random(sum(lens))
    c = Case(lens, news, Hq, Hkv, d, seed=sum(news))
    words = -(-max(news) // 64) + 1
    seen, mask = _masks(news, r, words)
    q, k, v, table, L = c.gpu()
    more = torch.full((table.shape[0], bound // PAGE + 1), -1, dtype=torch.int32, device="cuda")
    table = torch.cat([table, more], 1).contiguous()  # (a table with room for `bound` tokens)
    lse = torch.zeros(q.shape[:2], device="cuda")
    assert binding.paged_workspace_bytes(len(lens), max(news), Hq, Hkv, d, bound) > 0
    kw = dict(mask=mask.cuda(), max_len=bound, **c.kw())
    out = binding.tree_attn_paged(q, k, v, table, L, lse=lse, **kw)

    def visible(b, i, g):
        x = seen[b][i]
        return torch.tensor([True] * (lens[b] - news[b]) + [bool(x >> j & 1) for j in range(news[b])])
    c.check(out, lse, visible)
    assert torch.equal(out, binding.tree_attn_paged(q, k, v, table, L, **kw))


@pytest.mark.parametrize("lens,news,Hq,Hkv,d,top_k", [
    ([9000], [1], 32, 8, 128, 64),                                        # one sequence, cut in many places
    ([9000, 7000, 100, 0, 5000], [1, 2, 3, 0, 1], 32, 8, 128, 96),        # ragged, short and empty lists
    ([8000] * 16, [1] * 16, 32, 8, 128, 100),
    ([9000, 3000], [2, 1], 28, 4, 128, 128),
    ([6000, 4000], [2, 2], 65, 1, 128, 60),                               # four row tiles
    ([6000, 4000, 1], [2, 1, 1], 128, 1, 64, 50),
    ([6000, 2000], [1, 2], 200, 1, 128, 80),                              # two row groups of them
    ([6000, 3000], [2, 2], 264, 2, 64, 90),
    ([6000, 4000], [1, 1], 130, 2, 128, 70),
])
def test_lists_over_shared_pages(lens, news, Hq, Hkv, d, top_k):
    from paper_2505_11254_amd import binding
    r = random.Random(top_k)
    c = Case(lens, news, Hq, Hkv, d, seed=top_k)
    lists = torch.full((c.cu[-1], Hkv, top_k), -1, dtype=torch.int32)
    seen = {}
    for b, n in enumerate(lens):
        for i in range(news[b]):
            own = (n - news[b] + i) // PAGE
            for g in range(Hkv):
                most = min(own, top_k)
                mine = sorted(r.sample(range(own), r.choice([0, most // 2, most, most, most])))
                seen[b, i, g] = torch.tensor(mine + [own])
                row = mine + [-1] * (top_k - len(mine))
                if g % 2:
                    r.shuffle(row)  # (any order, and places that hold no page between)
                lists[c.cu[b] + i, g] = torch.tensor(row, dtype=torch.int32)
    q, k, v, table, L = c.gpu()
    lse = torch.zeros(q.shape[:2], device="cuda")
    assert binding.paged_workspace_bytes(len(lens), max(news), Hq, Hkv, d, 1, top_k) > 0
    out = binding.selected_attn_paged(q, k, v, table, L, lists.cuda(), lse=lse, **c.kw())

    def visible(b, i, g):
        j = torch.arange(lens[b])
        return torch.isin(j // PAGE, seen[b, i, g]) & (j <= lens[b] - news[b] + i)
    c.check(out, lse, visible)
    assert torch.equal(out, binding.selected_attn_paged(q, k, v, table, L, lists.cuda(), **c.kw()))
