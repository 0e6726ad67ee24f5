"""Precision of the attention over the paged cache where up to 32 query rows share a kv head
(single tokens, small drafts, lists), against the definition in 64 bits.

There the weights enter the second product as two bf16 parts, the nearest value and what it
leaves: half a step of half a step, 2^-16 of a weight, is lost.  The normaliser and the
log-sum-exp sum the fp32 weights.  So an output is off by its own rounding, half a step or 2^-8
of it; by (2^-16 + 2e-4) sqrt(sum_j p_j v_j^2 - out^2), where 2e-4 is twice the largest error of
a logit (test_gpu_paged_attn has its arithmetic); and by 1e-6 of the largest value, the sums'
own rounding.  The log-sum-exp is off by the logits' 2e-4."""
from __future__ import annotations

import random

import pytest
import torch

from paged_sim import PAGE, attend
from test_gpu_paged_attn import Case

pytestmark = pytest.mark.gpu


def check(c, out, lse, visible):
    out, G = out.float().cpu().double(), c.Hq // c.Hkv
    for b in range(len(c.lens)):
        for g in range(c.Hkv):
            k, v = c.keys(b, g)
            rows = c.q[c.cu[b]:c.cu[b + 1], g * G:(g + 1) * G].reshape(-1, c.d)
            if not len(rows):
                continue
            vis = torch.stack([visible(b, i, g) for i in range(c.news[b])]).repeat_interleave(G, 0)
            want, wlse = attend(rows, k, v, vis)
            sq, _ = attend(rows, k, v.double() ** 2, vis)
            dev = (sq - want ** 2).clamp(min=0).sqrt()
            tol = 2 ** -8 * want.abs() + (2 ** -16 + 2e-4) * dev + 1e-6 * v.double().abs().max()
            err = (out[c.cu[b]:c.cu[b + 1], g * G:(g + 1) * G].reshape(-1, c.d) - want).abs()
            assert (err <= tol).all(), (b, g, float((err / tol).max()))
            gl = lse.cpu().double()[c.cu[b]:c.cu[b + 1], g * G:(g + 1) * G].reshape(-1)
            seen = vis.any(1)
            assert (gl[~seen] == float("-inf")).all() and ((gl - wlse)[seen].abs() <= 2e-4).all()


@pytest.mark.parametrize("Hq,Hkv,d", [(32, 8, 128), (28, 4, 128), (7, 7, 128), (8, 2, 64), (32, 1, 64)])
@pytest.mark.parametrize("bound", [None, 40000])
def test_single_tokens(Hq, Hkv, d, bound):
    """Whole sequences and (with a bound that plans for long ones) cut ones."""
    from paper_2505_11254_amd import binding
    lens = [3, 0, 17, 64, 200, 1000, 5000]
    c = Case(lens, [1 if n else 0 for n in lens], Hq, Hkv, d, seed=d + Hq)
    q, k, v, table, L = c.gpu()
    if bound:
        table = torch.cat([table, torch.full((table.shape[0], bound // PAGE), -1, dtype=torch.int32, device="cuda")], 1)
        assert binding.paged_workspace_bytes(len(lens), 1, Hq, Hkv, d, bound) > 0
    lse = torch.zeros(q.shape[:2], device="cuda")
    out = binding.tree_attn_paged(q, k, v, table.contiguous(), L, lse=lse, max_len=bound, **c.kw())
    check(c, out, lse, lambda b, i, g: torch.ones(lens[b], dtype=torch.bool))


@pytest.mark.parametrize("Hq,Hkv,d,n", [(32, 8, 128, 8), (8, 2, 64, 7), (4, 4, 128, 32)])
def test_small_trees(Hq, Hkv, d, n):
    from paper_2505_11254_amd import binding
    r = random.Random(n)
    news = [n, n - 2, 1]
    lens = [n + 300, n - 2, 64]
    parents = [[r.randint(max(-1, i - 3), i - 1) for i in range(m)] for m in news]
    mask = binding.tree_mask(parents)
    mask[2] = 0  # (a row that sees the context alone, or nothing)
    mask[n + 1] = 0
    c = Case(lens, news, Hq, Hkv, d, seed=n)
    q, k, v, table, L = c.gpu()
    lse = torch.zeros(q.shape[:2], device="cuda")
    out = binding.tree_attn_paged(q, k, v, table, L, mask=mask.cuda(), lse=lse, **c.kw())

    def visible(b, i, g):
        w = int(mask[c.cu[b] + i, 0])
        return torch.tensor([True] * (lens[b] - news[b]) + [bool(w >> j & 1) for j in range(news[b])])
    check(c, out, lse, visible)


@pytest.mark.parametrize("Hq,Hkv,d,top_k", [(32, 8, 128, 12), (32, 8, 128, 96), (8, 1, 64, 40)])
def test_lists(Hq, Hkv, d, top_k):
    from paper_2505_11254_amd import binding
    r = random.Random(top_k)
    lens, news = [2, 900, 8000], [1, 2, 1]
    c = Case(lens, news, Hq, Hkv, d, seed=top_k)
    lists = torch.full((c.cu[-1], Hkv, top_k), -1, dtype=torch.int32)
    for b, n in enumerate(lens):
        for i in range(news[b]):
            own = (n - news[b] + i) // PAGE
            for g in range(Hkv):
                mine = sorted(r.sample(range(own), min(own, top_k)))
                lists[c.cu[b] + i, g, :len(mine)] = torch.tensor(mine, dtype=torch.int32)
    q, k, v, table, L = c.gpu()
    lse = torch.zeros(q.shape[:2], device="cuda")
    out = binding.selected_attn_paged(q, k, v, table, L, lists.cuda(), lse=lse, **c.kw())

    def visible(b, i, g):
        j, own = torch.arange(lens[b]), (lens[b] - news[b] + i) // PAGE
        return (torch.isin(j // PAGE, lists[c.cu[b] + i, g]) | (j // PAGE == own)) & (j <= lens[b] - news[b] + i)
    check(c, out, lse, visible)
