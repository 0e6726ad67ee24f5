"""Attention over the 8-bit cache, and over both caches under changed scores, against the definition in
64 bits of the values that the codes stand for.  Tolerances: scored.py; the log-sum-exp sums weights that
are each off by 2^-8 of themselves at most, and by their score's error."""
from __future__ import annotations

import random

import pytest
import torch

from paged_sim import PAGE, pages_of
from pages8_sim import NAN, VALUES, codes
from scored import HALF, attend, slopes_of, tolerance
from test_gpu_paged_attn import HEADS, Case

pytestmark = pytest.mark.gpu


class Case8(Case):
    """A cache of codes with scales far apart (eight), or of bf16; what lies behind the last token, and
    pages that no sequence has, are NaN."""

    def __init__(self, lens, news, Hq, Hkv, d, seed, eight=True, std=1.0, **kw):
        super().__init__(lens, news, Hq, Hkv, d, seed, **kw)
        self.q = (self.q.float() * std).to(torch.bfloat16)
        self.eight = eight
        if not eight:
            return
        g = torch.Generator().manual_seed(seed + 1)
        for name in ("k", "v"):
            x = getattr(self, name).float()
            held = torch.isfinite(x)
            # (scales as wide as a page's values allow: 448 times them holds the largest)
            e = torch.randint(-8, 3, x.shape[:2], generator=g)
            c = codes(torch.where(held, x, torch.zeros_like(x)).double() * torch.pow(2.0, -e.double())[..., None, None])
            c = torch.where(held, c, torch.full_like(c, NAN))
            sc = torch.pow(2.0, e.double())
            setattr(self, name, torch.where(held, VALUES[c.long()] * sc[..., None, None], float("nan")))
            setattr(self, name + "8", c.view(torch.float8_e4m3fn))
            setattr(self, name + "_scales", torch.where(held.any(-1).any(-1), sc, float("nan")).float())

    def gpu(self):
        if not self.eight:
            return super().gpu()
        return tuple(x.cuda() for x in (self.q, self.k8, self.v8, self.k_scales, self.v_scales, self.table, self.L))

    def verify(self, out, lse, visible, cap=0.0, slopes=None):
        out, G = out.float().cpu().double(), self.Hq // self.Hkv
        for b, n in enumerate(self.lens):
            for g in range(self.Hkv):
                k, v = self.keys(b, g)
                s, m = slice(self.cu[b], self.cu[b + 1]), self.news[b]
                if not m:
                    continue
                vis = torch.stack([visible(b, i, g) for i in range(m)])
                for h in range(g * G, (g + 1) * G):
                    bias = None
                    if slopes is not None:
                        dist = (torch.arange(n) - (n - m + torch.arange(m))[:, None]).abs().double()
                        bias = -float(slopes[h]) * dist
                    want, wlse, dev, dl = attend(self.q[s, h], k, v, vis, cap, bias)
                    got = out[s, h]
                    assert torch.isfinite(got).all()
                    err = (got - want).abs()
                    tol = tolerance(want, dev, dl, float(v.double().abs().max()) if n else 0.0)
                    assert (err <= tol).all(), (b, h, float((err - tol).max()))
                    if lse is not None:
                        gl = lse.cpu().double()[s, h]
                        empty = torch.isinf(wlse)
                        assert (torch.isinf(gl) == empty).all() and (gl[empty] < 0).all()
                        assert ((gl - wlse)[~empty].abs() <= HALF * (1 + 2 ** -7) + dl).all()


def call(c, **kw):
    from paper_2505_11254_amd import binding
    f = binding.tree_attn_paged8 if c.eight else binding.tree_attn_paged_scored
    return f(*c.gpu(), **c.kw(), **kw)


def upto(c):
    return lambda b, i, g: torch.arange(c.lens[b]) <= c.lens[b] - c.news[b] + i


SCORES = [(0.0, False), (12.0, False), (0.0, True), (12.0, True)]


@pytest.mark.parametrize("Hq,Hkv,d", HEADS)
@pytest.mark.parametrize("eight", [True, False])
@pytest.mark.parametrize("cap,biased", SCORES)
def test_single_tokens(Hq, Hkv, d, eight, cap, biased):
    """Lengths around the unit, page and split sizes, none and one token, in one ragged batch."""
    if not eight and not cap and not biased:
        return  # (the plain call's own tests)
    lens = [1, 0, 31, 32, 33, 63, 64, 65, 127, 257, 777, 2049]
    c = Case8(lens, [1 if n else 0 for n in lens], Hq, Hkv, d, seed=Hq, eight=eight, std=2.0)
    slopes = slopes_of(Hq) if biased else None
    lse = torch.full((c.cu[-1], Hq), 7.0, device="cuda")
    out = call(c, lse=lse, cap=cap, slopes=slopes.cuda() if biased else None)
    c.verify(out, lse, upto(c), cap, slopes)


@pytest.mark.parametrize("Hq,Hkv,d", [(8, 2, 64), (32, 8, 128), (64, 8, 128), (28, 4, 128)])
@pytest.mark.parametrize("n", [2, 9, 24, 70, 150])
@pytest.mark.parametrize("eight,cap", [(True, 0.0), (True, 9.0), (False, 9.0)])
def test_trees(Hq, Hkv, d, n, eight, cap):
    """Draft trees of each workgroup shape, rows that see nothing among them."""
    from paper_2505_11254_amd import binding
    r = random.Random(n * Hq)
    news = [n, max(1, n - 1), n // 2, 1]
    lens = [news[0] + 200, news[1], news[2] + 37, 1 + 64]
    c = Case8(lens, news, Hq, Hkv, d, seed=n, eight=eight)
    words = -(-n // 64) + 1
    seen, rows = [], []
    for b, m in enumerate(news):
        mask = binding.tree_mask([[r.randint(max(-1, i - 4), i - 1) for i in range(m)]])
        bits = [[bool(int(mask[i, j // 64]) >> (j % 64) & 1) for j in range(m)] for i in range(m)]
        for i in range(m):
            if r.random() < 0.1:
                bits[i] = [False] * m
            x = sum(1 << j for j, bit in enumerate(bits[i]) if bit) | (r.getrandbits(words * 64) >> m << m)
            w = [(x >> 64 * j) & (2 ** 64 - 1) for j in range(words)]
            rows.append([y - 2 ** 64 if y >> 63 else y for y in w])
        seen.append(bits)
    lse = torch.zeros((c.cu[-1], Hq), device="cuda")
    out = call(c, mask=torch.tensor(rows, dtype=torch.int64).cuda(), lse=lse, cap=cap)
    c.verify(out, lse, lambda b, i, g: torch.tensor([True] * (lens[b] - news[b]) + seen[b][i], dtype=torch.bool), cap)


@pytest.mark.parametrize("Hq,Hkv,d", [(4, 4, 128), (8, 1, 64), (16, 1, 128)])
@pytest.mark.parametrize("eight", [True, False])
@pytest.mark.parametrize("cap,biased", SCORES[1:])
def test_causal_chunks(Hq, Hkv, d, eight, cap, biased):
    c = Case8([300, 130, 64, 700], [300, 1, 20, 65], Hq, Hkv, d, seed=5, eight=eight)
    slopes = slopes_of(Hq) if biased else None
    out = call(c, cap=cap, slopes=slopes.cuda() if biased else None)
    c.verify(out, None, upto(c), cap, slopes)


@pytest.mark.parametrize("eight", [True, False])
@pytest.mark.parametrize("cap,slope", [(0.0, None), (8.0, None), (0.0, 1e-3), (0.0, 5.0)])
def test_long_contexts_in_many_splits(eight, cap, slope):
    if not eight and not cap and slope is None:
        return
    lens = [70000, 5]
    c = Case8(lens, [1, 1], 8, 2, 128, seed=3, eight=eight)
    slopes = None if slope is None else torch.full((8,), slope)
    lse = torch.zeros((2, 8), device="cuda")
    out = call(c, lse=lse, cap=cap, slopes=None if slope is None else slopes.cuda())
    c.verify(out, lse, upto(c), cap, slopes)


@pytest.mark.parametrize("B,Hkv", [(300, 2)])
def test_many_short_sequences(B, Hkv):
    r = random.Random(B)
    lens = [r.choice([0, 1, 63, 64, 200, 300]) for _ in range(B)]
    lens[7] = 40 * 64
    c = Case8(lens, [1 if n else 0 for n in lens], 4 * Hkv, Hkv, 64, seed=B)
    c.verify(call(c), None, upto(c))


def test_shares_of_more_pages_than_ids_are_held():
    """Sequences of 100,000 tokens that repeat the same few pages, biased so that the pages' order counts."""
    from paper_2505_11254_amd import binding
    g = torch.Generator().manual_seed(1)
    base = Case8([60 * PAGE], [1], 8, 8, 64, seed=4)
    n = 100_003
    order = torch.randint(0, 60, (40, pages_of(n)), generator=g)
    ids = base.table[base.slots[0], :60].long()
    table = ids[order].to(torch.int32)
    L = torch.full((40,), n, dtype=torch.int32)
    q = torch.randn((40, 8, 64), generator=g).to(torch.bfloat16)
    _, k8, v8, ks, vs, _, _ = base.gpu()
    for slopes in (None, torch.full((8,), 2e-5)):
        out = binding.tree_attn_paged8(q.cuda(), k8, v8, ks, vs, table.cuda(), L.cuda(), B=40,
                                       slopes=None if slopes is None else slopes.cuda()).cpu()
        for b in (0, 39):
            c = Case8([1], [1], 8, 8, 64, seed=0)
            c.q, c.lens = q[b:b + 1], [n]
            t = table[b].long()
            c.keys = lambda _, h: tuple(x[t, h].reshape(-1, 64)[:n] for x in (base.k, base.v))
            c.verify(out[b:b + 1], None, upto(c), 0.0, slopes)


def test_wrong_pages_are_skipped():
    c = Case8([300, 200, 90], [1, 2, 1], 8, 2, 128, seed=9)
    c.table[c.slots[0], 1] = 10 ** 6
    c.table[c.slots[0], 3] = -7
    dev, kw = c.gpu(), c.kw()
    kw["slots"][2] = 99
    from paper_2505_11254_amd import binding
    out = binding.tree_attn_paged8(*dev, **kw).float().cpu()
    assert (out[c.cu[2]:] == 0).all()
    c.table[c.slots[0], 1] = c.table[c.slots[0], 3] = c.table[c.slots[0], 0]
    c.lens, c.news, c.cu = c.lens[:2], c.news[:2], c.cu[:3]

    def visible(b, i, g):
        j = torch.arange(c.lens[b])
        return (j // 64 != 1) & (j // 64 != 3) if b == 0 else j <= c.lens[b] - c.news[b] + i
    c.verify(out, None, visible)


@pytest.mark.parametrize("Hq,Hkv,d,top_k", [(8, 2, 64, 5), (32, 8, 128, 16), (28, 4, 128, 3), (64, 1, 64, 40),
                                            (16, 16, 128, 9), (64, 1, 128, 7)])
def test_selected_pages(Hq, Hkv, d, top_k):
    """Lists of every size, empty ones, entries that are no candidate, and several tokens per sequence."""
    from paper_2505_11254_amd import binding
    r = random.Random(top_k)
    lens, news = [1, 64, 65, 700, 3001, 2048, 0], [1, 1, 2, 3, 1, 4, 0]
    c = Case8(lens, news, Hq, Hkv, d, seed=top_k)
    lists = torch.full((c.cu[-1], Hkv, top_k), -1, dtype=torch.int32)
    seen = {}
    for b, n in enumerate(lens):
        for i in range(news[b]):
            own = (n - news[b] + i) // PAGE
            for g in range(Hkv):
                mine = sorted(r.sample(range(own), r.randint(0, min(own, top_k))))
                seen[b, i, g] = mine + [own]
                row = mine + [own, own + 1, 10 ** 6][:max(0, min(3, top_k - len(mine)))]
                lists[c.cu[b] + i, g, :len(row)] = torch.tensor(row, dtype=torch.int32)
    lse = torch.zeros((c.cu[-1], Hq), device="cuda")
    out = binding.selected_attn_paged8(*c.gpu(), lists.cuda(), lse=lse, **c.kw())

    def visible(b, i, g):
        j = torch.arange(lens[b])
        return torch.isin(j // PAGE, torch.tensor(seen[b, i, g])) & (j <= lens[b] - news[b] + i)
    c.verify(out, lse, visible)


def test_select_then_attend():
    """Summaries of the codes, pages chosen by them, attention over those: a decoding step of the sparse kind."""
    from paper_2505_11254_amd import binding
    from paged_sim import choose, summary
    c = Case8([3000, 900], [1, 1], 8, 2, 128, seed=12)
    q, k8, v8, ks, vs, table, L = c.gpu()
    P = k8.shape[0]
    codes8, scales = torch.zeros((P, 2, 128), dtype=torch.int8, device="cuda"), torch.zeros((P, 2), device="cuda")
    binding.page8_summary(k8, ks, table, L, codes8, scales)
    pages = binding.select_pages(q, codes8, scales, table, L, top_k=6, n_sink=1, n_recent=2, slots=c.kw()["slots"], B=2)
    out = binding.selected_attn_paged8(q, k8, v8, ks, vs, table, L, pages, slots=c.kw()["slots"], B=2)
    seen = {}
    for b, n in enumerate(c.lens):
        for g in range(2):
            own = (n - 1) // PAGE
            keys = c.keys(b, g)[0][:own * PAGE].view(own, PAGE, 128)
            want = choose(c.q[b, 4 * g:4 * g + 4], *summary(keys), 6, 1, 2)
            assert pages[b, g].cpu().tolist() == want
            seen[b, g] = want + [own]
    c.verify(out, None, lambda b, i, g: torch.isin(torch.arange(c.lens[b]) // PAGE, torch.tensor(seen[b, g])))


def test_unchanged_scores_give_the_plain_calls_results():
    from paper_2505_11254_amd import binding
    c = Case([2000, 64, 7], [3, 1, 7], 32, 8, 128, seed=2)
    assert torch.equal(binding.tree_attn_paged_scored(*c.gpu(), **c.kw()), binding.tree_attn_paged(*c.gpu(), **c.kw()))


@pytest.mark.parametrize("eight", [True, False])
def test_streams_graphs_and_workspaces(eight):
    from paper_2505_11254_amd import binding
    a = Case8([5000, 33], [1, 3], 32, 8, 128, seed=1, eight=eight)
    b = Case8([900, 4000], [2, 1], 32, 8, 128, seed=2, eight=eight)
    f = binding.tree_attn_paged8 if eight else binding.tree_attn_paged_scored
    size = binding.paged8_workspace_bytes if eight else binding.paged_workspace_bytes
    ga, gb = a.gpu(), b.gpu()
    eager = [f(*g, cap=20.0, **c.kw()) for g, c in ((ga, a), (gb, b))]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    on_side = f(*ga, cap=20.0, stream=side, **a.kw())
    side.synchronize()
    assert torch.equal(on_side, eager[0])
    ws = torch.empty(max(size(2, 3, 32, 8, 128, ga[-2].shape[1] * 64), size(2, 2, 32, 8, 128, gb[-2].shape[1] * 64)),
                     dtype=torch.uint8, device="cuda")
    outs, graphs = [torch.empty_like(x) for x in eager], []
    for g, c, o in ((ga, a, outs[0]), (gb, b, outs[1])):
        kw = c.kw()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            f(*g, cap=20.0, out=o, workspace=ws, **kw)
        graphs.append((graph, kw))
    for _ in range(3):
        for (graph, _), o, want in zip(graphs, outs, eager):
            o.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(o, want)
        ws.fill_(255)


def test_repeats_are_bitwise_equal():
    c = Case8([9000, 100, 4000], [1, 1, 1], 32, 8, 128, seed=6)
    first = call(c)
    for _ in range(5):
        assert torch.equal(call(c), first)
