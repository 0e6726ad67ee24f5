"""Attention over the paged cache on the GPU: trees of drafts, single tokens, causal
chunks and selected pages, against the definition in 64 bits.

Tolerance of one output: it is rounded once to bf16 (half a step, 2^-8 of it).  Weights
are rounded to bf16 too, each by at most 2^-8 of itself, and the normaliser sums the
rounded ones: with p the exact weights, out moves by at most 2^-8 (1 + 2^-7) sum_j
p_j |v_j - out|, and that sum is at most sqrt(sum_j p_j v_j^2 - out^2).  fp32
arithmetic: a logit is a sum of d <= 128 products, off by at most d 2^-24 sum |q_c k_c|
/ sqrt d < 1e-4 for the unit normal inputs here (10 in all |q| |k| / sqrt d cases below
a factor of two), which moves out by as much times the same sum; 1e-6 of the largest
value covers the sums' own rounding.  The log-sum-exp sums weights that are each off by 2^-8 of
themselves at most."""
from __future__ import annotations

import random

import pytest
import torch

from paged_sim import PAGE, attend, pages_of

pytestmark = pytest.mark.gpu


class Case:
    """A cache whose rows behind each sequence's last token are NaN, and a batch of new tokens."""

    def __init__(self, lens, news, Hq, Hkv, d, seed, spare=3, scale=1.0):
        g = torch.Generator().manual_seed(seed)
        r = random.Random(seed)
        self.lens, self.news, self.Hq, self.Hkv, self.d = lens, news, Hq, Hkv, d
        S, M = len(lens) + 2, max(1, max(map(pages_of, lens))) + 1
        P = sum(map(pages_of, lens)) + spare
        self.k = torch.randn((P, Hkv, PAGE, d), generator=g).to(torch.bfloat16)
        self.v = (torch.randn((P, Hkv, PAGE, d), generator=g) * scale).to(torch.bfloat16)
        ids = r.sample(range(P), P)
        self.slots = r.sample(range(S), len(lens))
        self.table = torch.full((S, M), -1, dtype=torch.int32)
        self.L = torch.zeros(S, dtype=torch.int32)
        for s, n in zip(self.slots, lens):
            mine, ids = ids[:pages_of(n)], ids[pages_of(n):]
            self.table[s, :len(mine)] = torch.tensor(mine, dtype=torch.int32)
            self.L[s] = n
            if n % PAGE:
                self.k[mine[-1], :, n % PAGE:] = float("nan")
                self.v[mine[-1], :, n % PAGE:] = float("nan")
        for p in ids:
            self.k[p] = float("inf")
            self.v[p] = float("nan")
        self.cu = [0]
        for m in news:
            self.cu.append(self.cu[-1] + m)
        self.q = torch.randn((self.cu[-1], Hq, d), generator=g).to(torch.bfloat16)

    def gpu(self):
        return (self.q.cuda(), self.k.cuda(), self.v.cuda(), self.table.cuda(), self.L.cuda())

    def kw(self):
        return dict(slots=torch.tensor(self.slots, dtype=torch.int32).cuda(),
                    cu_seqlens=torch.tensor(self.cu, dtype=torch.int32).cuda(), max_seqlen=max(1, max(self.news)))

    def keys(self, b, g):
        n = self.lens[b]
        t = self.table[self.slots[b], :pages_of(n)].long()
        return tuple(x[t, g].reshape(-1, self.d)[:n] for x in (self.k, self.v))

    def check(self, out, lse, visible):
        """visible(b, i, g) -> bool [L]: the keys that row i of sequence b sees in kv head g."""
        out, G = out.float().cpu().double(), self.Hq // self.Hkv
        worst = 0.0
        for b in range(len(self.lens)):
            for g in range(self.Hkv):
                k, v = self.keys(b, g)
                rows = self.q[self.cu[b]:self.cu[b + 1], g * G:(g + 1) * G].reshape(-1, self.d)
                if not len(rows):
                    continue
                vis = torch.stack([visible(b, i, g) for i in range(self.news[b])]).repeat_interleave(G, 0)
                want, wlse = attend(rows, k, v, vis)
                sq, _ = attend(rows, k, v.double() ** 2, vis)
                dev = (sq - want ** 2).clamp(min=0).sqrt()
                top = v.double().abs().max() if v.numel() else 0.0
                tol = 2 ** -8 * want.abs() + (2 ** -8 * (1 + 2 ** -7) + 2e-4) * dev + 1e-6 * top
                got = out[self.cu[b]:self.cu[b + 1], g * G:(g + 1) * G].reshape(-1, self.d)
                assert torch.isfinite(got).all()
                err = (got - want).abs()
                assert (err <= tol).all(), (b, g, float((err - tol).max()))
                worst = max(worst, float(err.max()))
                if lse is not None:
                    gl = lse.cpu().double()[self.cu[b]:self.cu[b + 1], g * G:(g + 1) * G].reshape(-1)
                    empty = torch.isinf(wlse)
                    assert (torch.isinf(gl) == empty).all() and (gl[empty] < 0).all()
                    assert ((gl - wlse)[~empty].abs() <= 2 ** -8 * (1 + 2 ** -7) + 2e-4).all()
        return worst


HEADS = [(4, 1, 64), (32, 8, 128), (7, 7, 128), (28, 4, 128), (64, 1, 64), (64, 8, 128), (6, 2, 64)]


@pytest.mark.parametrize("Hq,Hkv,d", HEADS)
def test_single_tokens(Hq, Hkv, d):
    """Lengths around the unit, page and split sizes, none and one token, in one ragged batch."""
    from paper_2505_11254_amd import binding
    lens = [1, 0, 31, 32, 33, 64, 65, 127, 257, 777, 2049]
    c = Case(lens, [1 if n else 0 for n in lens], Hq, Hkv, d, seed=Hq)
    q, k, v, table, L = c.gpu()
    lse = torch.full((q.shape[0], Hq), 7.0, device="cuda")
    out = binding.tree_attn_paged(q, k, v, table, L, lse=lse, **c.kw())
    c.check(out, lse, lambda b, i, g: torch.ones(lens[b], dtype=torch.bool))


@pytest.mark.parametrize("Hq,Hkv,d", [(8, 2, 64), (32, 8, 128), (64, 8, 128), (28, 4, 128)])
@pytest.mark.parametrize("n", [2, 9, 24, 70, 150])
def test_trees(Hq, Hkv, d, n):
    """Draft trees of each workgroup shape, with rows that see nothing of a sequence without context,
    rows that see others but not themselves, and bits behind the last draft."""
    from paper_2505_11254_amd import binding
    r = random.Random(n * Hq)
    news = [n, max(1, n - 1), n // 2, 1, n]
    lens = [news[0] + 200, news[1], news[2] + 37, 1 + 64, news[4] + 900]
    c = Case(lens, news, Hq, Hkv, d, seed=n)
    words = -(-n // 64) + 1
    seen = []
    for b, m in enumerate(news):
        parents = [r.randint(max(-1, i - 4), i - 1) for i in range(m)]
        mask = binding.tree_mask([parents])
        bits = [[bool(int(mask[i, j // 64]) >> (j % 64) & 1) for j in range(m)] for i in range(m)]
        for i in range(m):
            if r.random() < 0.2:
                bits[i] = [r.random() < 0.5 for _ in range(m)]
            if r.random() < 0.1:
                bits[i] = [False] * m
        seen.append(bits)
    rows = []
    for b, m in enumerate(news):
        for i in range(m):
            x = sum(1 << j for j, bit in enumerate(seen[b][i]) if bit) | (r.getrandbits(words * 64) >> m << m)
            w = [(x >> 64 * j) & (2 ** 64 - 1) for j in range(words)]
            rows.append([y - 2 ** 64 if y >> 63 else y for y in w])
    mask = torch.tensor(rows, dtype=torch.int64).cuda()
    q, k, v, table, L = c.gpu()
    lse = torch.zeros((q.shape[0], Hq), device="cuda")
    out = binding.tree_attn_paged(q, k, v, table, L, mask=mask, lse=lse, **c.kw())

    def visible(b, i, g):
        return torch.tensor([True] * (lens[b] - news[b]) + seen[b][i], dtype=torch.bool)
    c.check(out, lse, visible)


@pytest.mark.parametrize("Hq,Hkv,d", [(4, 4, 128), (8, 1, 64)])
def test_causal_chunks(Hq, Hkv, d):
    from paper_2505_11254_amd import binding
    lens, news = [300, 130, 64, 700], [300, 1, 20, 65]
    c = Case(lens, news, Hq, Hkv, d, seed=5)
    q, k, v, table, L = c.gpu()
    out = binding.tree_attn_paged(q, k, v, table, L, **c.kw())
    c.check(out, None, lambda b, i, g: torch.arange(lens[b]) <= lens[b] - news[b] + i)


@pytest.mark.parametrize("n_split_len", [20000, 70000])
def test_long_context_in_many_splits(n_split_len):
    from paper_2505_11254_amd import binding
    lens = [n_split_len, 5]
    c = Case(lens, [1, 1], 8, 2, 128, seed=3, scale=3.0)
    q, k, v, table, L = c.gpu()
    lse = torch.zeros((2, 8), device="cuda")
    out = binding.tree_attn_paged(q, k, v, table, L, lse=lse, **c.kw())
    c.check(out, lse, lambda b, i, g: torch.ones(lens[b], dtype=torch.bool))
    # the same with a bound on the lengths, which only cuts the launch
    again = binding.tree_attn_paged(q, k, v, table, L, max_len=n_split_len, **c.kw())
    c.check(again, None, lambda b, i, g: torch.ones(lens[b], dtype=torch.bool))


@pytest.mark.parametrize("B,Hkv", [(300, 2), (700, 1)])
def test_many_short_sequences(B, Hkv):
    """More sequences than a wavefront or a workgroup holds, empty ones among them."""
    from paper_2505_11254_amd import binding
    r = random.Random(B)
    lens = [r.choice([0, 1, 63, 64, 200, 300]) for _ in range(B)]
    lens[7] = 40 * 64
    c = Case(lens, [1 if n else 0 for n in lens], 4 * Hkv, Hkv, 64, seed=B)
    q, k, v, table, L = c.gpu()
    out = binding.tree_attn_paged(q, k, v, table, L, **c.kw())
    c.check(out, None, lambda b, i, g: torch.ones(lens[b], dtype=torch.bool))
    # with a longer bound the work is shared differently
    long = torch.cat([table, torch.full_like(table, -1)[:, :1].expand(-1, 3000)], 1).contiguous()
    again = binding.tree_attn_paged(q, k, v, long, L, **c.kw())
    c.check(again, None, lambda b, i, g: torch.ones(lens[b], dtype=torch.bool))


def test_shares_of_more_pages_than_ids_are_held():
    """Forty sequences of 100,000 tokens that repeat the same few pages: every workgroup has almost
    2000 pages."""
    from paper_2505_11254_amd import binding
    g = torch.Generator().manual_seed(1)
    P, n, Hkv, d = 60, 100_003, 8, 64
    k, v = (torch.randn((P, Hkv, PAGE, d), generator=g).to(torch.bfloat16) for _ in range(2))
    table = torch.randint(0, P, (40, pages_of(n)), generator=g).to(torch.int32)
    L = torch.full((40,), n, dtype=torch.int32)
    q = torch.randn((40, 8, d), generator=g).to(torch.bfloat16)
    out = binding.tree_attn_paged(q.cuda(), k.cuda(), v.cuda(), table.cuda(), L.cuda(), B=40).cpu()
    for b in (0, 17, 39):
        c = Case([1], [1], 8, Hkv, d, seed=0)
        c.q, c.lens = q[b:b + 1], [n]
        t = table[b].long()
        c.keys = lambda _, h: tuple(x[t, h].reshape(-1, d)[:n] for x in (k, v))
        c.check(out[b:b + 1], None, lambda _, i, h: torch.ones(n, dtype=torch.bool))


def test_logits_far_apart_and_equal():
    """One key far above the rest, all keys alike, and logits that rise along the axis."""
    from paper_2505_11254_amd import binding
    c = Case([600, 600, 600], [1, 1, 1], 4, 1, 64, seed=8)
    for b in range(3):
        t = c.table[c.slots[b], :10].long()
        u = c.q[b, 0].float()
        for j in range(600):
            f = {0: 4.0 if j == 333 else 0.0, 1: 0.0, 2: j / 600}[b]
            c.k[t[j // 64], 0, j % 64] = (u * f).to(torch.bfloat16)
    for h in range(4):
        c.q[:, h] = c.q[:, 0]
    q, k, v, table, L = c.gpu()
    out = binding.tree_attn_paged(q, k, v, table, L, **c.kw())
    c.check(out, None, lambda b, i, g: torch.ones(600, dtype=torch.bool))


def test_wrong_pages_are_skipped():
    """Entries that name no page hide their keys; a slot out of range, or a length past the table or
    max_len, reads nothing out of place."""
    from paper_2505_11254_amd import binding
    c = Case([300, 200, 90], [1, 2, 1], 8, 2, 128, seed=9)
    c.table[c.slots[0], 1] = 10 ** 6
    c.table[c.slots[0], 3] = -7
    q, k, v, table, L = c.gpu()
    kw = c.kw()
    kw["slots"][2] = 99
    out = binding.tree_attn_paged(q, k, v, table, L, **kw).float().cpu()
    assert (out[c.cu[2]:] == 0).all()
    # (the oracle may have any finite keys there: they are not seen)
    c.table[c.slots[0], 1] = c.table[c.slots[0], 3] = c.table[c.slots[0], 0]
    c.lens, c.news, c.cu = c.lens[:2], c.news[:2], c.cu[:3]

    def visible(b, i, g):
        j = torch.arange(c.lens[b])
        if b == 0:
            return (j // 64 != 1) & (j // 64 != 3)
        return j <= c.lens[b] - c.news[b] + i
    c.check(out, None, visible)
    # a length past the table's room is cut there: what the rows behind the end hold is read, but no more
    L[c.slots[1]] = 10 ** 9
    binding.tree_attn_paged(q[:1], k, v, table, L, slots=kw["slots"][1:2], B=1)
    torch.cuda.synchronize()


@pytest.mark.parametrize("Hq,Hkv,d,top_k", [(8, 2, 64, 5), (32, 8, 128, 16), (28, 4, 128, 3), (64, 1, 64, 40),
                                            (16, 16, 128, 9)])
def test_selected_pages(Hq, Hkv, d, top_k):
    """Lists of every size, empty ones, entries that are no candidate, and several tokens per sequence."""
    from paper_2505_11254_amd import binding
    r = random.Random(top_k)
    lens, news = [1, 64, 65, 700, 3000, 2048, 0], [1, 1, 2, 3, 1, 4, 0]
    c = Case(lens, news, Hq, Hkv, d, seed=top_k)
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
    q, k, v, table, L = c.gpu()
    lse = torch.zeros((q.shape[0], Hq), device="cuda")
    out = binding.selected_attn_paged(q, k, v, table, L, lists.cuda(), lse=lse, **c.kw())

    def visible(b, i, g):
        j = torch.arange(lens[b])
        return torch.isin(j // PAGE, torch.tensor(seen[b, i, g])) & (j <= lens[b] - news[b] + i)
    c.check(out, lse, visible)


def test_streams_graphs_and_workspaces():
    """The call on another stream than the tensors', and captured with a workspace that two graphs
    share, replayed in turn with eager work between."""
    from paper_2505_11254_amd import binding
    a, b = Case([5000, 33], [1, 3], 32, 8, 128, seed=1), Case([900, 4000], [2, 1], 32, 8, 128, seed=2)
    ga, gb = a.gpu(), b.gpu()
    eager = [binding.tree_attn_paged(*g, **c.kw()) for g, c in ((ga, a), (gb, b))]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    on_side = binding.tree_attn_paged(*ga, stream=side, **a.kw())
    side.synchronize()
    assert torch.equal(on_side, eager[0])
    ws = torch.empty(max(binding.paged_workspace_bytes(2, 3, 32, 8, 128, ga[3].shape[1] * 64),
                         binding.paged_workspace_bytes(2, 2, 32, 8, 128, gb[3].shape[1] * 64)), dtype=torch.uint8,
                     device="cuda")
    outs, graphs = [torch.empty_like(x) for x in eager], []
    for g, c, o in ((ga, a, outs[0]), (gb, b, outs[1])):
        kw = c.kw()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            binding.tree_attn_paged(*g, out=o, workspace=ws, **kw)
        graphs.append((graph, kw))
    for _ in range(3):
        for (graph, _), o, want in zip(graphs, outs, eager):
            o.fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(o, want)
        ws.fill_(255)


def test_repeats_are_bitwise_equal():
    from paper_2505_11254_amd import binding
    c = Case([9000, 100, 4000], [1, 1, 1], 32, 8, 128, seed=6)
    g = c.gpu()
    first = binding.tree_attn_paged(*g, **c.kw())
    for _ in range(5):
        assert torch.equal(binding.tree_attn_paged(*g, **c.kw()), first)
