"""The 8-bit cache on the GPU against its rules on the host: codes, scales, tables and copies exactly."""
from __future__ import annotations

import random

import pytest
import torch

from pages8_sim import NAN, VALUES, Cache8, codes
from paged_sim import PAGE, attend, pages_of, summary

pytestmark = pytest.mark.gpu


def i32(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


def put(c, slot, n, pages):
    """A slot of n tokens in these pages: finite codes."""
    c.put(slot, n, pages)
    for p in pages[:pages_of(n)]:
        for x in (c.k, c.v):
            x[:, p] = torch.where((x[:, p] & 0x7F) == NAN, 0, x[:, p])


def wide(g, *shape):
    """Values of magnitudes far apart, zeros among them."""
    x = torch.randn(shape, generator=g) * torch.pow(2.0, torch.randint(-30, 12, shape[:-1] + (1,), generator=g).double()).float()
    return torch.where(torch.rand(shape, generator=g) < 0.05, 0.0, x).to(torch.bfloat16)


@pytest.mark.parametrize("layers,Hkv,d", [(1, 2, 64), (2, 3, 128), (1, 8, 128), (3, 1, 64)])
def test_append_in_pieces_and_read_back(layers, Hkv, d):
    """Prompts, chunks and single tokens of magnitudes far apart, one after the other: scales grow, older codes
    are recoded, full pages and rows behind the end stay."""
    from paper_2505_11254_amd import binding
    c = Cache8(layers, 30, Hkv, d, 5, 6, seed=d)
    g, r = torch.Generator().manual_seed(layers), random.Random(Hkv)
    dev = c.gpu8()
    lens = [0] * 5
    for step in range(9):
        slots = r.sample(range(5), r.randint(1, 4))
        news = [r.choice([1, 1, 1, 2, 17, 63, 64, 65, 130]) for _ in slots]
        news = [min(m, 6 * PAGE - lens[s]) for s, m in zip(slots, news)]
        slots, news = zip(*[(s, m) for s, m in zip(slots, news) if m] or [(0, 0)])
        if not news[0]:
            continue
        want = [lens[s] + m for s, m in zip(slots, news)]
        got = binding.pages8_resize(*dev, i32(slots), i32(want))
        assert got.cpu().tolist() == [list(x) for x in c.resize(list(slots), want)]
        cu = [0]
        for s, m in zip(slots, news):
            lens[s] += m
            cu.append(cu[-1] + m)
        k, v = wide(g, layers, cu[-1], Hkv, d), wide(g, layers, cu[-1], Hkv, d)
        one = (lambda x: x[0]) if layers == 1 else (lambda x: x)  # noqa: E731
        binding.pages8_append(one(k).contiguous().cuda(), one(v).contiguous().cuda(), *dev[:6], slots=i32(slots), cu_seqlens=i32(cu),
                              max_seqlen=max(news), new_lens=i32(want) if step % 2 else None)
        c.append8(slots, cu, k, v)
        c.equal8(*dev)
    # read back: whole slots, parts from the middle of pages, more rows than there are tokens
    first = [0, 5, 64, 100, 3]
    count = [max(0, n - f) + e for n, f, e in zip(lens, first, (0, 3, 0, 70, 1))]
    cu = [0]
    for m in count:
        cu.append(cu[-1] + m)
    marks = [torch.full((layers, cu[-1], Hkv, d) if layers > 1 else (cu[-1], Hkv, d), 7.0, dtype=torch.bfloat16, device="cuda")
             for _ in range(2)]
    got = binding.pages8_read(*dev[:6], cu[-1], first=i32(first), cu_seqlens=i32(cu), max_seqlen=max(count), k=marks[0],
                              v=marks[1])
    for name, x in zip("kv", got):
        x = x.float().cpu().double().view(layers, cu[-1], Hkv, d)
        for b, n in enumerate(lens):
            have = max(0, n - first[b])
            assert (x[:, cu[b] + have:cu[b + 1]] == 7.0).all()
            for layer in range(layers):
                for h in range(Hkv):
                    if have:
                        assert torch.equal(x[layer, cu[b]:cu[b] + have, h], c.rows(name, layer, b, h, first[b], n))


@pytest.mark.parametrize("peak", [-1, -133, -126, -120, -101, -3, 0, 8, 100, 127])
def test_every_bf16_value(peak):
    """All 65536 bit patterns beside a page's largest magnitude of about 2^peak (-1: whatever they are):
    subnormals, infinities and NaN among them."""
    from paper_2505_11254_amd import binding
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    if peak != -1:
        x = x[(x.double().abs() <= 2.0 ** peak * 1.9) | ~torch.isfinite(x.double())]
    d, Hkv = 128, 1
    x = torch.cat([x, x.new_zeros(-len(x) % d)]).view(1, -1, Hkv, d)
    T = x.shape[1]
    c = Cache8(1, pages_of(T) + 1, Hkv, d, 1, pages_of(T), seed=1)
    c.put(0, T, list(range(pages_of(T))))
    dev = c.gpu8()
    binding.pages8_append(x[0].cuda(), x[0].flip(0).contiguous().cuda(), *dev[:6])
    c.append8([0], [0, T], x, x.flip(1))
    c.equal8(*dev)
    k, _ = binding.pages8_read(*dev[:6], T)
    k = k.cpu().double().view(T, d)
    want = c.rows("k", 0, 0, 0, 0, T)
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(k), nan) and torch.equal(k[~nan], want[~nan])
    big = ~nan & (x[0, :, 0].double().abs() <= 448 * 2.0 ** 119)
    unit = torch.pow(2.0, c.ke[0, torch.arange(T) // PAGE, 0].double())[:, None]
    assert ((k - x[0, :, 0].double()).abs()[big] <= torch.maximum(x[0, :, 0].double().abs() * 2 ** -4, unit * 2 ** -10)[big]).all()


def test_writes_that_are_left_out():
    """Lengths that are not the ones asked for, slots and pages that do not exist, rows before a slot's first token."""
    from paper_2505_11254_amd import binding
    g = torch.Generator().manual_seed(2)
    c = Cache8(1, 9, 2, 64, 4, 3, seed=3)
    put(c, 0, 70, [3, 1])
    put(c, 1, 30, [2])
    put(c, 2, 100, [4, 5])
    put(c, 3, 20, [6])
    dev = list(c.gpu8())
    dev[4][2, 1] = 1000  # not a page
    k, v = wide(g, 1, 14, 2, 64), wide(g, 1, 14, 2, 64)
    # slot 0: written; 1: another length was asked for; 99: no slot; 2: its page does not exist
    binding.pages8_append(k[0].cuda(), v[0].cuda(), *dev[:6], slots=i32([0, 1, 99, 2]), cu_seqlens=i32([0, 10, 12, 13, 14]),
                          max_seqlen=10, new_lens=i32([70, 31, 5, 100]))
    c.append8([0], [0, 10], k, v)
    dev[4][2, 1] = 5
    c.equal8(*dev)
    # more rows than the slot has tokens: the last ones are its tokens
    k, v = wide(g, 1, 25, 2, 64), wide(g, 1, 25, 2, 64)
    binding.pages8_append(k[0].cuda(), v[0].cuda(), *dev[:6], slots=i32([3]))
    c.append8([3], [0, 20], k[:, 5:], v[:, 5:])
    c.equal8(*dev)
    # offsets outside the rows, and reads of what is not there
    binding.pages8_append(k[0].cuda(), v[0].cuda(), *dev[:6], slots=i32([1]), cu_seqlens=i32([20, 30]), max_seqlen=10)
    c.equal8(*dev)
    rows = torch.full((6, 2, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    for kw in (dict(first=i32([-1])), dict(first=i32([30])), dict(first=i32([2 ** 31 - 1]))):
        a, b = binding.pages8_read(*dev[:6], 6, slots=i32([1]), k=rows, v=rows.clone(), **kw)
        assert (a == 3.0).all() and (b == 3.0).all()
    a, _ = binding.pages8_read(*dev[:6], 6, slots=i32([77]), k=rows)
    assert (a == 3.0).all()


@pytest.mark.parametrize("layers,Hkv,d", [(1, 2, 64), (2, 3, 128)])
def test_a_step_of_all_calls(layers, Hkv, d):
    """Fork, grow with copies on write, append, attend to a tree, keep the accepted path, read back: steps in a row."""
    from paper_2505_11254_amd import binding
    c = Cache8(layers, 40, Hkv, d, 6, 5, seed=9)
    put(c, 0, 90, [7, 3])
    put(c, 1, 64, [5])
    dev = c.gpu8()
    g, r = torch.Generator().manual_seed(d), random.Random(7)
    assert binding.pages_fork(dev[4], dev[5], dev[6], i32([0, 0, 1]), i32([2, 3, 4])).cpu().tolist() == c.fork([0, 0, 1], [2, 3, 4])
    for step in range(4):
        slots = [0, 2, 3, 4]
        start = [int(c.lens[s]) for s in slots]
        news = [r.randint(1, 40) for _ in slots]
        want = [a + m for a, m in zip(start, news)]
        got = binding.pages8_resize(*dev, i32(slots), i32(want))
        assert got.cpu().tolist() == [list(x) for x in c.resize(slots, want)]
        cu = [0]
        for m in news:
            cu.append(cu[-1] + m)
        k, v = (torch.randn((layers, cu[-1], Hkv, d), generator=g) * 2.0 ** (step - 1) for _ in range(2))
        k, v = k.to(torch.bfloat16), v.to(torch.bfloat16)
        rows = [x if layers > 1 else x[0] for x in (k, v)]
        binding.pages8_append(*(x.contiguous().cuda() for x in rows), *dev[:6], slots=i32(slots), cu_seqlens=i32(cu),
                              max_seqlen=max(news), new_lens=i32(want))
        c.append8(slots, cu, k, v)
        c.equal8(*dev)
        parents = [[r.randint(-1, i - 1) for i in range(m)] for m in news]
        mask = binding.tree_mask(parents, "cuda")
        q = torch.randn((cu[-1], 2 * Hkv, d), generator=g).to(torch.bfloat16)
        layer = step % layers
        pages = [x if layers == 1 else x[layer] for x in dev[:4]]
        out = binding.tree_attn_paged8(q.cuda(), *pages, dev[4], dev[5], mask=mask, slots=i32(slots), cu_seqlens=i32(cu),
                                       max_seqlen=max(news)).float().cpu().double()
        seen = mask.cpu()
        for b, s in enumerate(slots):
            for h in range(Hkv):
                kk, vv = (c.rows(x, layer, s, h, 0, want[b]) for x in "kv")
                vis = torch.ones((news[b], want[b]), dtype=torch.bool)
                for i in range(news[b]):
                    w = seen[cu[b] + i].tolist()
                    vis[i, start[b]:] = torch.tensor([bool(w[j // 64] >> j % 64 & 1) for j in range(news[b])])
                heads = slice(2 * h, 2 * h + 2)
                qq = q[cu[b]:cu[b + 1], heads].reshape(-1, d)
                vis = vis.repeat_interleave(2, 0)
                o, _ = attend(qq, kk, vv, vis)
                sq, _ = attend(qq, kk, vv ** 2, vis)
                dev_ = (sq - o ** 2).clamp(min=0).sqrt()
                # (logits: d products in fp32, as in scored.py)
                dl = 2 * (d * 2.0 ** -24 * float((qq.double().abs() @ kk.abs().T).max()) / d ** 0.5 + 2.0 ** -15)
                tol = 2.0 ** -8 * o.abs() + (2.0 ** -8 + dl) * (1 + 2.0 ** -7) * dev_ + 1e-6 * float(vv.abs().max())
                assert ((out[cu[b]:cu[b + 1], heads].reshape(-1, d) - o).abs() <= tol).all()
        keep = []
        for m, p in zip(news, parents):
            path, i = [], r.randint(-1, m - 1)
            while i >= 0:
                path.append(i)
                i = p[i]
            keep.append(path[::-1])
        ck = [0]
        for p in keep:
            ck.append(ck[-1] + len(p))
        got = binding.pages8_compact(*dev, i32(slots), i32(start), i32([x for p in keep for x in p] or [0]), i32(ck))
        assert got[:, 0].cpu().tolist() == c.compact8(slots, start, keep)
        c.equal8(*dev)
    n = int(c.lens[3])
    k, v = binding.pages8_read(*dev[:6], n, slots=i32([3]))
    for name, x in (("k", k), ("v", v)):
        for layer in range(layers):
            for h in range(Hkv):
                got = (x if layers == 1 else x[layer])[:, h].float().cpu().double()
                assert torch.equal(got, c.rows(name, layer, 3, h, 0, n))


@pytest.mark.parametrize("d,Hkv", [(64, 3), (128, 2)])
def test_compact_over_pages_of_different_scales(d, Hkv):
    """Rows move over several pages whose scales lie far apart; refused requests change nothing."""
    from paper_2505_11254_amd import binding
    r = random.Random(d)
    c = Cache8(1, 30, Hkv, d, 4, 8, seed=5)
    put(c, 0, 450, [3, 9, 1, 12, 7, 20, 21, 22])
    put(c, 1, 200, [4, 5, 6, 8])
    put(c, 2, 128, [10, 11])
    c.ke[:] = torch.randint(-40, 30, c.ke.shape, generator=torch.Generator().manual_seed(1))
    c.ve[0, 9] += 25
    c.fork([2], [3])
    dev = c.gpu8()
    slots, start = [0, 1, 2, 0, 3], [37, 0, 60, 5, 64]
    keep = [sorted(r.sample(range(413), 300)), sorted(r.sample(range(200), 71)), [0, 1, 5], [0], [3, 2]]
    ck = [0]
    for p in keep:
        ck.append(ck[-1] + len(p))
    got = binding.pages8_compact(*dev, i32(slots), i32(start), i32([x for p in keep for x in p]), i32(ck))
    assert got[:, 0].cpu().tolist() == c.compact8(slots, start, keep)
    c.equal8(*dev)
    # nothing kept, all kept, and a slot emptied
    got = binding.pages8_compact(*dev, i32([0, 1]), i32([100, 0]), i32(list(range(71))), i32([0, 0, 71]))
    assert got[:, 0].cpu().tolist() == c.compact8([0, 1], [100, 0], [[], list(range(71))])
    c.equal8(*dev)
    got = binding.pages8_resize(*dev, i32([0, 1, 2, 3]))
    assert got[:, 0].cpu().tolist() == [0, 0, 0, 0] and (dev[6] == 0).all()


@pytest.mark.parametrize("d,Hkv", [(64, 3), (128, 8)])
def test_summaries(d, Hkv):
    from paper_2505_11254_amd import binding
    c = Cache8(1, 12, Hkv, d, 2, 6, seed=4)
    put(c, 0, 300, [3, 9, 1, 2, 7])
    put(c, 1, 63, [5])
    c.ke[:] = torch.randint(-100, 100, c.ke.shape, generator=torch.Generator().manual_seed(1))
    dev = c.gpu8()
    got, scales = torch.zeros((12, Hkv, d), dtype=torch.int8, device="cuda"), torch.zeros((12, Hkv), device="cuda")
    binding.page8_summary(dev[0], dev[2], dev[4], dev[5], got, scales)
    for j, p in enumerate([3, 9, 1, 2]):
        for h in range(Hkv):
            want, ws = summary(c.rows("k", 0, 0, h, 64 * j, 64 * j + 64)[None])
            assert torch.equal(got[p, h].cpu().long(), want[0]) and scales[p, h].cpu() == ws[0]
    rest = [p for p in range(12) if p not in (3, 9, 1, 2)]
    assert (got[rest] == 0).all() and (scales[rest] == 0).all()


def test_a_captured_step_replays():
    """Resize, append and read in one graph, replayed with other tokens and eager work between, on the pages as the
    replays before left them."""
    from paper_2505_11254_amd import binding
    c = Cache8(1, 20, 2, 64, 2, 8, seed=6)
    put(c, 0, 60, [3])
    put(c, 1, 10, [4])
    dev = c.gpu8()
    k, v = (torch.zeros((6, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    slots, want, first = i32([0, 1]), i32([63, 13]), i32([60, 10])
    result = torch.zeros((2, 4), dtype=torch.int32, device="cuda")
    rk, rv = torch.zeros_like(k), torch.zeros_like(v)

    def step():
        binding.pages8_resize(*dev, slots, want, result=result)
        binding.pages8_append(k, v, *dev[:6], slots=slots, B=2, new_lens=want)
        binding.pages8_read(*dev[:6], 6, first=first, slots=slots, B=2, k=rk, v=rv)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    g = torch.Generator().manual_seed(8)
    for n in range(6):
        x, y = (torch.randn((1, 6, 2, 64), generator=g) * 2.0 ** n for _ in range(2))
        x, y = x.to(torch.bfloat16), y.to(torch.bfloat16)
        k.copy_(x[0])
        v.copy_(y[0])
        lens = [63 + 3 * n, 13 + 3 * n]
        want.copy_(i32(lens))
        first.copy_(i32([z - 3 for z in lens]))
        graph.replay()
        torch.cuda.synchronize()
        c.resize([0, 1], lens)
        c.append8([0, 1], [0, 3, 6], x, y)
        c.equal8(*dev)
        for h in range(2):
            got = rk[:, h].float().cpu().double()
            assert torch.equal(got, torch.cat([c.rows("k", 0, s, h, lens[s] - 3, lens[s]) for s in (0, 1)]))


def test_codes_of_the_host_are_e4m3():
    """(of the oracle itself: against the cast that torch has)"""
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).float()
    x = x[torch.isfinite(x) & (x.abs() <= 448)]
    assert torch.equal(codes(x), x.to(torch.float8_e4m3fn).view(torch.uint8))
    assert torch.equal(VALUES[:127].float(), torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).float())


def test_pages_past_four_gigabytes():
    """Offsets inside the pages past 32 bits: written, read back, attended to, compacted."""
    from paper_2505_11254_amd import binding
    P, Hkv, d = 66_000, 8, 128
    k8, v8 = (torch.zeros((P, Hkv, PAGE, d), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    ks, vs = (torch.ones((P, Hkv), device="cuda") for _ in range(2))
    c = Cache8(1, 4, Hkv, d, 1, 3, seed=2)
    put(c, 0, 150, [0, 1, 2])
    far = [P - 1, P - 3, P - 2]
    table, lens = i32([far]), i32([150])
    refs = torch.zeros(P, dtype=torch.int32, device="cuda")
    refs[far] = 1
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn((1, 150, Hkv, d), generator=g).to(torch.bfloat16) for _ in range(2))
    cache = (k8, v8, ks, vs, table, lens)
    binding.pages8_append(k[0].cuda(), v[0].cuda(), *cache)
    c.append8([0], [0, 150], k, v)
    q = torch.randn((1, Hkv, d), generator=g).to(torch.bfloat16)
    out = binding.tree_attn_paged8(q.cuda(), *cache).float().cpu().double()
    for h in range(Hkv):
        kk, vv = (c.rows(x, 0, 0, h, 0, 150) for x in "kv")
        want, _ = attend(q[:, h], kk, vv, torch.ones((1, 150), dtype=torch.bool))
        assert (out[:, h] - want).abs().max() <= 2.0 ** -7 * max(1.0, float(vv.abs().max()))
    got = binding.pages8_compact(*cache, refs, i32([0]), i32([10]), i32([3, 77, 139]), i32([0, 3]))
    assert got[:, 0].cpu().tolist() == c.compact8([0], [10], [[3, 77, 139]]) == [3]
    rk, rv = binding.pages8_read(*cache, 13)
    for name, x in (("k", rk), ("v", rv)):
        for h in range(Hkv):
            assert torch.equal(x[:, h].float().cpu().double(), c.rows(name, 0, 0, h, 0, 13))
    assert (k8.view(torch.uint8)[:P - 3] == 0).all()
