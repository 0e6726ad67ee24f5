"""Pages of a cache on the GPU: forking, resizing with copy on write, appending and
compacting, against the same rules on the host, one request at a time.  Everything is
whole numbers or copies, so every comparison is exact, whole pools included (rows
behind a sequence's last token must stay as they were)."""
from __future__ import annotations

import random

import numpy as np
import pytest
import torch

from paged_sim import PAGE, Cache, pages_of

pytestmark = pytest.mark.gpu


def _t(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


def _filled(seed, layers=2, P=40, Hkv=3, d=64, S=12, M=6, n=5):
    r = random.Random(seed)
    c = Cache(layers, P, Hkv, d, S, M, seed)
    free = list(range(P))
    r.shuffle(free)
    for s in r.sample(range(S), n):
        L = r.choice([1, 63, 64, 65, 100, 128, 200, M * PAGE - 7, M * PAGE])
        k = pages_of(L)
        c.put(s, L, free[:k])
        free = free[k:]
    return r, c


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("d", [64, 128])
def test_random_steps_match_the_rules(seed, d):
    """A run of random calls, wrong requests among them, on one cache."""
    from paper_2505_11254_amd import binding
    r, c = _filled(seed, d=d, P=36, layers=1 + seed % 3)
    g = c.gpu()
    for step in range(14):
        what = r.choice(["fork", "resize", "resize", "compact"])
        n = r.randint(1, 7)
        if what == "fork":
            src = [r.randint(-1, c.S) for _ in range(n)]
            dst = [r.randint(-1, c.S) for _ in range(n)]
            got = binding.pages_fork(g[2], g[3], g[4], _t(src), _t(dst)).tolist()
            assert got == c.fork(src, dst), step
        elif what == "resize":
            slots = [r.randint(-1, c.S) for _ in range(n)]
            new = [r.choice([0, 1, 64, r.randint(0, c.M * PAGE), c.M * PAGE + 1, -3]) if r.random() < 0.4 else
                   min(c.M * PAGE, int(c.lens[s % c.S]) + r.randint(0, 70)) for s in slots]
            got = binding.pages_resize(*g, _t(slots), _t(new)).tolist()
            assert [tuple(x) for x in got] == c.resize(slots, new), step
        else:
            slots, start, keep = [], [], []
            for _ in range(n):
                s = r.randint(0, c.S - 1)
                L = int(c.lens[s])
                st = r.randint(0, L)
                slots.append(s)
                start.append(st if r.random() < 0.9 else L + 1)
                room = range(L - st)
                keep.append(sorted(r.sample(room, r.randint(0, len(room)))) if r.random() < 0.9 else [1, 1])
            cu = np.concatenate([[0], np.cumsum([len(x) for x in keep])]).tolist()
            flat = [x for k in keep for x in k]
            got = binding.pages_compact(*g, _t(slots), _t(start), _t(flat or [0]), _t(cu))[:, 0].tolist()
            assert got == c.compact(slots, start, keep), step
        c.equal(*g)
    binding.pages_resize(*g, _t(list(range(c.S))))
    c.resize(list(range(c.S)), [0] * c.S)
    c.equal(*g)
    assert (c.refs == 0).all()


def test_shared_last_page_of_several_growing_slots():
    """Five slots share a page that is not full; those that grow copy it, and the last keeps it when
    no other slot holds it."""
    from paper_2505_11254_amd import binding
    for growers, holders in (([4, 1, 3], 5), ([4, 1, 3, 0, 2], 5), ([2], 1)):
        c = Cache(2, 20, 2, 128, 6, 4, 1)
        c.put(0, 100, [7, 3])
        c.fork([0] * (holders - 1), list(range(1, holders)))
        if holders == 1:
            c.fork([0], [2])
            c.resize([0], [0])
        g = c.gpu()
        new = [101 + 60 * i for i in range(len(growers))]
        got = binding.pages_resize(*g, _t(growers), _t(new)).tolist()
        assert [tuple(x) for x in got] == c.resize(growers, new)
        c.equal(*g)


def test_pool_that_runs_out():
    from paper_2505_11254_amd import binding
    c = Cache(1, 6, 1, 64, 5, 8, 2)
    c.put(0, 64 * 3, [1, 2, 4])
    c.put(1, 30, [0])
    g = c.gpu()
    # slot 2 takes one of two free pages, slot 3 asks for three, slot 1 would need none but comes later
    got = binding.pages_resize(*g, _t([2, 3, 1, 0]), _t([64, 192, 40, 128])).tolist()
    # (slot 0 shrinks, and its page is given back before any is taken)
    want = c.resize([2, 3, 1, 0], [64, 192, 40, 128])
    assert [tuple(x) for x in got] == want
    assert [x[0] for x in want] == [64, -1, -1, 128]
    c.equal(*g)


def test_large_pool_and_long_slots():
    """More pages than one step of the scan of counts holds, and the most requests a call takes."""
    from paper_2505_11254_amd import binding
    S, M, P = 1100, 40, 40000
    c = Cache(1, 8, 1, 64, S, M, 3)  # (the pages themselves are checked elsewhere)
    c.refs = np.zeros(P, dtype=np.int32)
    c.P = P
    r = random.Random(5)
    c.refs[r.sample(range(P), 20000)] = 3  # held elsewhere
    slots = r.sample(range(S), 1024)
    new = [r.randint(0, 30 * PAGE) for _ in slots]
    k = torch.zeros((P, 1, PAGE, 64), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    t = lambda x: torch.from_numpy(x.copy()).cuda()  # noqa: E731
    table, lens, refs = t(c.table), t(c.lens), t(c.refs)
    for _ in range(2):
        got = binding.pages_resize(k, v, table, lens, refs, _t(slots), _t(new)).tolist()
        c.k = c.v = torch.zeros((1, P, 1, 1, 1))
        assert [tuple(x) for x in got] == c.resize(slots, new)
        np.testing.assert_array_equal(table.cpu().numpy(), c.table)
        np.testing.assert_array_equal(refs.cpu().numpy(), c.refs)
        np.testing.assert_array_equal(lens.cpu().numpy(), c.lens)
        new = [min(M * PAGE, x + r.randint(-200, 900)) if x > 300 else x for x in new]


@pytest.mark.parametrize("Hkv,d,layers", [(1, 64, 1), (8, 128, 3), (5, 128, 1)])
def test_append_writes_the_new_rows_alone(Hkv, d, layers):
    from paper_2505_11254_amd import binding
    r, c = _filled(11, layers=layers, Hkv=Hkv, d=d, P=40, n=6)
    slots = [s for s in range(c.S) if c.lens[s]]
    r.shuffle(slots)
    m = [r.randint(0, min(70, int(c.lens[s]))) for s in slots]
    cu = np.concatenate([[0], np.cumsum(m)]).tolist()
    g = torch.Generator().manual_seed(4)
    k, v = (torch.randn((layers, cu[-1], Hkv, d), generator=g).to(torch.bfloat16) for _ in range(2))
    k[:, 0] = float("nan")  # (copies, whatever the bits)
    dev = c.gpu()
    pages = dev[:2] if layers > 1 else (dev[0][0], dev[1][0])
    kk, vv = (k, v) if layers > 1 else (k[0], v[0])
    binding.pages_append(kk.cuda(), vv.cuda(), *pages, dev[2], dev[3], slots=_t(slots), cu_seqlens=_t(cu),
                         max_seqlen=max(m))
    c.append(slots, cu, k, v)
    c.equal(*dev)


def test_append_skips_what_has_no_place():
    """More new rows than tokens, a slot out of range, and an entry that names no page: nothing is
    written out of place."""
    from paper_2505_11254_amd import binding
    c = Cache(1, 4, 1, 64, 3, 2, 1)
    c.put(0, 3, [2])
    c.put(1, 70, [1, 3])
    c.table[1, 1] = 99  # a page that does not exist
    g = c.gpu()
    k = torch.ones((15, 1, 64), dtype=torch.bfloat16, device="cuda")
    binding.pages_append(k, k, g[0][0], g[1][0], g[2], g[3], slots=_t([0, 1, 7]), B=3)
    for x in (c.k, c.v):
        x[0, 2, :, :3] = 1.0  # rows 2, 3, 4 of slot 0's five
        # slot 1's rows are tokens 65..69, all in the page that does not exist
    c.equal(*g)


@pytest.mark.parametrize("d", [64, 128])
def test_compacting_long_selections(d):
    """Moves of many rows over pages, the chunks of one workgroup among them."""
    from paper_2505_11254_amd import binding
    r = random.Random(d)
    c = Cache(2, 60, 2, d, 3, 20, 9)
    c.put(0, 1200, r.sample(range(60), 19))
    free = [p for p in range(60) if not c.refs[p]]
    c.put(1, 1000, free[:16])
    g = c.gpu()
    keep = [sorted(r.sample(range(1100), 700)), list(range(0, 500))]
    start = [100, 500]
    flat = keep[0] + keep[1]
    got = binding.pages_compact(*g, _t([0, 1]), _t(start), _t(flat), _t([0, 700, 1200]))[:, 0].tolist()
    assert got == c.compact([0, 1], start, keep) == [700, 500]
    c.equal(*g)


def test_compacting_refuses_shared_pages():
    from paper_2505_11254_amd import binding
    c = Cache(1, 10, 1, 64, 4, 3, 4)
    c.put(0, 150, [5, 6, 7])
    c.fork([0], [1])
    c.resize([1], [160])  # slot 1 gets a last page of its own; the first two stay shared
    g = c.gpu()
    args = (_t([0, 1]), _t([60, 130]), _t([3, 4, 5, 9]), _t([0, 2, 4]))
    got = binding.pages_compact(*g, *args)[:, 0].tolist()
    assert got == c.compact([0, 1], [60, 130], [[3, 4], [5, 9]]) == [-1, 2]
    c.equal(*g)


def test_calls_replay_in_a_graph():
    """A step of fork, growth, append and compaction, captured once and replayed with the program's own
    copies between."""
    from paper_2505_11254_amd import binding
    c = Cache(2, 30, 2, 64, 6, 4, 7)
    c.put(0, 100, [9, 4])
    g = c.gpu()
    src, dst, new = _t([0, 0]), _t([3, 5]), _t([110, 105])
    k = torch.randn((2, 15, 2, 64), device="cuda").to(torch.bfloat16)
    cu, start, keep, cu_keep = _t([0, 10, 15]), _t([100, 100]), _t([1, 4, 7, 2]), _t([0, 3, 4])
    res = [_t([0] * 2), _t([[0] * 4] * 2), _t([[0] * 4] * 2)]

    def step():
        binding.pages_resize(*g, dst, result=res[1])
        binding.pages_fork(*g[2:], src, dst, result=res[0])
        binding.pages_resize(*g, dst, new, result=res[1])
        binding.pages_append(k, k, *g[:4], slots=dst, cu_seqlens=cu, max_seqlen=10)
        binding.pages_compact(*g, dst, start, keep, cu_keep, result=res[2])

    def host():
        c.resize([3, 5], [0, 0])
        c.fork([0, 0], [3, 5])
        c.resize([3, 5], [110, 105])
        c.append([3, 5], [0, 10, 15], k.cpu(), k.cpu())
        c.compact([3, 5], [100, 100], [[1, 4, 7], [2]])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    host()
    c.equal(*g)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        graph.replay()
        host()
        torch.cuda.synchronize()
        c.equal(*g)
        step()  # (an eager pass between the replays)
        host()
        c.equal(*g)


def test_append_after_a_refused_growth():
    """Branches that share a page grow past the pool: slots whose growth was refused, and the pages that
    others hold with them, keep every token, in a step that is captured whole, until pages are
    free again."""
    from paper_2505_11254_amd import binding
    c = Cache(2, 7, 2, 64, 5, 4, 8)
    c.put(0, 100, [5, 2])
    c.fork([0, 0, 0], [1, 2, 3])
    c.put(4, 128, [0, 6])
    g = c.gpu()
    slots, kept = [3, 1, 2, 0], _t([4])
    new = _t([0] * 4)
    m, cu = [2, 30, 1, 5], [0, 2, 32, 33, 38]
    k, v = (torch.randn((2, cu[-1], 2, 64), generator=torch.Generator().manual_seed(x)).to(torch.bfloat16) for x in (1, 2))
    on = (k.cuda(), v.cuda(), _t(slots), _t(cu))
    res = _t([[0] * 4] * 4)

    def step():
        binding.pages_resize(*g, on[2], new, result=res)
        binding.pages_append(*on[:2], *g[:4], slots=on[2], cu_seqlens=on[3], max_seqlen=30, new_lens=new)

    def host(ask):
        got = c.resize(slots, ask)
        ok = [x[0] >= 0 for x in got]
        rows = [i for b in range(4) if ok[b] for i in range(cu[b], cu[b + 1])]
        ends = [0]
        for b in range(4):
            if ok[b]:
                ends.append(ends[-1] + m[b])
        c.append([s for b, s in enumerate(slots) if ok[b]], ends, k[:, rows], v[:, rows])
        return got
    # (three pages are free: slot 3 copies the shared page, slot 1 copies it and takes one more; slot 2, which
    # would copy it too, finds none, and slot 0 comes after it)
    ask = [102, 130, 101, 105]
    new.copy_(_t(ask))
    step()
    got = host(ask)
    assert [x[0] for x in got] == [102, 130, -1, -1] and res.tolist() == [list(x) for x in got]
    c.equal(*g)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        if i == 2:  # pages are free again
            binding.pages_resize(*g, kept)
            c.resize([4], [0])
        ask = [int(c.lens[s]) + x for s, x in zip(slots, m)]
        new.copy_(_t(ask))
        graph.replay()
        torch.cuda.synchronize()
        got = host(ask)
        assert res.tolist() == [list(x) for x in got]
        c.equal(*g)
        assert (min(x[0] for x in got) < 0) == (i < 2)


def test_append_checks_new_lens():
    from paper_2505_11254_amd import binding
    c = Cache(1, 4, 1, 64, 3, 2, 1)
    g = c.gpu()
    k = torch.ones((4, 1, 64), dtype=torch.bfloat16, device="cuda")
    for bad in (_t([1]), _t([1, 2, 3]), _t([1, 2]).long(), torch.zeros(2, dtype=torch.int32)):
        with pytest.raises((ValueError, TypeError)):
            binding.pages_append(k, k, g[0][0], g[1][0], g[2], g[3], B=2, new_lens=bad)


def test_append_to_a_page_past_32_bits():
    """One page of more than 2^31 elements: its last kv heads' rows."""
    from paper_2505_11254_amd import binding
    Hkv, d = (1 << 18) + 3, 128
    kp = torch.zeros((1, Hkv, PAGE, d), dtype=torch.bfloat16, device="cuda")
    vp = torch.zeros_like(kp)
    assert kp.numel() > 1 << 31
    k = torch.randn((3, Hkv, d), device="cuda", dtype=torch.bfloat16)
    v = torch.randn_like(k)
    binding.pages_append(k, v, kp, vp, _t([[0]]), _t([PAGE - 1]), B=1)
    for pages, want in ((kp, k), (vp, v)):
        assert torch.equal(pages[0, :, 60:63], want.transpose(0, 1))
        assert not pages[0, :, :60].any() and not pages[0, :, 63:].any()


def test_compaction_after_a_refused_growth():
    """The drafts of a slot that found no page are not there to be kept: its compaction is refused and the
    slot stays as it was; with nothing to keep it changes nothing either."""
    from paper_2505_11254_amd import binding
    c = Cache(2, 3, 1, 64, 2, 3, 5)
    c.put(0, 60, [2])
    c.put(1, 128, [0, 1])
    g = c.gpu()
    slots, new, cu = [0, 1], [62, 131], [0, 2, 5]
    k = torch.randn((2, 5, 1, 64)).to(torch.bfloat16)
    got = binding.pages_resize(*g, _t(slots), _t(new)).tolist()
    assert [tuple(x) for x in got] == c.resize(slots, new) and [x[0] for x in got] == [62, -1]
    on = k.cuda()
    binding.pages_append(on, on, *g[:4], slots=_t(slots), cu_seqlens=_t(cu), max_seqlen=3, new_lens=_t(new))
    c.append([0], [0, 2], k[:, :2], k[:, :2])
    c.equal(*g)
    for keep in ([[1], [0, 2]], [[0], []]):
        flat, ends = keep[0] + keep[1], [0, len(keep[0]), len(keep[0] + keep[1])]
        got = binding.pages_compact(*g, _t(slots), _t([60, 128]), _t(flat), _t(ends))[:, 0].tolist()
        assert got == c.compact(slots, [60, 128], keep) == ([1, -1] if keep[1] else [1, 0])
        c.equal(*g)
