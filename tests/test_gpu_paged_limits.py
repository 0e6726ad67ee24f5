"""The paged cache, the attention over it and the block selection at the ends of what they
take: caches past 2^32 elements, the longest prompt, batches without tokens, rows behind
the last sequence, steps captured into graphs, and calls that the binding refuses.
Tolerances as in test_gpu_paged_attn; lists and copies are compared exactly."""
from __future__ import annotations

import pytest
import torch

from paged_sim import PAGE, choose, summary
from test_gpu_paged_attn import Case

pytestmark = pytest.mark.gpu


def _t(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


def _bf16(shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


def test_pages_past_32_bits():
    """A pool of more than 2^32 elements: every call on its far pages."""
    from paper_2505_11254_amd import binding
    P, Hkv, Hq, d, n = 66000, 8, 16, 128, 222
    kp = torch.zeros((P, Hkv, PAGE, d), dtype=torch.bfloat16, device="cuda")
    vp = torch.zeros_like(kp)
    assert kp.numel() > 1 << 32
    ids = [65999, 65536, 40000, 65535]
    table = torch.full((2, 8), -1, dtype=torch.int32)
    table[0, :4] = torch.tensor(ids, dtype=torch.int32)
    table, lens = table.cuda(), _t([n, 0])
    refs = torch.ones(P, dtype=torch.int32, device="cuda")
    refs[65998] = 0
    k, v = _bf16((n, Hkv, d), 1), _bf16((n, Hkv, d), 2)
    binding.pages_append(k.cuda(), v.cuda(), kp, vp, table, lens, slots=_t([0]))

    def held(s, m):
        row = table[s].cpu().tolist()
        return tuple(torch.cat([x[e].cpu().transpose(0, 1) for e in row[:-(-m // PAGE)]])[:m] for x in (kp, vp))
    for got, want in zip(held(0, n), (k, v)):
        assert torch.equal(got, want)
    # a fork, whose growth copies its last page to the only free one
    assert binding.pages_fork(table, lens, refs, _t([0]), _t([1])).tolist() == [n]
    assert binding.pages_resize(kp, vp, table, lens, refs, _t([1]), _t([n + 3])).tolist() == [[n + 3, 65535, 65998, 30]]
    nk, nv = _bf16((3, Hkv, d), 3), _bf16((3, Hkv, d), 4)
    binding.pages_append(nk.cuda(), nv.cuda(), kp, vp, table, lens, slots=_t([1]))
    hk, hv = torch.cat([k, nk]), torch.cat([v, nv])
    for got, want in zip(held(1, n + 3), (hk, hv)):
        assert torch.equal(got, want)
    # attention and selection over the fork
    c = Case([n + 3], [1], Hq, Hkv, d, seed=5)
    c.keys = lambda b, g: (hk[:, g], hv[:, g])
    q = c.q.cuda()
    out = binding.tree_attn_paged(q, kp, vp, table, lens, slots=_t([1]))
    c.check(out, None, lambda b, i, g: torch.ones(n + 3, dtype=torch.bool))
    codes = torch.zeros((P, Hkv, d), dtype=torch.int8, device="cuda")
    scales = torch.zeros((P, Hkv), device="cuda")
    binding.page_summary(kp, table, lens, codes, scales, slots=_t([1]))
    pages = binding.select_pages(q, codes, scales, table, lens, top_k=2, n_sink=0, n_recent=1, slots=_t([1]))
    for g in range(Hkv):
        x, s = summary(hk[:3 * PAGE, g].reshape(-1, PAGE, d))
        assert pages[0, g].tolist() == choose(c.q[0, 2 * g:2 * g + 2], x, s, 2, 0, 1)
    listed = pages.cpu()
    out = binding.selected_attn_paged(q, kp, vp, table, lens, pages, slots=_t([1]))
    c.check(out, None, lambda b, i, g: torch.isin(torch.arange(n + 3) // PAGE, listed[0, g]) | (torch.arange(n + 3) >= 192))
    # the fork is dropped, so that slot 0's pages are its own, and some of its tokens are kept
    binding.pages_resize(kp, vp, table, lens, refs, _t([1]))
    keep = [0, 1, 50, 51, 100, 160]
    got = binding.pages_compact(kp, vp, table, lens, refs, _t([0]), _t([60]), _t(keep), _t([0, 6]))
    assert got[0, 0].item() == 6
    rows = list(range(60)) + [60 + x for x in keep]
    for got, want in zip(held(0, 66), (k[rows], v[rows])):
        assert torch.equal(got, want)
    assert table[0].tolist() == ids[:2] + [-1] * 6


def test_the_longest_prompt():
    """24576 key tiles: as many candidates as a list's scores have room for."""
    from paper_2505_11254_amd import binding
    T, d, bq, top_k = 24576 * PAGE, 64, 256, 8
    q = torch.randn((T, 1, d), generator=torch.Generator("cuda").manual_seed(1), device="cuda", dtype=torch.bfloat16)
    g = torch.Generator().manual_seed(2)
    codes = torch.randint(-127, 128, (T // PAGE + 1, 1, d), generator=g).to(torch.int8)
    scales = torch.rand((T // PAGE + 1, 1), generator=g).bfloat16().float()
    ptr, idx = binding.select_blocks(q, codes.cuda(), scales.cuda(), top_k=top_k, block_q=bq)
    ptr = ptr[0, 0].tolist()
    for j in (0, 1, 2, 3, 255, 256, 257, 4000, 6143):
        rows = q[j * bq:(j + 1) * bq, 0].cpu()
        want = choose(rows, codes[:4 * j, 0].long(), scales[:4 * j, 0], top_k, 1, 1)
        assert idx[ptr[j]:ptr[j + 1]].tolist() == want, j


@pytest.mark.parametrize("B", [2, 100])
def test_rows_behind_the_last_sequence_stay(B):
    """A batch padded with rows that no sequence has, and one in which no sequence has any."""
    from paper_2505_11254_amd import binding
    c = Case([130, 40], [2, 1], 8, 2, 64, seed=3)
    q, k, v, table, L = c.gpu()
    q = torch.cat([q, torch.full((4, 8, 64), float("nan"), dtype=torch.bfloat16, device="cuda")])
    codes = torch.zeros((k.shape[0], 2, 64), dtype=torch.int8, device="cuda")
    scales = torch.zeros((k.shape[0], 2), device="cuda")
    slots = _t(c.slots + [c.slots[0]] * (B - 2))
    for ends in ([0, 2] + [3] * (B - 1), [0] * (B + 1)):
        n = ends[-1]
        out = torch.full_like(q, 7.0)
        lse = torch.full(q.shape[:2], 7.0, device="cuda")
        pages = torch.full((q.shape[0], 2, 3), 7, dtype=torch.int32, device="cuda")
        kw = dict(slots=slots, cu_seqlens=_t(ends), max_seqlen=2)
        binding.tree_attn_paged(q, k, v, table, L, out=out, lse=lse, **kw)
        assert (out[n:] == 7).all() and (lse[n:] == 7).all() and torch.isfinite(out[:n].float()).all()
        if n:
            c.check(out[:n], lse[:n], lambda b, i, g: torch.arange(c.lens[b]) <= c.lens[b] - c.news[b] + i)
        binding.select_pages(q, codes, scales, table, L, top_k=3, pages=pages, **kw)
        assert (pages[n:] == 7).all()
        out.fill_(7.0)
        binding.selected_attn_paged(q, k, v, table, L, pages, out=out, **kw)
        assert (out[n:] == 7).all() and torch.isfinite(out[:n].float()).all()


def test_sparse_steps_replay_in_graphs():
    """A step of summaries, selection and attention captured twice with one workspace, replayed in turn
    with eager work between, after lengths have changed."""
    from paper_2505_11254_amd import binding
    Hq, Hkv, d, top_k = 8, 2, 128, 6
    c = Case([3000, 700], [1, 1], Hq, Hkv, d, seed=4)
    q, k, v, table, L = c.gpu()
    k, v = k.nan_to_num(0.5, 0.5, 0.5), v.nan_to_num(0.5, 0.5, 0.5)
    slots = _t(c.slots)
    codes = torch.zeros((k.shape[0], Hkv, d), dtype=torch.int8, device="cuda")
    scales = torch.zeros((k.shape[0], Hkv), device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")

    def step(pages, out, **kw):
        binding.page_summary(k, table, L, codes, scales, slots=slots)
        binding.select_pages(q, codes, scales, table, L, top_k=top_k, slots=slots, B=2, pages=pages, **kw)
        return binding.selected_attn_paged(q, k, v, table, L, pages, slots=slots, B=2, out=out, **kw)
    new = lambda: (torch.zeros((2, Hkv, top_k), dtype=torch.int32, device="cuda"), torch.zeros_like(q))  # noqa: E731
    eager, held = new(), [new(), new()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(*eager, stream=side)
    side.synchronize()
    graphs = []
    for x in held:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            step(*x, workspace=ws)
    for less in (0, 100, 640):
        L[c.slots[0]] = 3000 - less
        step(*eager)
        for graph, x in zip(graphs, held):
            for y in x:
                y.fill_(3)
            graph.replay()
            for y, want in zip(x, eager):
                assert torch.equal(y, want)
            ws.fill_(255)


def test_prompt_selection_replays_in_a_graph():
    from paper_2505_11254_amd import binding
    q, k = _bf16((900, 4, 64), 1).cuda(), _bf16((900, 2, 64), 2).cuda()
    cu = _t([0, 500, 900])
    sums = binding.key_summary(k, cu_seqlens=cu, max_seqlen=900)
    lists = binding.select_blocks(q, *sums, top_k=3, block_q=64, cu_seqlens=cu, max_seqlen=900)

    def step():
        binding.key_summary(k, cu_seqlens=cu, max_seqlen=900, codes=sums[0], scales=sums[1])
        binding.select_blocks(q, *sums, top_k=3, block_q=64, cu_seqlens=cu, max_seqlen=900, block_ptr=lists[0],
                              block_idx=lists[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for ends in ([0, 500, 900], [0, 900, 900], [0, 10, 333]):
        cu.copy_(_t(ends))
        step()
        want = [x.clone() for x in lists]
        for x in lists:
            x.fill_(-5)
        sums[0].fill_(1)
        graph.replay()
        for x, y in zip(lists, want):
            assert torch.equal(x, y)


def test_compaction_counts_pages_that_it_gives_back():
    """Two slots share a page that the first of them gives back in the call: the second may not write it yet."""
    from paper_2505_11254_amd import binding
    k = torch.arange(4 * PAGE, device="cuda").reshape(4, 1, PAGE, 1).expand(4, 1, PAGE, 64).to(torch.bfloat16).contiguous()
    v = k.clone()
    table, lens, refs = _t([[0, 1, -1], [2, 1, -1]]), _t([100, 100]), _t([1, 2, 1, 0])
    cache = (k, v, table, lens, refs)
    args = (_t([0, 1]), _t([10, 70]), _t([0, 3]), _t([0, 1, 2]))
    assert binding.pages_compact(*cache, *args)[:, 0].tolist() == [1, -1]
    assert refs.tolist() == [1, 1, 1, 0] and lens.tolist() == [11, 100] and table.tolist() == [[0, -1, -1], [2, 1, -1]]
    assert binding.pages_compact(*cache, _t([1]), _t([70]), _t([3]), _t([0, 1]))[0, 0].item() == 1
    assert lens.tolist() == [11, 71] and (k[1, 0, 6] == k[1, 0, 9]).all() and (v[1, 0, 6] == v[1, 0, 9]).all()


def test_outputs_inside_the_cache_are_refused():
    from paper_2505_11254_amd import binding
    c = Case([100], [1], 4, 1, 64, seed=1)
    q, k, v, table, L = c.gpu()
    lists = torch.full((1, 1, 2), -1, dtype=torch.int32, device="cuda")
    for x in (k, v, q):
        out = x.reshape(-1)[:q.numel()].view(q.shape)
        with pytest.raises(ValueError, match="overlap"):
            binding.tree_attn_paged(q, k, v, table, L, out=out, slots=_t(c.slots))
        with pytest.raises(ValueError, match="overlap"):
            binding.selected_attn_paged(q, k, v, table, L, lists, out=out, slots=_t(c.slots))


@pytest.mark.parametrize("lens,news,Hq,Hkv,d", [
    ([9000, 5000], [64, 62], 16, 2, 128),        # two row groups of 256 rows each
    ([9000, 700, 64, 4000], [64, 0, 63, 61], 16, 2, 128),
    ([9000, 5000], [64, 20], 16, 2, 128),        # (one sequence has one group only)
    ([7000, 6500, 6800], [64, 64, 60], 20, 4, 64),  # three of 128
    ([20000], [30], 5, 1, 64),                   # two, on a single kv head
    ([6400] * 3 + [5000] * 67, [34] * 70, 8, 1, 64),
])
def test_row_groups_over_long_contexts(lens, news, Hq, Hkv, d):
    """Sequences whose rows fill several workgroups and whose pages are shared among many."""
    from paper_2505_11254_amd import binding
    c = Case(lens, news, Hq, Hkv, d, seed=len(lens))
    q, k, v, table, L = c.gpu()
    lse = torch.zeros(q.shape[:2], device="cuda")
    assert binding.paged_workspace_bytes(len(lens), max(news), Hq, Hkv, d, max(lens)) > 0
    out = binding.tree_attn_paged(q, k, v, table, L, lse=lse, max_len=max(lens), **c.kw())
    c.check(out, lse, lambda b, i, g: torch.arange(lens[b]) <= lens[b] - news[b] + i)
    again = binding.tree_attn_paged(q, k, v, table, L, max_len=max(lens), **c.kw())
    assert torch.equal(out, again)
