"""Block selection on the GPU: summaries, lists of key tiles for query blocks and of
pages for single tokens, against the documented definition.  Codes and choices are
whole numbers and scores are rounded in one place, so lists have to be equal; scales
are one rounding of a 64-bit quotient, equal too."""
from __future__ import annotations

import random

import numpy as np
import pytest
import torch

import oracle
from paged_sim import PAGE, choose, pages_of, summary
from sampling import assert_parity, to_oracle_bits
from test_gpu_paged_attn import Case

pytestmark = pytest.mark.gpu


def _t(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


def _cu(lens):
    return np.concatenate([[0], np.cumsum(lens)]).tolist()


def _values(shape, seed, kind):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(shape, generator=g)
    if kind == "offset":
        x = x + torch.randn(shape[1:], generator=g)
    elif kind == "few":  # few different values: ties in codes and scores
        x = torch.randint(-1, 2, shape, generator=g).float()
    elif kind == "zero":
        x = x * 0
    return x.to(torch.bfloat16)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind", ["normal", "offset", "few", "zero"])
def test_key_summary(d, kind):
    from paper_2505_11254_amd import binding
    lens = [0, 63, 64, 700, 129, 1]
    k = _values((sum(lens), 3, d), 1, kind)
    cu = _cu(lens)
    blocks = sum(lens) // PAGE + len(lens)
    codes = torch.full((blocks, 3, d), 99, dtype=torch.int8, device="cuda")
    scales = torch.full((blocks, 3), -5.0, device="cuda")
    binding.key_summary(k.cuda(), cu_seqlens=_t(cu), max_seqlen=max(lens), codes=codes, scales=scales)
    want_c = torch.full((blocks, 3, d), 99, dtype=torch.int64)
    want_s = torch.full((blocks, 3), -5.0)
    for b, n in enumerate(lens):
        for h in range(3):
            c, s = summary(k[cu[b]:cu[b] + n // PAGE * PAGE, h].reshape(-1, PAGE, d))
            at = cu[b] // PAGE + b
            want_c[at:at + n // PAGE, h], want_s[at:at + n // PAGE, h] = c, s
    assert torch.equal(codes.cpu().long(), want_c)
    assert torch.equal(scales.cpu(), want_s)


@pytest.mark.parametrize("d", [64, 128])
def test_page_summary_of_the_pages_that_changed(d):
    from paper_2505_11254_amd import binding
    c = Case([0, 64, 200, 1000, 63], [0] * 5, 2, 2, d, seed=3)
    _, k, _, table, L = c.gpu()
    P = k.shape[0]
    codes = torch.full((P, 2, d), 77, dtype=torch.int8, device="cuda")
    scales = torch.full((P, 2), -1.0, device="cuda")
    want_c, want_s = torch.full((P, 2, d), 77, dtype=torch.int64), torch.full((P, 2), -1.0)

    def check(first, pages):
        binding.page_summary(k, table, L, codes, scales, slots=_t(c.slots), **first)
        for b, n in enumerate(c.lens):
            for j in range(n // PAGE):
                if j in pages(b):
                    p = int(c.table[c.slots[b], j])
                    x, s = summary(c.k[p])
                    want_c[p], want_s[p] = x, s
        assert torch.equal(codes.cpu().long(), want_c)
        assert torch.equal(scales.cpu(), want_s)

    check(dict(first=_t([0, 0, 70, 900, 0]), max_new=100), lambda b: {2: [1, 2], 3: [14, 15], 1: [0], 0: [], 4: []}[b])
    check({}, lambda b: range(99))


@pytest.mark.parametrize("Hq,Hkv,d,bq", [(8, 2, 64, 64), (32, 8, 128, 64), (8, 2, 128, 256), (7, 1, 64, 256),
                                         (64, 1, 64, 64), (16, 2, 128, 128), (2, 2, 128, 256)])
@pytest.mark.parametrize("kind", ["offset", "few"])
def test_select_blocks(Hq, Hkv, d, bq, kind):
    """Packed batches with empty and odd lengths; every list, and the marks where there is none."""
    from paper_2505_11254_amd import binding
    lens = [700, 0, 1, 2500, 64]
    cu, N = _cu(lens), max(lens)
    q, k = _values((sum(lens), Hq, d), 5, "normal" if kind == "offset" else kind), _values((sum(lens), Hkv, d), 6, kind)
    for top_k, sink, recent in ((1, 0, 0), (6, 1, 2), (40, 0, 3)):
        codes, scales = binding.key_summary(k.cuda(), cu_seqlens=_t(cu), max_seqlen=N)
        ptr, idx = binding.select_blocks(q.cuda(), codes, scales, top_k=top_k, block_q=bq, n_sink=sink, n_recent=recent,
                                         cu_seqlens=_t(cu), max_seqlen=N)
        ptr, idx = ptr.cpu(), idx.cpu().tolist()
        R, nqb = bq // PAGE, -(-N // bq)
        total = sum(min(top_k, j * R) for j in range(nqb))
        G, used = Hq // Hkv, set()
        for b, n in enumerate(lens):
            for g in range(Hkv):
                c, s = summary(k[cu[b]:cu[b] + n // PAGE * PAGE, g].reshape(-1, PAGE, d))
                at = (b * Hkv + g) * total
                assert int(ptr[b, g, 0]) == at
                for j in range(nqb):
                    rows = q[cu[b] + j * bq:cu[b] + min(n, (j + 1) * bq), g * G:(g + 1) * G].reshape(-1, d)
                    want = choose(rows, c[:j * R], s[:j * R], top_k, sink, recent) if j * bq < n else []
                    assert idx[int(ptr[b, g, j]):int(ptr[b, g, j + 1])] == want, (b, g, j)
                    used.update(range(at, at + len(want)))
                    at += len(want)
                assert at == int(ptr[b, g, nqb])
        assert all(x == -1 for i, x in enumerate(idx) if i not in used and i < B_entries(len(lens), Hkv, total))
        if total:
            assert binding.check_inputs(max_seqlen=N, cu_seqlens=_t(cu), Hkv=Hkv, block_q=bq, block_ptr=ptr.cuda(),
                                        block_idx=torch.tensor(idx, dtype=torch.int32).cuda()) == 0


def B_entries(B, Hkv, total):
    return B * Hkv * total


@pytest.mark.parametrize("Hq,Hkv,d,top_k", [(8, 2, 64, 4), (32, 8, 128, 16), (28, 4, 128, 1), (64, 1, 64, 7),
                                            (16, 16, 128, 33)])
@pytest.mark.parametrize("few", [False, True])
def test_select_pages(Hq, Hkv, d, top_k, few):
    from paper_2505_11254_amd import binding
    lens, news = [1, 64, 65, 700, 3000, 2048, 0, 9000], [1, 1, 2, 3, 1, 4, 0, 2]
    c = Case(lens, news, Hq, Hkv, d, seed=top_k)
    if few:
        whole = torch.isfinite(c.k)
        c.k = torch.where(whole, (c.k.nan_to_num(0.0) * 2).round().clamp(-1, 1), c.k)
        c.q = c.q.round().clamp(-1, 1)
    q, k, _, table, L = c.gpu()
    codes = torch.zeros((k.shape[0], Hkv, d), dtype=torch.int8, device="cuda")
    scales = torch.zeros((k.shape[0], Hkv), device="cuda")
    kw = c.kw()
    binding.page_summary(k, table, L, codes, scales, slots=kw["slots"])
    sink, recent = (1, 2) if top_k > 3 else (0, 0)
    got = binding.select_pages(q, codes, scales, table, L, top_k=top_k, n_sink=sink, n_recent=recent, **kw).cpu()
    G = Hq // Hkv
    for b, n in enumerate(lens):
        for g in range(Hkv):
            x, s = summary(c.keys(b, g)[0][:n // PAGE * PAGE].reshape(-1, PAGE, d))
            for i in range(news[b]):
                own = (n - news[b] + i) // PAGE
                want = choose(c.q[c.cu[b] + i, g * G:(g + 1) * G], x[:own], s[:own], top_k, sink, recent)
                assert got[c.cu[b] + i, g].tolist() == want + [-1] * (top_k - len(want)), (b, g, i)


@pytest.mark.parametrize("bits", [0x3FFE, 0x3F80, 0x3FFF, 0x4055, 0x0100, 0x7F7E, 0x7F7F, 0x0002, 0x8000, 0xC07E])
def test_query_codes_on_every_border(bits):
    """Token t's row holds a largest value in channel 0 and in channel 1 the t-th of all bf16 magnitudes
    from there down by ten octaves, with either sign: ties among them, many where the largest has the
    significand 254.  Of its two pages the first scores c times the code of channel 0, the second 127
    times that of channel 1, so the choice for c around the expected code tells it."""
    from paper_2505_11254_amd import binding
    top = torch.tensor([bits], dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    most = bits & 0x7FFF
    rows = torch.arange(max(0, most - 1400), most + 1).to(torch.int16).view(torch.bfloat16)
    T = len(rows)
    rows = torch.where(torch.arange(T) % 2 == 0, rows, -rows)
    q = torch.zeros((T, 1, 64), dtype=torch.bfloat16)
    q[:, 0, 0], q[:, 0, 1] = top, rows
    a = top.double().abs()
    code = (torch.round(q[:, 0, :2].double() * 127 / a) if float(a) else q[:, 0, :2].double() * 0).long()
    table = torch.arange(3 * T, dtype=torch.int32).view(T, 3)
    L = torch.full((T,), 2 * PAGE + 1, dtype=torch.int32)
    for off in (-1, 0, 1):
        c = (code[:, 1] * code[:, 0].sign() + off).clamp(-127, 127)
        pages = torch.zeros((T, 3, 1, 64), dtype=torch.int8)
        pages[:, 0, 0, 0], pages[:, 1, 0, 1] = c.to(torch.int8), 127
        got = binding.select_pages(q.cuda(), pages.view(3 * T, 1, 64).cuda(), torch.ones((3 * T, 1)).cuda(), table.cuda(),
                                   L.cuda(), top_k=1, n_sink=0, n_recent=0, B=T).cpu()[:, 0, 0]
        want = (c * code[:, 0] < 127 * code[:, 1]).long()  # (ties go to the first)
        assert torch.equal(got.long(), want), off


@pytest.mark.parametrize("n_pages,top_k", [(3000, 128), (20000, 64), (2049, 2048)])
def test_select_pages_of_long_sequences(n_pages, top_k):
    """Far more candidates than one stripe of the selection, with codes drawn at random, so that no keys are
    needed: whole numbers throughout."""
    from paper_2505_11254_amd import binding
    g = torch.Generator().manual_seed(n_pages)
    P = n_pages + 5
    codes = torch.randint(-127, 128, (P, 1, 64), generator=g).to(torch.int8)
    scales = torch.rand((P, 1), generator=g).bfloat16().float()  # (coarse: ties)
    codes[::3] = codes[0]
    scales[::3] = scales[0]
    table = torch.randperm(P, generator=g)[:n_pages].to(torch.int32)[None]
    table[0, 17] = -1  # a page that is missing comes last
    L = torch.tensor([n_pages * PAGE - 3], dtype=torch.int32)
    q = torch.randn((1, 3, 64), generator=g).to(torch.bfloat16)
    got = binding.select_pages(q.cuda(), codes.cuda(), scales.cuda(), table.cuda(), L.cuda(), top_k=top_k)[0, 0].tolist()
    own = n_pages - 1
    t = table[0, :own].long().clamp(min=0)
    x, s = codes[t, 0].long(), scales[t, 0].clone()
    x[17], s[17] = 0, 0
    a = q.double().abs().max()
    best = (torch.round(q[0].double() * 127 / a) @ x.double().T).max(0).values
    score = (best * s.double()).float()
    score[17] = float("-inf")
    score[0] = score[own - 1] = float("inf")
    want = sorted(torch.sort(score, descending=True, stable=True).indices[:top_k].tolist())
    assert got == want


def test_prompt_then_decode_end_to_end():
    """A run as a serving program makes it: summaries and lists of a prompt, Delta Attention over them, the
    prompt's keys into the cache, a fork, then steps of sparse and tree decoding on both branches."""
    from paper_2505_11254_amd import binding
    Hq, Hkv, d, N, gamma = 8, 2, 128, 1500, 64
    q, k, v = (_values((N, h, d), i, "normal") for i, h in ((1, Hq), (2, Hkv), (3, Hkv)))
    qc, kc, vc = q.cuda(), k.cuda(), v.cuda()
    codes, scales = binding.key_summary(kc)
    ptr, idx = binding.select_blocks(qc, codes, scales, top_k=6, block_q=64)
    out = binding.delta_attn_prefill_blocksparse(qc, kc, vc, block_q=64, block_ptr=ptr, block_idx=idx, gamma=gamma)
    bits = [to_oracle_bits(x) for x in (q, k, v)]
    want = oracle.block_delta_attention(*bits, None, block_q=64, blk_ptr=ptr.cpu().numpy(),
                                        blk_idx=idx.cpu().numpy(), gamma=gamma)
    assert_parity(out, want, "Delta over selected blocks")

    S, M, P = 4, 40, 60
    kp = torch.full((P, Hkv, PAGE, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    vp = kp.clone()
    table, lens = torch.full((S, M), -1, dtype=torch.int32, device="cuda"), torch.zeros(S, dtype=torch.int32, device="cuda")
    refs = torch.zeros(P, dtype=torch.int32, device="cuda")
    pc, ps = torch.zeros((P, Hkv, d), dtype=torch.int8, device="cuda"), torch.zeros((P, Hkv), device="cuda")
    cache = (kp, vp, table, lens, refs)
    assert binding.pages_resize(*cache, _t([2]), _t([N]))[0, 0].item() == N
    binding.pages_append(kc, vc, kp, vp, table, lens, slots=_t([2]))
    binding.page_summary(kp, table, lens, pc, ps, slots=_t([2]))
    assert binding.pages_fork(table, lens, refs, _t([2]), _t([0])).tolist() == [N]
    hist = {2: (k, v), 0: (k, v)}
    r = random.Random(3)
    for step in range(4):
        m = r.choice([1, 2, 70])
        slots = [0, 2]
        L0 = [hist[s][0].shape[0] for s in slots]
        assert binding.pages_resize(*cache, _t(slots), _t([n + m for n in L0]))[:, 0].tolist() == [n + m for n in L0]
        nq, nk, nv = (_values((2 * m, h, d), 10 * step + i, "normal") for i, h in ((4, Hq), (5, Hkv), (6, Hkv)))
        binding.pages_append(nk.cuda(), nv.cuda(), kp, vp, table, lens, slots=_t(slots), B=2)
        for i, s in enumerate(slots):
            hist[s] = tuple(torch.cat([a, b[i * m:(i + 1) * m]]) for a, b in zip(hist[s], (nk, nv)))
        binding.page_summary(kp, table, lens, pc, ps, slots=_t(slots), first=_t(L0), max_new=m)
        dense = binding.tree_attn_paged(nq.cuda(), kp, vp, table, lens, slots=_t(slots), B=2)
        pages = binding.select_pages(nq.cuda(), pc, ps, table, lens, top_k=5, slots=_t(slots), B=2)
        some = binding.selected_attn_paged(nq.cuda(), kp, vp, table, lens, pages, slots=_t(slots), B=2)
        for i, s in enumerate(slots):
            c = Case([L0[i] + m], [m], Hq, Hkv, d, seed=0)
            c.q = nq[i * m:(i + 1) * m]
            hk, hv = hist[s]
            c.keys = lambda b, g: (hk[:, g], hv[:, g])
            n = L0[i] + m
            c.check(dense[i * m:(i + 1) * m], None, lambda b, j, g: torch.arange(n) <= n - m + j)
            for g in range(Hkv):
                x, sc = summary(hk[:n // PAGE * PAGE, g].reshape(-1, PAGE, d))
                for j in range(m):
                    own = (n - m + j) // PAGE
                    want = choose(c.q[j, g * 4:(g + 1) * 4], x[:own], sc[:own], 5, 1, 1)
                    assert [y for y in pages[i * m + j, g].tolist() if y >= 0] == want
            listed = pages.cpu()

            def visible(b, j, g):
                at = torch.arange(n)
                own = (n - m + j) // PAGE
                return (torch.isin(at // PAGE, listed[i * m + j, g]) | (at // PAGE == own)) & (at <= n - m + j)
            c.check(some[i * m:(i + 1) * m], None, visible)
        # the last rows of each branch but one are rejected
        keep = list(range(m - 1)) if m > 1 else [0]
        start = [n for n in L0]
        got = binding.pages_compact(*cache, _t(slots), _t(start), _t(keep * 2), _t([0, len(keep), 2 * len(keep)]))
        assert got[:, 0].tolist() == [len(keep)] * 2
        for i, s in enumerate(slots):
            hist[s] = tuple(x[:L0[i] + len(keep)] for x in hist[s])
    binding.pages_resize(*cache, _t([0, 2]))
    assert int(refs.sum()) == 0 and (table == -1).all() and int(lens.sum()) == 0


@pytest.mark.parametrize("block_q", [64, 128, 256])
@pytest.mark.parametrize("top_k", [200, 2 ** 31 - 2, 2 ** 31 - 1])
def test_more_blocks_than_there_are(block_q, top_k):
    """top_k past all candidates, the largest integer too: every tile before a query block, in a
    ragged batch."""
    from paper_2505_11254_amd import binding
    cu, Hq, Hkv, d = [0, 1000, 1000, 1064, 3000], 4, 2, 64
    g = torch.Generator().manual_seed(block_q)
    q = torch.randn((cu[-1], Hq, d), generator=g).to(torch.bfloat16).cuda()
    k = torch.randn((cu[-1], Hkv, d), generator=g).to(torch.bfloat16).cuda()
    kw = dict(cu_seqlens=torch.tensor(cu, dtype=torch.int32).cuda(), max_seqlen=1936)
    ptr, idx = binding.select_blocks(q, *binding.key_summary(k, **kw), top_k=top_k, block_q=block_q, **kw)
    ptr, idx, R = ptr.tolist(), idx.tolist(), block_q // 64
    for b in range(4):
        n_qb = -(-(cu[b + 1] - cu[b]) // block_q)
        for h in range(Hkv):
            for j in range(n_qb):
                assert idx[ptr[b][h][j]:ptr[b][h][j + 1]] == list(range(min(top_k, j * R)))


@pytest.mark.parametrize("lens,block_q", [([1], 64), ([64], 64), ([200, 256, 0, 13], 256)])
def test_prompts_within_one_query_block(lens, block_q):
    """No lists at all: block_idx holds nothing but -1, on another stream too, and the attention over it is
    each block's own tiles."""
    from paper_2505_11254_amd import binding
    g = torch.Generator().manual_seed(block_q)
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    q, k, v = (torch.randn((cu[-1], h, 64), generator=g).to(torch.bfloat16).cuda() for h in (8, 2, 2))
    kw = dict(cu_seqlens=torch.tensor(cu, dtype=torch.int32).cuda(), max_seqlen=max(lens))
    sums = binding.key_summary(k, **kw)
    torch.full((1000,), 7, dtype=torch.int32, device="cuda")  # (freed memory that is not -1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (None, side):
        ptr, idx = binding.select_blocks(q, *sums, top_k=4, block_q=block_q, stream=stream, **kw)
        side.synchronize()
        assert idx.tolist() == [-1] and not ptr.any()
    out = binding.blocksparse_attn_prefill(q, k, v, block_q=block_q, block_ptr=ptr, block_idx=idx, **kw)
    dense = binding.dense_causal_attn_prefill(q, k, v, **kw)
    assert (out.float() - dense.float()).abs().max() <= 2 ** -6 * v.abs().max()


def test_selection_finds_the_blocks_that_queries_look_for():
    """Blocks whose keys share a direction, and queries along one of them each: that block is chosen in
    every query block and for every decoded token, and with it the softmax keeps its mass.  Directions
    are orthogonal: a query's score of its own block is |q| 3, of another |q| times what the noise of 64
    keys leaves of its mean, 0.5 / 8 a channel."""
    from paper_2505_11254_amd import binding
    g = torch.Generator().manual_seed(3)
    n, Hq, Hkv, d, top_k = 64, 8, 2, 128, 4
    T, G = n * 64, Hq // Hkv
    dirs = torch.linalg.qr(torch.randn((Hkv, d, d), generator=g, dtype=torch.float64))[0].transpose(1, 2)[:, :n]
    k = 3 * dirs.transpose(0, 1).repeat_interleave(64, 0) + 0.5 * torch.randn((T, Hkv, d), generator=g)
    want = torch.tensor([[int(torch.randint(0, max(j, 1), (1,), generator=g)) for _ in range(Hkv)] for j in range(n)])
    aim = torch.stack([dirs[h, want[:, h]] for h in range(Hkv)], 1).repeat_interleave(64, 0)  # [T, Hkv, d]
    size = 16 + 16 * torch.rand((T, Hq, 1), generator=g)  # (rows of other norms)
    q = size * aim.repeat_interleave(G, 1) + 0.5 * torch.randn((T, Hq, d), generator=g)
    q, k = q.to(torch.bfloat16), k.to(torch.bfloat16)
    ptr, idx = binding.select_blocks(q.cuda(), *binding.key_summary(k.cuda()), top_k=top_k, block_q=64)
    ptr, idx = ptr.tolist(), idx.tolist()
    for h in range(Hkv):
        for j in range(n):
            mine = idx[ptr[0][h][j]:ptr[0][h][j + 1]]
            assert j == 0 or int(want[j, h]) in mine
            if j == n - 1:
                a = q[j * 64:(j + 1) * 64, h * G:(h + 1) * G].double().reshape(-1, d) @ k[:j * 64, h].double().T / d ** 0.5
                mass = torch.softmax(a, 1).reshape(len(a), j, 64).sum(2)
                best = mass.sort(1, descending=True).values[:, :top_k].sum(1)
                assert (mass[:, mine].sum(1) >= 0.95 * best).all()
    # decoding: tokens of their own, each with its own block to find
    kp = k.reshape(n, 64, Hkv, d).transpose(1, 2).contiguous().cuda()
    table, lens = torch.arange(n, dtype=torch.int32).reshape(1, n).cuda(), torch.tensor([T], dtype=torch.int32).cuda()
    codes, scales = torch.zeros((n, Hkv, d), dtype=torch.int8, device="cuda"), torch.zeros((n, Hkv), device="cuda")
    binding.page_summary(kp, table, lens, codes, scales)
    pages = binding.select_pages(q[::64][-32:].contiguous().cuda(), codes, scales, table, lens, top_k=top_k).tolist()
    for i, j in enumerate(range(n - 32, n)):
        for h in range(Hkv):
            assert int(want[j, h]) in pages[i][h]
