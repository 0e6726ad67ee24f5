"""The 8-bit cache, and attention whose scores are capped or biased by distance.

Each case is one pass of a serving program through one of these operators:

  write    new tokens go into the cache as 8-bit codes, and the pages they touch are read back
  read     cached sequences are read back as rows of bf16
  attend   attention of new tokens (single ones, trees of drafts, causal chunks) over the 8-bit cache
  pick     attention of single tokens over selected pages of the 8-bit cache
  prefill  attention of prompts, dense (with a prefix that every row sees, or without) or corrected
           sparse, under capped or biased scores
  decode   attention of new tokens over the bf16 cache under capped or biased scores

An 8-bit cache is pages of 64 tokens [P, Hkv, 64, d] of e4m3 codes (with a leading axis of layers where a
call takes all layers at once) and for keys and values a power of two for each page and kv head,
[P, Hkv] in fp32: a value is its code times that. ``run`` computes the plain form with torch
operations, or calls the library's operators.
"""
from __future__ import annotations

import random

import torch

own = False

PAGE = 64
DEV = "cuda" if torch.cuda.is_available() else "cpu"
LEAST, MOST = -110, 119  # exponents of the scales


def _binding():
    from paper_2505_11254_amd import binding  # (the plain forms run without the library)
    return binding


# ------------------------------------------------------------------------------------- the cases

def listed():
    llama = dict(Hq=32, Hkv=8, d=128)
    return [
        # One new token of one short conversation, in a small model: the smallest call.
        dict(name="write_1", kind="write", layers=1, B=1, len=333, n=1, Hkv=2, d=64),
        # One step of speculative decoding of a batch, 16 drafts each, four layers at a time.
        dict(name="write_64x16", kind="write", layers=4, B=64, len=2000, n=16, Hkv=8, d=128),
        # The keys and values of a packed batch of prompts after their prefill.
        dict(name="write_87k", kind="write", layers=1, B=5, len=24011, n=24011, Hkv=8, d=128),
        # One cached conversation is read back in front of its next chunk.
        dict(name="read_1", kind="read", layers=1, B=1, len=3001, Hkv=8, d=128),
        # A whole ragged batch is read back.
        dict(name="read_64", kind="read", layers=1, B=64, len=8192, Hkv=8, d=128),
        # A single token of a single short sequence.
        dict(name="attend_1", kind="attend", B=1, n=1, len=777, tree=False, cap=0.0, biased=False, Hq=8, Hkv=2, d=64),
        # Everyday decoding of a ragged batch in an 8B-shaped layer.
        dict(name="attend_64", kind="attend", B=64, n=1, len=8192, tree=False, cap=0.0, biased=False, **llama),
        # Eight drafts after a long prompt, in a model that caps its scores.
        dict(name="attend_131k", kind="attend", B=1, n=8, len=131072, tree=True, cap=30.0, biased=False, **llama),
        # Two prompts of no round length in a model that caps its scores.
        dict(name="capped_2k", kind="prefill", mode="dense", B=2, len=2011, cap=30.0, biased=False, prefix=0, **llama),
        # Packed prompts that see their instructions whole, in a model that biases scores by distance.
        dict(name="prefix_8k", kind="prefill", mode="dense", B=3, len=8100, cap=0.0, biased=True, prefix=900, Hq=16,
             Hkv=16, d=128),
        # A long prompt by corrected sparse attention, scores capped.
        dict(name="delta_32k", kind="prefill", mode="delta", B=1, len=32768, cap=30.0, biased=False, prefix=0, window=2048,
             n_sink=64, gamma=64, **llama),
        # Decoding of a batch, scores biased by distance.
        dict(name="decode_32", kind="decode", B=32, n=1, len=6000, tree=False, cap=0.0, biased=True, **llama),
    ]


def draw(rng):
    def log(lo, hi):
        return min(hi, int(lo * (hi / lo) ** rng.random() + 0.5))

    Hq, Hkv, d = rng.choice([(32, 8, 128), (8, 2, 64), (16, 16, 128), (28, 4, 128), (64, 8, 128), (16, 2, 64),
                             (20, 4, 64), (12, 3, 128)])
    kind = rng.choice(["write", "write", "read", "attend", "attend", "pick", "prefill", "prefill", "decode"])
    heads = dict(Hq=Hq, Hkv=Hkv, d=d)
    if kind == "write":
        if rng.random() < 0.5:
            return dict(kind=kind, layers=log(1, 4), B=log(1, 64), len=log(1, 2000), n=log(1, 64), Hkv=rng.randint(1, 8), d=d)
        n = log(50, 24000)
        return dict(kind=kind, layers=1, B=log(1, 5), len=n, n=n, Hkv=rng.randint(1, 8), d=d)
    if kind == "read":
        B = log(1, 64)
        return dict(kind=kind, layers=rng.choice([1, 1, 2]), B=B, len=log(1, min(100000, 250000 // B)), Hkv=rng.randint(1, 8),
                    d=d)
    biased = rng.random() < 0.4
    cap = rng.choice([0.0, 15.0, 50.0]) if kind == "attend" or biased else rng.choice([15.0, 30.0, 50.0])
    if kind in ("attend", "decode"):
        tree = not biased and rng.random() < 0.5
        n = log(2, 64) if tree else rng.choice([1, 1, 1, log(2, 40)])
        B = log(1, 48)
        return dict(kind=kind, B=B, n=n, len=log(n, max(n + 1, min(100000, 500000 // (B * n) + 200))), tree=tree, cap=cap,
                    biased=biased, **heads)
    if kind == "pick":
        B = log(1, 32)
        return dict(kind=kind, B=B, n=rng.choice([1, 1, 3]), len=log(100, 400000 // B), top_k=log(4, 96), **heads)
    mode = rng.choice(["dense", "delta"])
    prefix = log(1, 1500) if mode == "dense" and rng.random() < 0.5 else 0
    more = dict(window=log(64, 2048), n_sink=rng.randint(0, 70), gamma=rng.choice([16, 48, 64, 128])) if mode == "delta" else {}
    return dict(kind=kind, mode=mode, B=rng.choice([1, 1, 2, 3]), len=log(60, 8100), cap=cap, biased=biased, prefix=prefix,
                **more, **heads)


def _lens(case):
    """The sequences' lengths: the first has `len`, the others between a quarter of it and all of it."""
    return [max(1, int(case["len"] * (1.0 if b == 0 else 0.25 + 0.75 * (b * 0.618034 % 1.0)))) for b in range(case["B"])]


def _news(case):
    """New tokens of each sequence: all of them, or `n` for the first and at least one for each."""
    if case["n"] == case["len"]:
        return _lens(case)
    return [min(L, max(1, case["n"] - (3 * b) % max(1, case["n"] // 2))) for b, L in enumerate(_lens(case))]


def _pages(n):
    return -(-n // PAGE)


def _touched(case):
    """Where the pages that a write touches begin, sequence by sequence."""
    return [(L - m) // PAGE * PAGE for L, m in zip(_lens(case), _news(case))]


def _visible(case, n):
    """(pairs of a dense causal row set with the case's prefix, pairs of the sparse rows, of the dense rows)."""
    p = min(case["prefix"], n)
    dense = n * (n + 1) // 2 + p * (p - 1) // 2
    if case["mode"] == "dense":
        return dense, 0, 0
    w, s, g = case["window"], case["n_sink"], case["gamma"]
    full = w + s
    sparse = n * (n + 1) // 2 if n <= full else full * (full + 1) // 2 + (n - full) * full
    rows = list(range(0, n // g * g, g)) + list(range(n // g * g, n))
    return dense, sparse, sum(i + 1 for i in rows)


def work(case):
    """What a pass cannot do without: inputs read once, outputs written once."""
    kind, d, Hkv = case["kind"], case["d"], case["Hkv"]
    row = 2 * Hkv * d  # the key and the value of a token, a byte each
    lens = _lens(case)
    if kind == "write":
        new = sum(_news(case)) * case["layers"]
        back = sum(L - t for L, t in zip(lens, _touched(case))) * case["layers"]
        return {"bytes": new * row * 3 + back * row * 3 + len(lens) * 8, "flops": 0}
    if kind == "read":
        return {"bytes": sum(lens) * row * 3 * case["layers"], "flops": 0}
    Hq = case["Hq"]
    if kind in ("attend", "decode"):
        news = _news(case)
        size = row * (1 if kind == "attend" else 2)
        pairs = sum(n * m for n, m in zip(lens, news))
        return {"bytes": sum(lens) * size + 2 * sum(news) * Hq * d * 2, "flops": 4 * pairs * Hq * d}
    if kind == "pick":
        b = f = 0
        for n, m in zip(lens, _news(case)):
            keys = min(case["top_k"], n // PAGE) * PAGE + n % PAGE
            b += m * keys * row + 2 * m * Hq * d * 2
            f += 4 * m * keys * Hq * d
        return {"bytes": b, "flops": f}
    b = f = 0
    for n in lens:
        dense, sparse, strided = _visible(case, n)
        b += 2 * n * Hq * d * 2 + 2 * n * row
        f += 4 * (dense if case["mode"] == "dense" else sparse + strided) * Hq * d
    return {"bytes": b, "flops": f}


# ------------------------------------------------------------------------------- what is in hand

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _randn(g, *shape, std=1.0, offset=None):
    """Normal bf16 values; `offset` shifts keys as trained models do."""
    out = torch.empty(shape, dtype=torch.bfloat16, device=DEV)
    flat = out.view(shape[0], -1)
    step = max(1, (1 << 27) // max(1, flat.shape[1]))
    for i in range(0, shape[0], step):
        x = torch.randn((min(step, shape[0] - i),) + tuple(shape[1:]), generator=g, device=DEV) * std
        out[i:i + step] = x if offset is None else x + offset
    return out


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _cu(v):
    cu = [0]
    for n in v:
        cu.append(cu[-1] + n)
    return _ints(cu)


def _cache(g, layers, Hkv, d, lens, spare, eight):
    """A cache that holds sequences of these lengths, in pages scattered over the pool."""
    M = _pages(max(lens)) + 1
    P = sum(map(_pages, lens)) + spare
    off = torch.randn((Hkv, 1, d), generator=g, device=DEV) * 0.5
    perm = torch.randperm(P, generator=g, device=DEV).to(torch.int32)
    table = torch.full((len(lens), M), -1, dtype=torch.int32, device=DEV)
    at = 0
    for i, n in enumerate(lens):
        table[i, :_pages(n)] = perm[at:at + _pages(n)]
        at += _pages(n)
    lead = () if layers == 1 else (layers,)
    s = dict(table=table, lens=_ints(lens))
    for name, o in (("k", off), ("v", None)):
        pages = _randn(g, layers * P, Hkv, PAGE, d, offset=o)
        if eight:  # as an earlier pass has left them
            codes = torch.empty(pages.shape, dtype=torch.float8_e4m3fn, device=DEV)
            scales = torch.empty(pages.shape[:2], device=DEV)
            for i in range(0, len(pages), 2048):
                e = _exponent(pages[i:i + 2048].abs().amax((-1, -2)).float())
                scales[i:i + 2048] = _pow2(e)
                codes.view(torch.uint8)[i:i + 2048] = _code(pages[i:i + 2048], e[..., None, None]).view(torch.uint8)
            pages = codes
            s[name + "_scales"] = scales.view(lead + (P, Hkv))
        s[name + "_pages"] = pages.view(lead + (P, Hkv, PAGE, d))
    return s


def _parents(r, n):
    """A draft tree in the order its nodes are drafted: the parent of each node, -1 under the context."""
    return [r.randint(max(-1, i - 1 - r.randint(0, 5)), i - 1) for i in range(n)]


def _tree_masks(parents_of, words):
    """Bit j of row i: draft j is i or an ancestor of it."""
    rows = []
    for parents in parents_of:
        bits = []
        for i, p in enumerate(parents):
            bits.append((bits[p] if p >= 0 else 0) | 1 << i)
        for x in bits:
            w = [x >> 64 * k & (1 << 64) - 1 for k in range(words)]
            rows.append([v - (1 << 64) if v >> 63 else v for v in w])
    return torch.tensor(rows, dtype=torch.int64, device=DEV)


def _slopes(Hq):
    """A slope for each head, from 2^(-8 / Hq) down to 2^-8."""
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / Hq) for h in range(Hq)], device=DEV)


def prepare(case, seed):
    g, r = _gen(seed), random.Random(seed)
    kind, Hkv, d = case["kind"], case["Hkv"], case["d"]
    lens = _lens(case)
    s = dict(case=case)
    if kind in ("write", "read"):
        s.update(_cache(g, case["layers"], Hkv, d, lens, 3, True))
    if kind == "write":
        news, first = _news(case), _touched(case)
        lead = () if case["layers"] == 1 else (case["layers"],)
        shape = lead + (sum(news), Hkv, d)
        off = torch.randn((Hkv, d), generator=g, device=DEV) * 0.5
        order = list(range(len(lens)))
        r.shuffle(order)  # the batch takes the slots in no order
        s.update(k=_randn(g, *shape, std=1.3, offset=off), v=_randn(g, *shape, std=1.3), slots=_ints(order),
                 cu=_cu([news[i] for i in order]), max_new=max(news), first=_ints([first[i] for i in order]),
                 back=_cu([lens[i] - first[i] for i in order]), max_back=max(a - b for a, b in zip(lens, first)),
                 n_back=sum(lens) - sum(first))
    elif kind == "read":
        s.update(cu=_cu(lens), n=sum(lens), max_len=max(lens))
    elif kind in ("attend", "decode", "pick"):
        news = _news(case)
        s.update(_cache(g, 1, Hkv, d, lens, 5, kind != "decode"))
        std = 3.0 if kind != "pick" and (case["cap"] or case["biased"]) else 1.0
        s.update(q=_randn(g, sum(news), case["Hq"], d, std=std), cu=_cu(news), max_q=max(news), max_len=max(lens), mask=None)
        if kind != "pick":
            if case["tree"]:
                s["mask"] = _tree_masks([_parents(r, n) for n in news], -(-max(news) // 64))
            s["slopes"] = _slopes(case["Hq"]) if case["biased"] else None
        else:
            top_k = case["top_k"]
            lists = torch.full((sum(news), Hkv, top_k), -1, dtype=torch.int32)
            t = 0
            for n, m in zip(lens, news):
                for i in range(m):
                    own_page = (n - m + i) // PAGE
                    for h in range(Hkv):
                        at = sorted(r.sample(range(own_page), min(top_k, own_page)))
                        lists[t, h, :len(at)] = torch.tensor(at, dtype=torch.int32)
                    t += 1
            s["lists"] = lists.to(DEV)
    else:
        off = torch.randn((Hkv, d), generator=g, device=DEV) * 0.5
        T = sum(lens)
        s.update(q=_randn(g, T, case["Hq"], d, std=3.0), k=_randn(g, T, Hkv, d, offset=off), v=_randn(g, T, Hkv, d),
                 cu=_cu(lens), max_len=max(lens), slopes=_slopes(case["Hq"]) if case["biased"] else None, prefix=None)
        if case["prefix"]:
            s["prefix"] = _ints([min(n, r.randint(0, case["prefix"])) if b else min(n, case["prefix"])
                                 for b, n in enumerate(lens)])
    return s


# -------------------------------------------------------------------------------- the plain forms

def _exponent(top):
    """The least exponent whose scale brings magnitudes up to `top` within e4m3's 448."""
    m, x = torch.frexp(top)
    return torch.where(top > 0, x - 9 + (m > 0.875).to(x.dtype), LEAST).clamp(LEAST, MOST)


def _pow2(e):
    return (e + 127 << 23).to(torch.int32).view(torch.float32)


def _code(x, e):
    """The e4m3 codes nearest to x / 2^e."""
    return (x.float() * _pow2(-e)).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _layered(s, *names):
    """Views with an axis of layers."""
    one = s["case"]["layers"] == 1
    return [s[x][None] if one else s[x] for x in names]


def _rows_of(cu, n):
    """The sequence of each of n packed rows, and its place in it."""
    cu = cu.long()
    t = torch.arange(n, device=DEV)
    b = torch.searchsorted(cu[1:], t, right=True)
    return b, t - cu[b]


def _plain_write(s):
    """The new tokens become the last ones of their sequences. A page's scale covers its tokens: where it grows,
    those it held before are recoded."""
    sl, table = s["slots"].long(), s["table"].long()
    b, i = _rows_of(s["cu"], s["k"].shape[-3])
    start = (s["lens"].long()[sl] - (s["cu"][1:] - s["cu"][:-1]).long())
    pos = start[b] + i
    page = table[sl[b], pos // PAGE]
    # pages that held tokens before: at most one of a sequence, its first
    part = start % PAGE > 0
    first = torch.where(part, table[sl, (start // PAGE).clamp(max=table.shape[1] - 1)], 0)
    below = part[:, None] & (torch.arange(PAGE, device=DEV) < (start % PAGE)[:, None])
    for name in ("k", "v"):
        pages, scales, new = _layered(s, name + "_pages", name + "_scales", name)
        raw = pages.view(torch.uint8)
        for layer in range(pages.shape[0]):
            x = new[layer].float()
            top = x.abs().amax(-1)  # [T, Hkv]
            most = torch.zeros_like(scales[layer]).scatter_reduce_(0, page[:, None].expand_as(top), top, "amax")
            need = _exponent(most)
            old = torch.frexp(scales[layer])[1] - 1
            keep = torch.zeros(scales.shape[1], dtype=torch.bool, device=DEV)
            keep[first] |= part
            fresh = torch.where(keep[:, None], torch.maximum(old, need), need)
            written = torch.zeros(scales.shape[1], dtype=torch.bool, device=DEV)
            written[page] = True
            e = torch.where(written[:, None], fresh, old)
            was = pages[layer][first].float()
            again = _code(was * _pow2(old[first])[..., None, None], e[first][..., None, None]).view(torch.uint8)
            raw[layer][first] = torch.where(below[:, None, :, None], again, raw[layer][first])
            raw[layer][page, :, pos % PAGE] = _code(x, e[page][..., None]).view(torch.uint8)
            scales[layer] = _pow2(e)


def _plain_read(s, slots, first, cu, n):
    """Rows of the cached tokens from `first` of each sequence on."""
    b, i = _rows_of(cu, n)
    sl = slots.long()[b]
    pos = first.long()[b] + i
    page = s["table"].long()[sl, pos // PAGE]
    out = {}
    for name in ("k", "v"):
        pages, scales = _layered(s, name + "_pages", name + "_scales")
        rows = torch.stack([(raw[page, :, pos % PAGE].view(torch.float8_e4m3fn).float() * sc[page][..., None]).bfloat16()
                            for raw, sc in zip(pages.view(torch.uint8), scales)])
        out[name] = rows[0] if s["case"]["layers"] == 1 else rows
    return out


def _softmax_v(scores, vis, v):
    """softmax over the visible keys of scores [..., rows, keys] times v [..., keys, d]; rows that see none: 0."""
    scores = scores.masked_fill(~vis, float("-inf"))
    top = scores.amax(-1, keepdim=True)
    p = torch.exp(scores - torch.where(top > float("-inf"), top, 0.0))
    p = p.masked_fill(~vis, 0.0)
    return (p @ v) / p.sum(-1, keepdim=True).clamp(min=1e-30)


def _scores(a, case, slopes, dist):
    """Scores a [..., rows, keys] capped, and biased by slopes (broadcast to a) times the distances."""
    if case["cap"]:
        a = torch.tanh(a / case["cap"]) * case["cap"]
    return a if slopes is None else a - slopes * dist


def _gather(s, name, pages):
    """Keys or values [..., Hkv, pages * 64, d] of pages [..., pages] in fp32."""
    x = s[name + "_pages"]
    if x.dtype == torch.bfloat16:
        x = x[pages].float()
    else:
        x = x.view(torch.uint8)[pages].view(torch.float8_e4m3fn).float() * s[name + "_scales"][pages][..., None, None]
    return x.transpose(-4, -3).flatten(-3, -2)


def _plain_attend(s):
    c, q, table, lens, cu = s["case"], s["q"], s["table"].long(), s["lens"].long(), s["cu"].long()
    T, Hq, d = q.shape
    B, Hkv, N = lens.numel(), c["Hkv"], s["max_q"]
    G = Hq // Hkv
    b, i = _rows_of(cu, T)
    new = cu[1:] - cu[:-1]
    qs = torch.zeros((B, N, Hq, d), device=DEV)
    qs[b, i] = q.float()
    qs = qs.view(B, N, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, d)
    k, v = _gather(s, "k", table.clamp(min=0)), _gather(s, "v", table.clamp(min=0))
    pos = torch.arange(k.shape[2], device=DEV)
    j = pos - (lens - new)[:, None]  # place among the new tokens
    if s["mask"] is None:
        vis = j[:, None] <= torch.arange(N, device=DEV)[:, None]
    else:
        bits = torch.zeros((B, N, s["mask"].shape[1]), dtype=torch.int64, device=DEV)
        bits[b, i] = s["mask"]
        jc = j.clamp(min=0, max=64 * bits.shape[2] - 1)[:, None].expand(B, N, -1)
        vis = (torch.gather(bits, 2, jc // 64) >> jc % 64 & 1).bool() | (j < 0)[:, None]
    vis &= (pos < lens[:, None])[:, None]
    vis = vis[:, None, :, None].expand(B, 1, N, G, -1).reshape(B, 1, -1, pos.numel())
    slopes = dist = None
    if s["slopes"] is not None:
        slopes = s["slopes"].view(Hkv, 1, G).expand(Hkv, N, G).reshape(Hkv, -1, 1)
        dist = (torch.arange(N, device=DEV)[:, None] - j[:, None]).abs().float()
        dist = dist[:, None, :, None].expand(B, 1, N, G, -1).reshape(B, 1, -1, pos.numel())
    out = _softmax_v(_scores(qs @ k.transpose(-1, -2) * d ** -0.5, c, slopes, dist), vis, v)
    out = out.view(B, Hkv, N, G, d).permute(0, 2, 1, 3, 4).reshape(B, N, Hq, d)
    return out[b, i].to(q.dtype)


def _plain_pick(s):
    c, q, table = s["case"], s["q"], s["table"].long()
    T, Hq, d = q.shape
    Hkv = c["Hkv"]
    b, i = _rows_of(s["cu"], T)
    pos = s["lens"].long()[b] - (s["cu"][1:] - s["cu"][:-1]).long()[b] + i
    at = torch.cat([s["lists"].long(), (pos // PAGE)[:, None, None].expand(T, Hkv, 1)], -1)
    page = torch.gather(table[b][:, None].expand(T, Hkv, -1), 2, at.clamp(min=0)).clamp(min=0)
    h = torch.arange(Hkv, device=DEV)[:, None]
    k, v = ((s[x + "_pages"].view(torch.uint8)[page, h].view(torch.float8_e4m3fn).float()
             * s[x + "_scales"][page, h][..., None, None]).flatten(2, 3) for x in ("k", "v"))
    keys = (at[..., None] * PAGE + torch.arange(PAGE, device=DEV)).flatten(2, 3)
    vis = (keys >= 0) & (keys <= pos[:, None, None])
    qg = q.view(T, Hkv, Hq // Hkv, d).float()
    return _softmax_v(qg @ k.transpose(-1, -2) * d ** -0.5, vis[:, :, None], v).reshape(T, Hq, d).to(q.dtype)


def _plain_prefill(s):
    c = s["case"]
    Hq, Hkv, d = c["Hq"], c["Hkv"], c["d"]
    G = Hq // Hkv
    slopes = None if s["slopes"] is None else s["slopes"].view(Hkv, G, 1, 1)
    out = torch.empty_like(s["q"])
    base = 0
    for b, n in enumerate(_lens(c)):
        q, k, v = (s[x][base:base + n].float().transpose(0, 1) for x in ("q", "k", "v"))
        q = q.reshape(Hkv, G, n, d)
        prefix = 0 if s["prefix"] is None else s["prefix"][b].long()

        def rows(at, keys, seen):
            """Attention of the rows `at` over the keys `keys` where seen(rows, keys)."""
            i, j = at[:, None], keys[None, :]
            a = q[:, :, at] @ k[:, keys].transpose(-1, -2)[:, None] * d ** -0.5
            return _softmax_v(_scores(a, c, slopes, (i - j).abs().float()), seen(i, j), v[:, keys][:, None])

        def causal(i, j):
            return j <= torch.clamp(i, min=prefix - 1)

        def dense(at, keys):
            step = max(1, (1 << 28) // (Hq * keys))
            all_keys = torch.arange(keys, device=DEV)
            return torch.cat([rows(x, all_keys, causal) for x in at.split(step)], 2)

        if c["mode"] == "dense":
            res = dense(torch.arange(n, device=DEV), n)
        else:
            w, ns, g = c["window"], c["n_sink"], c["gamma"]
            step, res = 1024, []
            for r0 in range(0, n, step):
                at = torch.arange(r0, min(n, r0 + step), device=DEV)
                lo = max(0, r0 - w + 1)
                keys = torch.cat([torch.arange(min(ns, lo), device=DEV), torch.arange(lo, min(n, r0 + step), device=DEV)])
                res.append(rows(at, keys, lambda i, j: (j <= i) & ((j < ns) | (i - j < w))))
            res = torch.cat(res, 2)
            whole = n // g * g
            anchors = torch.cat([torch.arange(0, whole, g, device=DEV), torch.arange(whole, n, device=DEV)])
            full = dense(anchors, n)
            if whole:
                delta = full[:, :, :whole // g] - res[:, :, 0:whole:g]
                res[:, :, :whole] += delta.repeat_interleave(g, 2)
            res[:, :, whole:] = full[:, :, whole // g:]
        out[base:base + n] = res.reshape(Hq, n, d).transpose(0, 1)
        base += n
    return out


# ------------------------------------------------------------------------------------ one pass

def run(s):
    c = s["case"]
    kind = c["kind"]
    if own:
        b = _binding()
        if kind != "prefill":
            bf16 = (s["k_pages"], s["v_pages"])
            cache = bf16 + ((s["k_scales"], s["v_scales"]) if kind != "decode" else ()) + (s["table"], s["lens"])
    if kind == "write":
        if own:
            b.pages8_append(s["k"], s["v"], *cache, slots=s["slots"], cu_seqlens=s["cu"], max_seqlen=s["max_new"])
            k, v = b.pages8_read(*cache, s["n_back"], first=s["first"], slots=s["slots"], cu_seqlens=s["back"],
                                 max_seqlen=s["max_back"])
            back = {"k": k, "v": v}
        else:
            _plain_write(s)
            back = _plain_read(s, s["slots"], s["first"], s["back"], s["n_back"])
        return dict(back, k_scales=s["k_scales"], v_scales=s["v_scales"])
    if kind == "read":
        if own:
            k, v = b.pages8_read(*cache, s["n"], cu_seqlens=s["cu"], max_seqlen=s["max_len"])
            return {"k": k, "v": v}
        zero = torch.zeros_like(s["lens"])
        return _plain_read(s, torch.arange(zero.numel(), device=DEV), zero, s["cu"], s["n"])
    if kind in ("attend", "decode"):
        if not own:
            return _plain_attend(s)
        call = b.tree_attn_paged8 if kind == "attend" else b.tree_attn_paged_scored
        return call(s["q"], *cache, mask=s["mask"], cap=c["cap"], slopes=s["slopes"], cu_seqlens=s["cu"],
                    max_seqlen=s["max_q"], max_len=s["max_len"])
    if kind == "pick":
        if not own:
            return _plain_pick(s)
        return b.selected_attn_paged8(s["q"], *cache, s["lists"], cu_seqlens=s["cu"], max_seqlen=s["max_q"])
    if not own:
        return _plain_prefill(s)
    kw = dict(cap=c["cap"], slopes=s["slopes"], cu_seqlens=s["cu"], max_seqlen=s["max_len"])
    if c["mode"] == "dense":
        return b.dense_attn_prefill_scored(s["q"], s["k"], s["v"], prefix=s["prefix"], **kw)
    return b.delta_attn_prefill_scored(s["q"], s["k"], s["v"], window=c["window"], n_sink=c["n_sink"], gamma=c["gamma"], **kw)


# ------------------------------------------------------------------------ the definition, in 64 bits

def _round8(y):
    """The values of e4m3 nearest to y, ties to the even code: 3 bits behind the first, steps of 2^-9 at the least."""
    y = y.double()
    steps = torch.tensor([2.0 ** (x - 9) for x in range(16)], dtype=torch.float64, device=y.device)
    step = steps[(torch.frexp(y)[1].long() + 5).clamp(min=0)]
    return torch.round(y / step) * step


def _least(top):
    """The exponent of the scale of values up to the number `top`."""
    e = LEAST
    while e < MOST and top > 448.0 * 2.0 ** e:
        e += 1
    return e


def _exact_write(case, s):
    Hkv, out = case["Hkv"], {}
    lens, first = _lens(case), _touched(case)
    news, order = _news(case), s["slots"].tolist()
    sizes = [lens[i] - first[i] for i in order]
    if sum(_pages(n) for n in sizes) * Hkv * case["layers"] > 60000:
        return None
    for name in ("k", "v"):
        pages, scales, new = _layered(s, name + "_pages", name + "_scales", name)
        got = torch.zeros((case["layers"], sum(sizes), Hkv, case["d"]), dtype=torch.float64, device=DEV)
        after = scales.double().clone()
        for layer in range(case["layers"]):
            at = back = 0
            for b in order:
                L, m, f = lens[b], news[b], first[b]
                rows = new[layer, at:at + m].double()
                for p0 in range(f, L, PAGE):
                    page = int(s["table"][b, p0 // PAGE])
                    a0, a1 = max(p0, L - m), min(p0 + PAGE, L)
                    x = rows[a0 - (L - m):a1 - (L - m)]
                    tops = x.abs().amax((0, 2)).tolist()
                    before = scales[layer, page].double()
                    e = [_least(t) for t in tops]
                    if a0 > p0:
                        e = [max(y, int(torch.frexp(o)[1]) - 1) for y, o in zip(e, before.cpu())]
                    unit = torch.tensor([2.0 ** y for y in e], dtype=torch.float64, device=DEV)
                    got[layer, back + a0 - f:back + a1 - f] = _round8(x / unit[:, None]) * unit[:, None]
                    if a0 > p0:
                        old = pages[layer, page, :, :a0 - p0].float().double() * before[:, None, None]
                        old = _round8(old / unit[:, None, None]) * unit[:, None, None]
                        got[layer, back:back + a0 - p0] = old.transpose(0, 1)
                    after[layer, page] = unit
                at += m
                back += L - f
        one = case["layers"] == 1
        out[name], out[name + "_scales"] = (got[0], after[0]) if one else (got, after)
    return out


def _held(s, name, pages, h, n):
    """The first n keys or values of kv head h in these pages, in 64 bits."""
    x = s[name + "_pages"]
    if x.dtype == torch.bfloat16:
        return x[pages, h].double().reshape(-1, x.shape[-1])[:n]
    x = x.view(torch.uint8)[pages, h].view(torch.float8_e4m3fn).float().double()
    return (x * s[name + "_scales"][pages, h].double()[:, None, None]).reshape(-1, x.shape[-1])[:n]


def _attend(q, k, v, vis, cap=0.0, bias=None):
    """Rows q [..., rows, d] over keys k, v [keys, d] where vis [rows, keys], in 64 bits."""
    a = (q.double() @ k.double().T) / q.shape[-1] ** 0.5
    if cap:
        a = cap * torch.tanh(a / cap)
    if bias is not None:
        a = a + bias
    a = torch.where(vis, a, torch.full_like(a, -1e300))
    a = torch.where(vis, torch.exp(a - a.max(-1, keepdim=True).values), torch.zeros_like(a))
    z = a.sum(-1, keepdim=True)
    return torch.where(z > 0, a @ v.double() / torch.where(z > 0, z, torch.ones_like(z)), torch.zeros_like(z))


def exact(case, seed):
    kind, Hkv, d = case["kind"], case["Hkv"], case["d"]
    s = prepare(case, seed)
    if kind == "write":
        return _exact_write(case, s)
    lens, at = _lens(case), 0
    if kind == "read":
        lead = (case["layers"],) if case["layers"] > 1 else ()
        got = {x: torch.zeros(lead + (sum(lens), Hkv, d), dtype=torch.float64, device=DEV) for x in ("k", "v")}
        for b, L in enumerate(lens):
            pages = s["table"][b, :_pages(L)].long()
            for name in got:
                raw, sc = s[name + "_pages"].view(torch.uint8), s[name + "_scales"].double()
                for layer in range(case["layers"]):
                    r, c, o = (raw[layer], sc[layer], got[name][layer]) if lead else (raw, sc, got[name])
                    x = r[pages].view(torch.float8_e4m3fn).float().double() * c[pages][:, :, None, None]
                    o[at:at + L] = x.transpose(1, 2).reshape(-1, Hkv, d)[:L]
            at += L
        return got
    q, G = s["q"], case["Hq"] // Hkv
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    if kind == "prefill":
        if sum(n * n for n in lens) * case["Hq"] > 80_000_000_000:
            return None
        for b, n in enumerate(lens):
            p = 0 if s["prefix"] is None else int(s["prefix"][b])
            j = torch.arange(n, device=DEV)
            for h in range(case["Hq"]):
                k, v, qh = s["k"][at:at + n, h // G], s["v"][at:at + n, h // G], q[at:at + n, h]
                slope = 0.0 if s["slopes"] is None else float(s["slopes"][h])

                def part(i, vis):
                    bias = -slope * (i[:, None] - j).abs().double() if slope else None
                    return _attend(qh[i], k, v, vis, case["cap"], bias)

                for i in j.split(4096):
                    out[at + i, h] = part(i, j <= torch.clamp(i, min=p - 1)[:, None])
                if case["mode"] == "delta":
                    g, whole = case["gamma"], n // case["gamma"] * case["gamma"]
                    full = out[at:at + n, h].clone()
                    for i in j.split(4096):
                        near = (i[:, None] - j < case["window"]) | (j < case["n_sink"])
                        out[at + i, h] = part(i, (j <= i[:, None]) & near)
                    a = j // g * g
                    shift = (full - out[at:at + n, h])[a]
                    out[at:at + n, h] = torch.where((j < whole)[:, None], out[at:at + n, h] + shift, full)
            at += n
        return out
    if sum(lens) * Hkv > 12_000_000:
        return None
    for b, (L, m) in enumerate(zip(lens, _news(case))):
        pages = s["table"][b, :_pages(L)].long()
        for h in range(Hkv):
            k, v = _held(s, "k", pages, h, L), _held(s, "v", pages, h, L)
            heads = slice(h * G, (h + 1) * G)
            for i in range(m):
                pos, row = L - m + i, q[at + i, heads]
                j = torch.arange(L, device=DEV)
                if kind == "pick":
                    mine = [x for x in s["lists"][at + i, h].tolist() if x >= 0] + [pos // PAGE]
                    vis = torch.isin(j // PAGE, torch.tensor(mine, device=DEV)) & (j <= pos)
                    out[at + i, heads] = _attend(row, k, v, vis)
                    continue
                vis = j <= pos
                if s["mask"] is not None:
                    w = s["mask"][at + i].tolist()
                    vis = torch.ones(L, dtype=torch.bool, device=DEV)
                    vis[L - m:] = torch.tensor([bool(w[x // 64] >> x % 64 & 1) for x in range(m)], device=DEV)
                bias = None
                if s["slopes"] is not None:
                    bias = -s["slopes"][heads].double()[:, None] * (pos - j).abs().double()
                out[at + i, heads] = _attend(row, k, v, vis, case["cap"], bias)
        at += m
    return out
