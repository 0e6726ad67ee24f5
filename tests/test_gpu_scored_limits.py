"""Attention under changed scores at the ends of what its arguments may be, against the definition in 64 bits
(tolerances: scored.py)."""
from __future__ import annotations

import pytest
import torch

from paged_sim import PAGE
from pages8_sim import NAN
from scored import HALF, attend, slopes_of, tolerance
from test_gpu_paged8_attn import Case8, call, upto
from test_gpu_scored import bias_of, check_dense, i32, inputs

pytestmark = pytest.mark.gpu

INT_MIN, INT_MAX = -2 ** 31, 2 ** 31 - 1


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap,biased", [(0.0, False), (0.0, True), (6.0, True), (6.0, False)])
def test_every_int_is_a_prefix(d, cap, biased):
    """Below 1: no token; past the sequence: all of them."""
    from paper_2505_11254_amd import binding
    prefix = (INT_MIN, INT_MIN + 1, INT_MIN + 70, -1, 0, INT_MAX, INT_MAX - 1, INT_MIN, INT_MAX)
    lens = (130, 70, 65, 64, 33, 130, 1, 1, 0)
    q, k, v, cu = inputs(lens, 4, 2, d, seed=d)
    slopes = slopes_of(4) if biased else None
    out = binding.dense_attn_prefill_scored(q.cuda(), k.cuda(), v.cuda(), cap=cap,
                                            slopes=slopes.cuda() if biased else None, prefix=i32(prefix),
                                            cu_seqlens=i32(cu), max_seqlen=130)
    check_dense(out, q, k, v, cu, cap, slopes, prefix)


@pytest.mark.parametrize("Hq,Hkv,d", [(4, 2, 64), (8, 2, 128)])
@pytest.mark.parametrize("cap,std,biased", [(50.0, 0.5, False), (2.0, 4.0, False), (1.0, 30.0, False), (1.0, 30.0, True),
                                            (0.0, 4.0, True)])
@pytest.mark.parametrize("bad", [0, 37, 129])
def test_rows_that_see_a_nan_key_are_nan_and_the_others_as_without_it(Hq, Hkv, d, cap, std, biased, bad):
    """(the cap's three forms: small, wide and mixed scores)"""
    from paper_2505_11254_amd import binding
    n, window = 200, 50
    q, k, v, cu = inputs((n,), Hq, Hkv, d, seed=bad + d, std=std)
    slopes = slopes_of(Hq) if biased else None
    broken = k.clone()
    broken[bad, 1, 5] = float("nan")
    kw = dict(cap=cap, slopes=slopes.cuda() if biased else None)
    dev = [x.cuda() for x in (q, broken, v)]
    i, top = torch.arange(n), float(v.double().abs().max())
    causal = i <= i[:, None]
    for out, vis in ((binding.dense_attn_prefill_scored(*dev, **kw), causal),
                     (binding.sparse_attn_prefill_scored(*dev, window=window, n_sink=3, **kw),
                      causal & ((i < 3) | (i[:, None] - i < window)))):
        out = out.float().cpu().double()
        for h in range(Hq):
            g = h * Hkv // Hq
            sees = vis[:, bad] if g == 1 else torch.zeros(n, dtype=torch.bool)
            want, _, dev_, dl = attend(q[:, h], k[:, g], v[:, g], vis, cap, bias_of(slopes, h, n))
            assert torch.isnan(out[sees, h]).all(), h
            assert ((out[:, h] - want).abs() <= tolerance(want, dev_, dl, top))[~sees].all(), h


@pytest.mark.parametrize("eight", [True, False])
@pytest.mark.parametrize("Hq,Hkv,d,m", [(8, 2, 64, 1), (8, 2, 128, 1), (32, 8, 128, 3), (16, 2, 128, 12)])
@pytest.mark.parametrize("cap,std", [(50.0, 0.5), (0.25, 20.0), (0.0, 2.0)])
def test_a_nan_key_in_the_cache(eight, Hq, Hkv, d, m, cap, std):
    """Of three sequences two have a broken key: one that all rows see, one that only the last row does."""
    lens = [300, 300, 90 + m]
    c = Case8(lens, [m] * 3, Hq, Hkv, d, seed=m + d, eight=eight, std=std)
    bad = {1: 70, 2: 90 + m - 1}
    for b, j in bad.items():
        page = int(c.table[c.slots[b], j // PAGE])
        if eight:
            c.k8.view(torch.uint8)[page, 0, j % PAGE, 9] = NAN
        else:
            c.k[page, 0, j % PAGE, 9] = float("nan")
    lse = torch.zeros((c.cu[-1], Hq), device="cuda")
    out = call(c, lse=lse, cap=cap).float().cpu().double()
    lse, G = lse.cpu().double(), Hq // Hkv
    for b, n in enumerate(lens):
        for g in range(Hkv):
            k, v = c.keys(b, g)
            k = torch.nan_to_num(k.double(), nan=0.0)
            s = slice(c.cu[b], c.cu[b + 1])
            vis = torch.stack([upto(c)(b, i, g) for i in range(m)])
            sees = vis[:, bad[b]] if b in bad and g == 0 else torch.zeros(m, dtype=torch.bool)
            for h in range(g * G, (g + 1) * G):
                want, wlse, dev, dl = attend(c.q[s, h], k, v, vis, cap)
                assert torch.isnan(out[s, h][sees]).all(), (b, h)
                assert ((out[s, h] - want).abs() <= tolerance(want, dev, dl, float(v.double().abs().max())))[~sees].all()
                assert ((lse[s, h] - wlse).abs() <= HALF * (1 + 2 ** -7) + dl)[~sees].all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("slope", [1024.0, -1024.0])
@pytest.mark.parametrize("cap", [0.0, 30.0])
def test_the_steepest_slopes(d, slope, cap):
    """One key has all the weight: the nearest, or the farthest that a row sees."""
    from paper_2505_11254_amd import binding
    lens, Hq = (700, 0, 1, 65), 4
    q, k, v, cu = inputs(lens, Hq, 2, d, seed=d)
    slopes = torch.full((Hq,), slope)
    dev = [x.cuda() for x in (q, k, v)]
    kw = dict(cap=cap, slopes=slopes.cuda(), cu_seqlens=i32(cu), max_seqlen=700)
    for prefix in (None, (130, 5, 1, 64)):
        out = binding.dense_attn_prefill_scored(*dev, prefix=i32(prefix) if prefix else None, **kw)
        check_dense(out, q, k, v, cu, cap, slopes, prefix)
    # (sinks and window: the first key is among those seen; the correction's three attentions agree.  Each is one
    # weight times one value, exact in 32 bits, over that weight, with a rounding of the reciprocal, of the product and
    # of a merge: 3 2^-24 of its value, of which a corrected row adds those of its anchor's.)
    tiny = 9 * 2.0 ** -24 * float(v.float().abs().max())
    for out in (binding.sparse_attn_prefill_scored(*dev, window=100, n_sink=2, **kw),
                binding.delta_attn_prefill_scored(*dev, window=100, n_sink=2, gamma=32, **kw)):
        out = out.float().cpu()
        for b in range(len(lens)):
            rows = torch.arange(cu[b], cu[b + 1]) if slope > 0 else torch.full((lens[b],), cu[b])
            for h in range(Hq):
                want = v[rows, h // 2].float()
                assert ((out[cu[b]:cu[b + 1], h] - want).abs() <= HALF * 2 * want.abs() + tiny).all()


@pytest.mark.parametrize("eight", [True, False])
@pytest.mark.parametrize("Hq,Hkv,d,m", [(8, 2, 64, 1), (8, 2, 128, 1), (32, 8, 128, 3), (16, 2, 128, 12)])
@pytest.mark.parametrize("slope,cap", [(1024.0, 0.0), (-1024.0, 0.0), (1024.0, 20.0), (-1024.0, 20.0)])
def test_the_steepest_slopes_over_the_cache(eight, Hq, Hkv, d, m, slope, cap):
    c = Case8([300, 64 + m, 5000, m], [m] * 4, Hq, Hkv, d, seed=m + d, eight=eight)
    slopes = torch.full((Hq,), slope)
    lse = torch.zeros((c.cu[-1], Hq), device="cuda")
    c.verify(call(c, lse=lse, cap=cap, slopes=slopes.cuda()), lse, upto(c), cap, slopes)


@pytest.mark.parametrize("eight", [True, False])
@pytest.mark.parametrize("slope", [-0.84, -0.0123, 0.0123, 3e-5])
def test_biased_scores_of_far_keys(eight, slope):
    """The log-sum-exp of a single token over 131075 keys: off by no more than its scores may be (the bound:
    test_scored_error.py), and by its own steps in 32 bits, 2^-22 of it and of 1, with 2^-12 for the weights' sum (that
    many keys have weight, in sums of some 2^11 terms a lane)."""
    n, d = 131075, 64
    c = Case8([n], [1], 4, 1, d, seed=8, eight=eight)
    slopes = torch.full((4,), slope)
    lse = torch.zeros((1, 4), device="cuda")
    c.verify(call(c, lse=lse, slopes=slopes.cuda()), None, upto(c), 0.0, slopes)
    k, v = c.keys(0, 0)
    bias = -float(slopes[0]) * torch.arange(n - 1, -1, -1).double()[None]
    for h in range(4):
        _, want, _, _ = attend(c.q[:, h], k, v, torch.ones((1, n), dtype=torch.bool), 0.0, bias)
        products = d * 2.0 ** -24 * float((c.q[0, h].double().abs() @ k.double().abs().T).max()) / d ** 0.5 + 2.0 ** -20
        top = float((c.q[0, h].double() @ k.double().T / d ** 0.5 + bias).abs().max())
        bound = 2.0 ** -10 * abs(slope) + 2.0 ** -21 * (float(bias.abs().max()) + top) + products
        assert abs(float(lse[0, h]) - float(want)) <= bound + 2.0 ** -22 * (abs(float(want)) + 1) + 2.0 ** -12
