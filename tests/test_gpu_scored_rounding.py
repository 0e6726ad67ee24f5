"""The weights of corrected rows under changed scores round alike in every chunk of the key axis and in the sparse rows,
so that the roundings of the keys that an anchor's dense and sparse rows share cancel in their difference.

The keys that the sparse rows of the last group leave out are set to have no weight there (their scores lie some 200
below the others', 50 under the cap).  What is left of the correction are roundings in 32 bits: sums of some 2100
terms, a few 2^-18 of them, and weights that lie so near the border between two bf16 values that those steps take
them across (of 2100 a handful, each by 2^-8 of itself: 2^-13 of the output).  They turn the rounding of an output,
whose half step is 2^-9 of it at the least, in one of ten outputs at most; a fifth are allowed.  Were the weights
rounded otherwise in the chunks, independent errors of 2^-9 / sqrt 3 of each, twice, would come to 2^-9.3 of an output
and turn every third."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap,slope", [(0.0, None), (60.0, None), (0.0, 1e-3), (0.0, 1e-5), (60.0, 1e-4), (0.0, -1e-4)])
def test_corrections_without_difference(d, cap, slope):
    from paper_2505_11254_amd import binding
    N, Hq, window, gamma, n_sink = 4096, 4, 2048, 64, 64
    g = torch.Generator().manual_seed(d)
    q, k, v = (torch.randn((N, h, d), generator=g) for h in (Hq, 1, 1))
    q[..., 0] = 2.0 * d ** 0.5
    k[..., 0] = 0.0
    k[n_sink:N - window + 1, :, 0] = -100.0
    q, k, v = (x.to(torch.bfloat16).cuda() for x in (q, k, v))
    kw = dict(window=window, n_sink=n_sink, cap=cap, slopes=None if slope is None else torch.full((Hq,), slope, device="cuda"))
    want = binding.sparse_attn_prefill_scored(q, k, v, **kw)[N - gamma:]
    got = binding.delta_attn_prefill_scored(q, k, v, gamma=gamma, **kw)[N - gamma:]
    turned = (got != want).float().mean().item()
    print(f"turned {turned:.4f}")
    assert (got - want).float().abs().max() <= 2.0 ** -7 * want.float().abs().max()
    assert turned <= 0.2
