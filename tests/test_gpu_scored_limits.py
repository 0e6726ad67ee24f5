"""Attention under changed scores at the ends of what its arguments may be, against the definition in 64 bits
(tolerances: scored.py)."""
from __future__ import annotations

import pytest
import torch

from scored import slopes_of
from test_gpu_scored import check_dense, i32, inputs

pytestmark = pytest.mark.gpu

INT_MIN, INT_MAX = -2 ** 31, 2 ** 31 - 1


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap,biased", [(0.0, False), (0.0, True), (6.0, True)])
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
