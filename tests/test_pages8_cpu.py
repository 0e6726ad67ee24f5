"""The 8-bit cache's calls and the attentions under changed scores without a GPU: argument checks of the C
ABI, which come before any HIP call, workspaces, and the binding's own checks."""
from __future__ import annotations

import ctypes
import math
import os

import pytest
import torch

from paper_2505_11254_amd import binding
from test_paged_cpu import ALIGN, HIP, NULL, PARAM, PTR, SHAPE, UNSUP, WORKSPACE

TREE = dict(out=PTR, lse=None, table=PTR, lens=PTR, S=4, M=8, P=16, slots=None, cu=None, B=2, N=3, max_len=512, Hq=8,
            Hkv=2, d=128, mask=None, words=0, cap=0.0, slopes=None, ws=PTR, size=1 << 40, stream=None)
PAGES = dict(k=PTR, v=PTR, ks=PTR, vs=PTR)
PREFILL = dict(q=PTR, k=PTR, v=PTR, out=PTR, cu=None, B=2, N=100, Hq=8, Hkv=2, d=128)
SCORE = dict(cap=0.0, slopes=None)
ARGS = {
    "dense_attn_prefill_scored": dict(**PREFILL, **SCORE, prefix=None, stream=None),
    "sparse_attn_prefill_scored": dict(**PREFILL, window=16, n_sink=2, **SCORE, stream=None),
    "delta_attn_prefill_scored": dict(**PREFILL, window=16, n_sink=2, gamma=8, **SCORE, ws=PTR, size=1 << 40, stream=None),
    "tree_attn_paged_scored": dict(q=PTR, k=PTR, v=PTR, **TREE),
    "tree_attn_paged8": dict(q=PTR, **PAGES, **TREE),
    "selected_attn_paged8": dict(q=PTR, **PAGES, out=PTR, lse=None, table=PTR, lens=PTR, S=4, M=8, P=16, slots=None, cu=None,
                                 B=2, N=3, Hq=8, Hkv=2, d=128, pages=PTR, top_k=4, ws=PTR, size=1 << 40, stream=None),
    "da_pages8_resize": dict(**PAGES, layers=2, Hkv=2, d=128, table=PTR, lens=PTR, refs=PTR, S=4, M=8, P=16, slots=PTR,
                             new_lens=PTR, n=2, result=PTR, stream=None),
    "da_pages8_append": dict(nk=PTR, nv=PTR, T=6, **PAGES, layers=2, Hkv=2, d=128, table=PTR, lens=PTR, S=4, M=8, P=16,
                             slots=PTR, cu=PTR, B=2, N=3, new_lens=None, stream=None),
    "da_pages8_compact": dict(**PAGES, layers=2, Hkv=2, d=128, table=PTR, lens=PTR, refs=PTR, S=4, M=8, P=16, slots=PTR,
                              start=PTR, keep=PTR, n_keep=3, cu_keep=PTR, n=2, result=PTR, stream=None),
    "da_pages8_read": dict(nk=PTR, nv=PTR, T=6, **PAGES, layers=2, Hkv=2, d=128, table=PTR, lens=PTR, S=4, M=8, P=16,
                           slots=PTR, cu=PTR, B=2, N=3, first=None, stream=None),
    "da_page8_summary": dict(k=PTR, ks=PTR, Hkv=2, d=128, table=PTR, lens=PTR, S=4, M=8, P=16, slots=None, first=None, B=2,
                             max_new=100, codes=PTR, scales=PTR, stream=None),
}
PREFILLS = ["dense_attn_prefill_scored", "sparse_attn_prefill_scored", "delta_attn_prefill_scored"]
SCORED = PREFILLS + ["tree_attn_paged_scored", "tree_attn_paged8"]
NO_CAP = [-1.0, -2.0 ** -10, 2.0 ** -10 * 0.999, 1024.5, 2.0 ** 60, math.inf, -math.inf, math.nan, -math.nan]
ROWS = ["da_pages8_append", "da_pages8_read"]
REFUSED = (
    [(f, PARAM, {"cap": c}) for f in SCORED for c in NO_CAP]
    + [(f, ALIGN, {"slopes": PTR + 2}) for f in SCORED]
    + [(f, NULL, {n: None}) for f in PREFILLS for n in "qkv"] + [(f, NULL, {"out": None}) for f in PREFILLS]
    + [(f, SHAPE, {n: 0}) for f in PREFILLS for n in ("B", "N", "Hq", "Hkv")] + [(f, UNSUP, {"d": 96}) for f in PREFILLS]
    + [(f, ALIGN, {n: PTR + 8}) for f in PREFILLS for n in "qkv"]
    + [("dense_attn_prefill_scored", ALIGN, {"prefix": PTR + 1}), ("sparse_attn_prefill_scored", PARAM, {"window": 0}),
       ("delta_attn_prefill_scored", PARAM, {"gamma": 0}), ("delta_attn_prefill_scored", WORKSPACE, {"ws": None}),
       ("delta_attn_prefill_scored", WORKSPACE, {"size": 10})]
    + [(f, PARAM, {"slopes": PTR, "mask": PTR, "words": 1}) for f in ("tree_attn_paged_scored", "tree_attn_paged8")]
    + [(f, PARAM, {"mask": PTR, "words": 0}) for f in ("tree_attn_paged_scored", "tree_attn_paged8")]
    + [(f, SHAPE, {n: 0}) for f in ("tree_attn_paged_scored", "tree_attn_paged8") for n in ("B", "N", "max_len", "S", "M", "P")]
    + [(f, NULL, {n: None}) for f in ARGS for n in ("ks", "vs") if n in ARGS[f]]
    + [(f, ALIGN, {n: PTR + 2}) for f in ARGS for n in ("ks", "vs") if n in ARGS[f]]
    + [(f, NULL, {n: None}) for f in ROWS for n in ("nk", "nv", "k", "v", "table", "lens")]
    + [(f, SHAPE, {n: 0}) for f in ROWS for n in ("B", "N", "layers", "Hkv", "S", "M", "P")]
    + [(f, SHAPE, {"T": -1}) for f in ROWS] + [(f, SHAPE, {"cu": None, "T": 7}) for f in ROWS]
    + [(f, SHAPE, {"slots": None, "B": 5}) for f in ROWS] + [(f, UNSUP, {"d": 32}) for f in ROWS]
    + [(f, ALIGN, {n: PTR + 8}) for f in ROWS for n in ("nk", "nv", "k", "v")]
    # a workgroup for each page that a sequence may touch, layer, keys or values and head
    + [(f, SHAPE, {"N": (1 << 31) - 1, "T": 1 << 40}) for f in ROWS]
    + [(f, SHAPE, {"layers": 32767, "Hkv": (1 << 31) - 1}) for f in ROWS]
    + [("da_pages8_append", ALIGN, {"new_lens": PTR + 2}), ("da_pages8_read", ALIGN, {"first": PTR + 2}),
       ("da_pages8_resize", UNSUP, {"d": 256}), ("da_pages8_resize", SHAPE, {"n": 1025}),
       ("da_pages8_resize", NULL, {"refs": None}), ("da_pages8_resize", ALIGN, {"result": PTR + 8}),
       ("da_pages8_compact", NULL, {"cu_keep": None}), ("da_pages8_compact", SHAPE, {"n_keep": -1}),
       ("da_pages8_compact", SHAPE, {"layers": 128, "Hkv": 65, "n": 1024}), ("da_pages8_compact", ALIGN, {"result": PTR + 4}),
       ("da_page8_summary", SHAPE, {"max_new": 0}), ("da_page8_summary", NULL, {"codes": None}),
       ("selected_attn_paged8", NULL, {"pages": None}), ("selected_attn_paged8", PARAM, {"top_k": 0})])


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        pytest.skip("library not built")
    return binding.load_library()


@pytest.mark.parametrize("fn", sorted(ARGS))
def test_calls_refuse_bad_arguments(lib, fn):
    seen = 0
    for name, status, change in REFUSED:
        if name == fn:
            args = dict(ARGS[fn])
            assert set(change) <= set(args)
            args.update(change)
            assert getattr(lib, fn)(*args.values()) == status, change
            seen += 1
    assert seen


@pytest.mark.parametrize("fn", sorted(ARGS))
def test_calls_pass_their_checks_with_good_arguments(lib, fn):
    if torch.cuda.is_available():
        pytest.skip("the pointers are not real ones")
    for cap in (0.0, -0.0, 2.0 ** -10, 50.0, 1024.0) if "cap" in ARGS[fn] else (0.0,):
        args = dict(ARGS[fn])
        if "cap" in args:
            args["cap"] = cap
        assert getattr(lib, fn)(*args.values()) == HIP


def test_workspaces(lib):
    f = lib.da_paged8_workspace_bytes
    assert f(0, 1, 8, 2, 128, 100, 0) == 0 and f(1, 1, 8, 3, 128, 100, 0) == 0 and f(1, 1, 8, 2, 96, 100, 0) == 0
    assert f(1, 1, 8, 2, 128, 0, 0) == 0 and f(1, 1, 8, 2, 128, 64, 0) == 0
    assert f(1, 1, 32, 8, 128, 131072, 0) > 0
    args = dict(ARGS["tree_attn_paged8"], B=1, M=4096, max_len=131072, Hq=32, Hkv=8)
    need = f(1, 3, 32, 8, 128, 131072, 0)
    assert lib.tree_attn_paged8(*dict(args, size=need - 1).values()) == WORKSPACE
    assert lib.tree_attn_paged8(*dict(args, ws=PTR + 8).values()) == ALIGN


def test_binding_checks(monkeypatch):
    """Types, shapes and devices are looked at before anything is called."""
    def refuse(*a, **k):
        raise AssertionError("the C library was reached")
    monkeypatch.setattr(binding, "load_library", refuse)
    f8, bf = torch.float8_e4m3fn, torch.bfloat16
    k8 = torch.zeros(4, 2, 64, 64, dtype=torch.uint8).view(f8)
    sc = torch.ones(4, 2)
    table, lens = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    rows = torch.zeros(6, 2, 64, dtype=bf)
    with pytest.raises(ValueError):  # tensors on the CPU
        binding.pages8_append(rows, rows, k8, k8, sc, sc, table, lens, B=2)
    with pytest.raises(ValueError):
        binding.tree_attn_paged8(rows, k8, k8, sc, sc, table, lens, B=2)
    with pytest.raises(ValueError):
        binding.dense_attn_prefill_scored(rows, rows, rows)
    assert isinstance(binding.SIGNATURES["tree_attn_paged8"], str) and ctypes.sizeof(ctypes.c_float) == 4


class OnGpu:
    """The binding's checks with tensors that count as being on the device they are compared with."""

    def __init__(self, monkeypatch):
        monkeypatch.setattr(binding, "_on_device", self.check)

    @staticmethod
    def check(name, t, dev, dtype):
        if dtype is not None and t.dtype != dtype:
            raise ValueError(f"{name} must be {dtype}")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")


def test_shapes_of_codes_and_scales(monkeypatch):
    OnGpu(monkeypatch)
    f8 = torch.float8_e4m3fn

    def c(*shape):
        return torch.zeros(*shape, dtype=torch.uint8).view(f8)
    ok = c(4, 2, 64, 64)
    assert binding._pages8(ok, ok, torch.ones(4, 2), torch.ones(4, 2))[1:] == (1, 4, 2, 64)
    deep = c(3, 4, 2, 64, 64)
    assert binding._pages8(deep, deep, torch.ones(3, 4, 2), torch.ones(3, 4, 2), layered=True)[1:] == (3, 4, 2, 64)
    bad = [(c(4, 2, 64, 64).view(torch.uint8), ok, torch.ones(4, 2), torch.ones(4, 2)),
           (ok, c(4, 2, 64, 128), torch.ones(4, 2), torch.ones(4, 2)),
           (ok, ok, torch.ones(4, 2).double(), torch.ones(4, 2)), (ok, ok, torch.ones(4, 2), torch.ones(4, 3)),
           (ok, ok, torch.ones(4), torch.ones(4, 2)), (ok, ok, torch.ones(2, 4).T, torch.ones(4, 2)),
           (c(4, 2, 32, 64), c(4, 2, 32, 64), torch.ones(4, 2), torch.ones(4, 2)),
           (ok.transpose(0, 1), ok.transpose(0, 1), torch.ones(2, 4), torch.ones(2, 4)),
           (deep, deep, torch.ones(3, 4, 2), torch.ones(3, 4, 2))]
    for args in bad:
        with pytest.raises(ValueError):
            binding._pages8(*args)
    for slopes in (torch.ones(7), torch.ones(8, 1), torch.ones(8).double(), torch.ones(16)[::2]):
        with pytest.raises(ValueError):
            binding._slopes(slopes, 8, torch.device("cpu"))
