"""The paged cache's calls, the attention over it and the block selection without a
GPU: argument checks of the C ABI (which come before any HIP call), launch plans, and
the binding's own checks."""
from __future__ import annotations

import ctypes
import os

import pytest
import torch

from paper_2505_11254_amd import binding

OK, NULL, SHAPE, PARAM, UNSUP, ALIGN, WORKSPACE, HIP = range(8)
# Pointers that are never followed: every refusal here comes before the device is looked at,
# and on a machine without a GPU what passes all checks ends in DA_ERR_HIP.
PTR = 1 << 20


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        pytest.skip("library not built")
    return binding.load_library()


ARGS = {
    "da_pages_fork": dict(table=PTR, lens=PTR, refs=PTR, S=4, M=8, P=16, src=PTR, dst=PTR, n=2, result=PTR, stream=None),
    "da_pages_resize": dict(k=PTR, v=PTR, layers=2, Hkv=2, d=128, table=PTR, lens=PTR, refs=PTR, S=4, M=8, P=16, slots=PTR,
                            new_lens=PTR, n=2, result=PTR, stream=None),
    "da_pages_append": dict(k=PTR, v=PTR, T=6, k_pages=PTR, v_pages=PTR, layers=2, Hkv=2, d=128, table=PTR, lens=PTR, S=4,
                            M=8, P=16, slots=PTR, cu=PTR, B=2, N=3, stream=None),
    "da_pages_compact": dict(k=PTR, v=PTR, layers=2, Hkv=2, d=128, table=PTR, lens=PTR, refs=PTR, S=4, M=8, P=16, slots=PTR,
                             start=PTR, keep=PTR, n_keep=3, cu_keep=PTR, n=2, result=PTR, stream=None),
    "tree_attn_paged": dict(q=PTR, k=PTR, v=PTR, out=PTR, lse=None, table=PTR, lens=PTR, S=4, M=8, P=16, slots=None, cu=None,
                            B=2, N=3, max_len=512, Hq=8, Hkv=2, d=128, mask=PTR, words=1, ws=PTR, size=1 << 40,
                            stream=None),
    "selected_attn_paged": dict(q=PTR, k=PTR, v=PTR, out=PTR, lse=None, table=PTR, lens=PTR, S=4, M=8, P=16, slots=None,
                                cu=None, B=2, N=3, Hq=8, Hkv=2, d=128, pages=PTR, top_k=4, ws=PTR, size=1 << 40,
                                stream=None),
    "da_key_summary": dict(k=PTR, cu=None, B=2, N=100, Hkv=2, d=128, codes=PTR, scales=PTR, stream=None),
    "da_page_summary": dict(k=PTR, Hkv=2, d=128, table=PTR, lens=PTR, S=4, M=8, P=16, slots=None, first=None, B=2,
                            max_new=100, codes=PTR, scales=PTR, stream=None),
    "da_select_blocks": dict(q=PTR, codes=PTR, scales=PTR, cu=None, B=2, N=1000, Hq=8, Hkv=2, d=128, top_k=4, n_sink=1,
                             n_recent=1, block_q=64, ptr=PTR, idx=PTR, stream=None),
    "da_select_pages": dict(q=PTR, codes=PTR, scales=PTR, table=PTR, lens=PTR, S=4, M=8, P=16, slots=None, cu=None, B=2, N=3,
                            max_len=512, Hq=8, Hkv=2, d=128, top_k=4, n_sink=1, n_recent=1, pages=PTR, ws=PTR,
                            size=1 << 40, stream=None),
}

REFUSED = [
    ("da_pages_fork", NULL, ["table", "lens", "refs", "src", "dst", "result"], None),
    ("da_pages_fork", SHAPE, ["S", "M", "P", "n"], 0),
    ("da_pages_fork", SHAPE, ["n"], 1025),
    ("da_pages_fork", SHAPE, ["M"], (1 << 31) // 64),
    ("da_pages_fork", ALIGN, ["table", "lens", "refs", "src", "dst", "result"], PTR + 2),
    ("da_pages_resize", NULL, ["k", "v", "table", "lens", "refs", "slots", "result"], None),
    ("da_pages_resize", SHAPE, ["layers", "Hkv", "S", "M", "P", "n"], 0),
    ("da_pages_resize", SHAPE, ["n"], 1025),
    ("da_pages_resize", SHAPE, ["layers"], 32768),
    ("da_pages_resize", UNSUP, ["d"], 96),
    ("da_pages_resize", ALIGN, ["k", "v", "result"], PTR + 4),
    ("da_pages_append", NULL, ["k", "v", "k_pages", "v_pages", "table", "lens"], None),
    ("da_pages_append", SHAPE, ["B", "N"], 0),
    ("da_pages_append", SHAPE, ["T"], -1),
    ("da_pages_append", UNSUP, ["d"], 32),
    ("da_pages_append", ALIGN, ["k", "v", "k_pages", "v_pages"], PTR + 8),
    ("da_pages_compact", NULL, ["k", "v", "table", "lens", "refs", "slots", "start", "keep", "cu_keep", "result"], None),
    ("da_pages_compact", SHAPE, ["n_keep"], -1),
    ("da_pages_compact", SHAPE, ["n"], 0),
    ("da_pages_compact", ALIGN, ["result"], PTR + 8),
    ("tree_attn_paged", NULL, ["q", "k", "v", "out", "table", "lens"], None),
    ("tree_attn_paged", SHAPE, ["S", "M", "P", "B", "N", "max_len", "Hq", "Hkv"], 0),
    ("tree_attn_paged", SHAPE, ["Hq"], 7),
    ("tree_attn_paged", SHAPE, ["B"], 5),
    ("tree_attn_paged", UNSUP, ["d"], 256),
    ("tree_attn_paged", ALIGN, ["q", "k", "v", "out", "ws"], PTR + 8),
    ("tree_attn_paged", ALIGN, ["mask"], PTR + 4),
    ("tree_attn_paged", PARAM, ["words"], 0),
    ("selected_attn_paged", NULL, ["q", "k", "v", "out", "table", "lens", "pages"], None),
    ("selected_attn_paged", PARAM, ["top_k"], 0),
    ("selected_attn_paged", SHAPE, ["B"], 5),
    ("da_key_summary", NULL, ["k", "codes", "scales"], None),
    ("da_key_summary", SHAPE, ["B", "N", "Hkv"], 0),
    ("da_key_summary", UNSUP, ["d"], 127),
    ("da_key_summary", ALIGN, ["k", "codes"], PTR + 8),
    ("da_page_summary", NULL, ["k", "table", "lens", "codes", "scales"], None),
    ("da_page_summary", SHAPE, ["B", "max_new", "S", "M", "P"], 0),
    ("da_select_blocks", NULL, ["q", "codes", "scales", "ptr", "idx"], None),
    ("da_select_blocks", SHAPE, ["B", "N", "Hq", "Hkv"], 0),
    ("da_select_blocks", PARAM, ["top_k"], 1),
    ("da_select_blocks", PARAM, ["n_sink", "n_recent"], -1),
    ("da_select_blocks", PARAM, ["n_sink"], (1 << 31) - 1),
    ("da_select_blocks", PARAM, ["block_q"], 32),
    ("da_select_blocks", UNSUP, ["N"], 24576 * 64 + 1),
    ("da_select_pages", NULL, ["q", "codes", "scales", "table", "lens", "pages"], None),
    ("da_select_pages", PARAM, ["top_k"], 1),
    ("da_select_pages", PARAM, ["n_recent"], 4),
]


@pytest.mark.parametrize("fn,status,names,value", REFUSED)
def test_calls_refuse_bad_arguments(lib, fn, status, names, value):
    for name in names:
        args = dict(ARGS[fn])
        assert name in args
        args[name] = value
        assert getattr(lib, fn)(*args.values()) == status, (name, value)


@pytest.mark.parametrize("fn,sizes", [
    ("da_pages_resize", dict(layers=32767, Hkv=(1 << 31) - 1)),
    ("da_pages_resize", dict(n=1024, layers=128, Hkv=65)),
    ("da_pages_compact", dict(n=1024, layers=128, Hkv=65)),
    ("da_pages_append", dict(B=16, slots=PTR, N=(1 << 27) - 1, Hkv=1)),
    ("tree_attn_paged", dict(B=4, N=1 << 20, Hq=64, Hkv=64, words=1 << 20)),
    ("tree_attn_paged", dict(B=4, N=(1 << 31) - 1, Hq=(1 << 31) - 1, Hkv=1, words=1 << 30)),
    ("selected_attn_paged", dict(B=4, N=1 << 20, Hq=32, Hkv=32)),
    ("da_key_summary", dict(B=1 << 15, cu=PTR, N=1 << 20, Hkv=1)),
    ("da_page_summary", dict(B=1 << 26, slots=PTR, max_new=64, Hkv=1)),
    ("da_select_blocks", dict(B=1 << 20, cu=PTR, N=64, Hkv=8)),
    ("da_select_blocks", dict(B=1, N=512, Hq=1 << 16, Hkv=1, block_q=256)),
    ("da_select_pages", dict(B=4, N=1 << 20, Hq=4, Hkv=4)),
    ("da_select_pages", dict(B=1, N=1 << 20, Hq=4, Hkv=4, M=8192, max_len=8192 * 64)),
])
def test_calls_refuse_what_no_launch_can_hold(lib, fn, sizes):
    """Threads are counted in 32 bits in a launch, byte offsets inside a query block too."""
    assert getattr(lib, fn)(*dict(ARGS[fn], **sizes).values()) == SHAPE


@pytest.mark.parametrize("sizes", [dict(N=(1 << 31) - 1, Hkv=(1 << 31) - 1), dict(N=(1 << 31) - 1, Hkv=1 << 30, d=64),
                                   dict(N=1 << 30, Hkv=1 << 30), dict(N=3, Hkv=1 << 28)])
def test_append_refuses_sizes_whose_product_wraps(lib, sizes):
    a = dict(ARGS["da_pages_append"], B=1, T=1, **sizes)
    assert lib.da_pages_append(*a.values()) == SHAPE


@pytest.mark.parametrize("Hq,Hkv,d", [(1 << 24, 1, 128), (1 << 26, 2, 64), ((1 << 27) - 1, 1, 128)])
def test_page_selection_refuses_groups_past_32_bits(lib, Hq, Hkv, d):
    """Channels of a token's heads on one kv head are counted in 32 bits."""
    a = dict(ARGS["da_select_pages"], B=1, N=1, Hq=Hq, Hkv=Hkv, d=d)
    assert lib.da_select_pages(*a.values()) == SHAPE


@pytest.mark.parametrize("top_k", [(1 << 30) + 1, (1 << 31) - 2, (1 << 31) - 1])
def test_attention_refuses_lists_past_what_is_counted(lib, top_k):
    """A list and its own page are counted in 32 bits: one page more than the largest int is no small list."""
    assert lib.selected_attn_paged(*dict(ARGS["selected_attn_paged"], B=1, N=1, Hq=4, Hkv=1, top_k=top_k).values()) == SHAPE
    assert binding.paged_workspace_bytes(1, 1, 4, 1, 128, 1, top_k) == 0
    assert binding.paged_workspace_bytes(1, 1, 4, 1, 128, 1, 1 << 30) > 0


@pytest.mark.parametrize("top_k", [(1 << 30) + 1, (1 << 31) - 1])
def test_selection_refuses_lists_past_what_is_counted(lib, top_k):
    """Threads step past the end of a list in 32 bits."""
    assert lib.da_select_pages(*dict(ARGS["da_select_pages"], top_k=top_k).values()) == SHAPE


def test_append_to_refuses_as_append_does(lib):
    """The call with lengths to append to: the same checks, and its own argument's."""
    for fn, status, names, value in REFUSED:
        for name in names if fn == "da_pages_append" else ():
            *args, stream = dict(ARGS[fn], **{name: value}).values()
            for lens in (None, PTR):
                assert lib.da_pages_append_to(*args, lens, stream) == status, (name, value)
    *args, stream = ARGS["da_pages_append"].values()
    assert lib.da_pages_append_to(*args, PTR + 2, stream) == ALIGN


@pytest.mark.parametrize("fn", sorted(ARGS))
def test_the_arguments_above_are_good(lib, fn):
    """(so that each refusal is that of the one argument that was changed)"""
    if torch.cuda.is_available():
        pytest.skip("the pointers are made up: nothing may be launched")
    import threading
    got = []  # (in a thread of its own: the last HIP error is kept per thread)
    t = threading.Thread(target=lambda: got.append(getattr(lib, fn)(*ARGS[fn].values())))
    t.start()
    t.join()
    assert got[0] in (HIP, UNSUP)


def test_workspaces_that_are_too_small(lib):
    for fn, more, need in (("tree_attn_paged", dict(M=5000, max_len=300000), binding.paged_workspace_bytes(2, 3, 8, 2, 128, 300000)),
                           ("selected_attn_paged", dict(top_k=100), binding.paged_workspace_bytes(2, 3, 8, 2, 128, 1, 100))):
        a = dict(ARGS[fn], **{**more, "size": need - 1})  # (keeps the order of the arguments)
        assert need > 0 and getattr(lib, fn)(*a.values()) == WORKSPACE
        a["size"], a["ws"] = need, None
        assert getattr(lib, fn)(*a.values()) == WORKSPACE
    need = lib.da_select_pages_workspace_bytes(2, 3, 2, 1025 * 64)
    a = dict(ARGS["da_select_pages"], M=1025, max_len=1025 * 64, size=need - 1)
    assert need == 2 * 3 * 2 * 1025 * 4 and lib.da_select_pages(*a.values()) == WORKSPACE
    a["size"], a["ws"] = need, None
    assert lib.da_select_pages(*a.values()) == WORKSPACE
    assert lib.da_select_pages_workspace_bytes(2, 3, 2, 1025 * 64 - 1) == 0
    # few pages: no rows are cut, nothing is needed
    assert binding.paged_workspace_bytes(2, 3, 8, 2, 128, 512) == binding.paged_workspace_bytes(2, 3, 8, 2, 128, 1, 4) == 0


@pytest.mark.parametrize("B,N,Hq,Hkv,d", [(1, 1, 32, 8, 128), (64, 1, 32, 8, 128), (3, 64, 64, 8, 128), (1, 1, 8, 1, 64),
                                          (500, 7, 28, 4, 128), (20000, 1, 8, 2, 64)])
def test_workspaces_of_any_length_are_bounded(lib, B, N, Hq, Hkv, d):
    """At most two tiles of partial results for each workgroup that runs at once, and a count per sequence."""
    most = 768 * 2 * 256 * (d + 2) * 4 + 4 * B + 512
    for n in (1, 64, 100, 1000, 10 ** 4, 10 ** 5, 10 ** 6):
        assert 0 <= binding.paged_workspace_bytes(B, N, Hq, Hkv, d, n) <= most
    for k in (1, 8, 64, 500):
        assert 0 <= binding.paged_workspace_bytes(B, N, Hq, Hkv, d, 1, k) <= most
    assert binding.paged_workspace_bytes(0, N, Hq, Hkv, d, 64) == 0
    assert binding.paged_workspace_bytes(B, N, Hq, Hkv, 80, 64) == 0
    assert binding.paged_workspace_bytes(50000, 1, 64, 64, 64, 1 << 30) == 0  # more pages than are counted


def test_list_entries(lib):
    for N, top_k, bq in ((64, 3, 64), (65, 3, 64), (1000, 4, 64), (5000, 7, 256), (4096, 1, 128)):
        R = bq // 64
        want = sum(min(top_k, j * R) for j in range(-(-N // bq)))
        assert lib.da_select_blocks_entries(3, N, 2, top_k, bq) == 6 * want
    assert lib.da_select_blocks_entries(1, 100, 1, 4, 48) == 0
    assert lib.da_key_summary_blocks(1000, 3) == 1000 // 64 + 3


def test_binding_refuses_host_tensors():
    i = torch.zeros(4, dtype=torch.int32)
    table = torch.zeros((4, 4), dtype=torch.int32)
    pages = torch.zeros((4, 2, 64, 64), dtype=torch.bfloat16)
    q = torch.zeros((4, 4, 64), dtype=torch.bfloat16)
    codes, scales = torch.zeros((4, 2, 64), dtype=torch.int8), torch.zeros((4, 2))
    calls = [
        lambda: binding.pages_fork(table, i, i, i, i),
        lambda: binding.pages_resize(pages, pages, table, i, i, i),
        lambda: binding.pages_append(q, q, pages, pages, table, i),
        lambda: binding.pages_compact(pages, pages, table, i, i, i, i, i, i),
        lambda: binding.tree_attn_paged(q, pages, pages, table, i),
        lambda: binding.selected_attn_paged(q, pages, pages, table, i, i),
        lambda: binding.key_summary(q),
        lambda: binding.page_summary(pages, table, i, codes, scales),
        lambda: binding.select_blocks(q, codes, scales, top_k=2, block_q=64),
        lambda: binding.select_pages(q, codes, scales, table, i, top_k=2),
    ]
    for call in calls:
        with pytest.raises(ValueError):
            call()


def test_tree_mask():
    """Bits of a row: itself and its ancestors, in words of 64."""
    m = binding.tree_mask([[-1, 0, 0, 1], [], [-1, -1]])
    assert m.tolist() == [[1], [3], [5], [11], [1], [2]]
    chain = binding.tree_mask([list(range(-1, 129))])
    assert chain.shape == (130, 3)
    for i in (0, 63, 64, 129):
        x = sum((int(w) & (2 ** 64 - 1)) << 64 * k for k, w in enumerate(chain[i]))
        assert x == (1 << i + 1) - 1
    for bad in ([[0]], [[-1, 1]], [[-2]]):
        with pytest.raises(ValueError):
            binding.tree_mask(bad)


def test_kernel_dma_has_its_wait_states():
    """The attention's LDS DMA is issued from the same asm as the prefill kernels': the wait states the
    hardware needs before it (see test_isa_hazards) have to be there in this file's assembly too."""
    import shutil
    import subprocess
    import tempfile

    from test_isa_hazards import dma_hazards
    from paper_2505_11254_amd import build
    cc = build.hipcc()
    if not (os.path.isabs(cc) and os.path.exists(cc)) and shutil.which(cc) is None:
        pytest.skip("hipcc not available")
    flags = [f for f in build.compile_flags() if f not in ("-shared", "-fPIC")]
    src = os.path.join(build.CSRC, "da_paged_attn.hip")
    with tempfile.TemporaryDirectory() as td:
        out = os.path.join(td, "k.s")
        subprocess.run([cc] + flags + ["--cuda-device-only", "-S", src, "-o", out], check=True, capture_output=True)
        text = open(out).read().splitlines()
    assert any("buffer_load_dwordx4" in t and t.rstrip().endswith("lds") for t in text)
    assert dma_hazards(text) == []
