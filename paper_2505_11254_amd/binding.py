"""ctypes binding of ``libdelta_attn.so`` (C ABI in ``include/delta_attn.h``).

Argument marshalling only: every step of the attention path runs in the HIP
kernels of the library.  torch supplies device memory and the stream.  There
is no fallback: a missing library or a non-gfx950 device raises.

Tensors are token-major bf16 on the GPU: q [T, Hq, d], k/v [T, Hkv, d].
A fixed-length batch passes ``B`` (T = B * N); a ragged batch passes
``cu_seqlens`` (int32, B + 1 entries, on the GPU) and ``max_seqlen``.
"""
from __future__ import annotations

import ctypes
import functools
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdelta_attn.so")

STATUS = {0: "DA_OK", 1: "DA_ERR_NULL", 2: "DA_ERR_SHAPE", 3: "DA_ERR_PARAM",
          4: "DA_ERR_UNSUPPORTED", 5: "DA_ERR_ALIGN", 6: "DA_ERR_WORKSPACE", 7: "DA_ERR_HIP"}

# C entry points and their argument types: p = pointer, i = int, z = size_t, u = unsigned,
# f = float
SIGNATURES = {
    "delta_attn_prefill": "ppppiiiiiiiipzp",
    "delta_attn_prefill_varlen": "pppppiiiiiiiipzp",
    "delta_attn_prefill_steps": "pppppiiiiiiiipzpu",
    "delta_attn_prefill_correction": "pppppiiiiiiiiifffpzp",
    "sparse_attn_prefill": "ppppiiiiiiip",
    "sparse_attn_prefill_varlen": "pppppiiiiiiip",
    "dense_causal_attn_prefill": "ppppiiiiip",
    "dense_causal_attn_prefill_varlen": "pppppiiiiip",
    "blocksparse_attn_prefill": "pppppiiiiiippp",
    "delta_attn_prefill_blocksparse": "pppppiiiiiippipzpu",
    "da_check_inputs": "piiiipplpp",
    "delta_attn_prefill_noalloc": "pppppiiiiiiiip",
    "da_pages_fork": "pppiiippipp",
    "da_pages_resize": "ppiiipppiiippipp",
    "da_pages_append": "pplppiiippiiippiip",
    "da_pages_append_to": "pplppiiippiiippiipp",
    "da_pages_compact": "ppiiipppiiippplpipp",
    "tree_attn_paged": "pppppppiiippiiiiiipipzp",
    "selected_attn_paged": "pppppppiiippiiiiipipzp",
    "da_key_summary": "ppiiiippp",
    "da_page_summary": "piippiiippiippp",
    "da_select_blocks": "ppppiiiiiiiiippp",
    "da_select_pages": "pppppiiippiiiiiiiiippzp",
}


class Plan(ctypes.Structure):
    """da_plan of include/delta_attn.h: how the library tiles a problem."""
    _fields_ = [(n, ctypes.c_int) for n in ("fused", "sparse_heads", "rows_heads", "key_chunks",
                                            "chunk_keys", "key_tile", "rows_per_wave",
                                            "waves_per_block", "sparse_slab_rows")]

    def as_dict(self):
        return {n: int(getattr(self, n)) for n, _ in self._fields_}


class Workgroups(ctypes.Structure):
    """da_workgroups of include/delta_attn.h: the workgroups the launches take."""
    _fields_ = [(n, ctypes.c_int) for n in ("sparse_waves", "sparse_heads", "rows_waves",
                                            "rows_heads", "together", "base_waves", "base_heads",
                                            "dense_waves", "dense_heads")]

    as_dict = Plan.as_dict


class DeltaAttnError(RuntimeError):
    def __init__(self, fn, status, hip_error=0):
        self.status = status
        self.hip_error = hip_error
        msg = f"{fn} returned {STATUS.get(status, status)}"
        if status == 7:
            msg += f" (hipError_t {hip_error})"
        super().__init__(msg)


_lib = None


# DA_ABI_VERSION of include/delta_attn.h that this binding's structures follow.
ABI_VERSION = 2


def load_library(path: str = LIB_PATH, check_abi: bool = True):
    """Load the HIP library (raises if it has not been built, or, with check_abi,
    if it was built against another ABI version than this binding's)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with __graft_entry__.build() "
                           "(hipcc for gfx950); there is no fallback implementation")
    lib = ctypes.CDLL(path)
    codes = {"p": ctypes.c_void_p, "i": ctypes.c_int, "z": ctypes.c_size_t,
             "u": ctypes.c_uint, "f": ctypes.c_float, "l": ctypes.c_int64}
    for name, sig in SIGNATURES.items():
        f = getattr(lib, name)
        f.argtypes = [codes[c] for c in sig]
        f.restype = ctypes.c_int
    lib.da_workspace_bytes.argtypes = [ctypes.c_int] * 6
    lib.da_workspace_bytes.restype = ctypes.c_size_t
    lib.da_workspace_bytes_correction.argtypes = [ctypes.c_int] * 7
    lib.da_workspace_bytes_correction.restype = ctypes.c_size_t
    lib.da_paged_workspace_bytes.argtypes = [ctypes.c_int] * 7
    lib.da_paged_workspace_bytes.restype = ctypes.c_size_t
    lib.da_select_pages_workspace_bytes.argtypes = [ctypes.c_int] * 4
    lib.da_select_pages_workspace_bytes.restype = ctypes.c_size_t
    lib.da_select_blocks_entries.argtypes = [ctypes.c_int] * 5
    lib.da_select_blocks_entries.restype = ctypes.c_int64
    lib.da_key_summary_blocks.argtypes = [ctypes.c_int64, ctypes.c_int]
    lib.da_key_summary_blocks.restype = ctypes.c_int64
    lib.da_fused_supported.argtypes = [ctypes.c_int] * 3
    lib.da_fused_supported.restype = ctypes.c_int
    lib.da_fused_supported_blocksparse.argtypes = [ctypes.c_int] * 4
    lib.da_fused_supported_blocksparse.restype = ctypes.c_int
    lib.da_status_string.argtypes = [ctypes.c_int]
    lib.da_status_string.restype = ctypes.c_char_p
    lib.da_last_hip_error.argtypes = []
    lib.da_last_hip_error.restype = ctypes.c_int
    lib.da_abi_version.argtypes = []
    lib.da_abi_version.restype = ctypes.c_int
    lib.da_launch_plan.argtypes = [ctypes.c_int] * 7 + [ctypes.POINTER(Plan)]
    lib.da_launch_plan.restype = ctypes.c_int
    lib.da_launch_workgroups.argtypes = [ctypes.c_int] * 11 + [ctypes.POINTER(Workgroups)]
    lib.da_launch_workgroups.restype = ctypes.c_int
    if check_abi and lib.da_abi_version() != ABI_VERSION:
        raise RuntimeError(f"{path} has ABI version {lib.da_abi_version()}, this binding needs "
                           f"{ABI_VERSION}: rebuild it with __graft_entry__.build()")
    _lib = lib
    return lib


def _call(name, *args):
    lib = load_library()
    rc = getattr(lib, name)(*args)
    if rc != 0:
        raise DeltaAttnError(name, rc, lib.da_last_hip_error())


def _ptr(t):
    return t.data_ptr() if t is not None else None


def _stream(device, stream):
    s = stream if stream is not None else torch.cuda.current_stream(device)
    return s.cuda_stream


def _on_device(name, t, dev, dtype):
    """t must be a contiguous tensor of `dtype` on the GPU `dev` (the kernels
    dereference its pointer on that device)."""
    if not getattr(t, "is_cuda", False) or t.device != dev:
        raise ValueError(f"{name} must be on {dev} (got {t.device})")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype} (got {t.dtype})")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _span(t):
    n = t.numel() * t.element_size()
    return t.data_ptr(), t.data_ptr() + n


def _check(q, k, v, out=None, cu_seqlens=None, workspace=None, block_ptr=None,
           block_idx=None):
    """Everything the C ABI takes on trust about the tensors behind its
    pointers: device, dtype, layout, matching shapes and no aliasing of the
    output with an input.  Raises ValueError before anything is launched."""
    dev = q.device
    for name, t in (("q", q), ("k", k), ("v", v)):
        _on_device(name, t, dev, torch.bfloat16)
        if t.dim() != 3:
            raise ValueError(f"{name} must be [T, H, d]")
    if tuple(k.shape) != tuple(v.shape):
        raise ValueError(f"k and v must have the same shape (got {tuple(k.shape)} and "
                         f"{tuple(v.shape)})")
    if k.shape[0] != q.shape[0] or k.shape[2] != q.shape[2]:
        raise ValueError("k and v must be [T, Hkv, d] with the T and d of q")
    if cu_seqlens is not None:
        _on_device("cu_seqlens", cu_seqlens, dev, torch.int32)
        if cu_seqlens.dim() != 1 or cu_seqlens.numel() < 2:
            raise ValueError("cu_seqlens must be 1-D with B + 1 >= 2 entries")
    _check_rest(q, k, v, out, workspace, block_ptr, block_idx)


def _check_rest(q, k, v, out=None, workspace=None, block_ptr=None, block_idx=None):
    """The part of _check beyond the tensors that _shapes has checked."""
    dev = q.device
    if out is not None:
        _on_device("out", out, dev, torch.bfloat16)
        if tuple(out.shape) != tuple(q.shape):
            raise ValueError(f"out must have the shape of q {tuple(q.shape)}")
        o0, o1 = _span(out)
        for name, t in (("q", q), ("k", k), ("v", v)):
            t0, t1 = _span(t)
            if o0 < t1 and t0 < o1:
                raise ValueError(f"out must not overlap {name}")
    if workspace is not None:
        _on_device("workspace", workspace, dev, None)
    for name, t in (("block_ptr", block_ptr), ("block_idx", block_idx)):
        if t is not None:
            _on_device(name, t, dev, torch.int32)


def _shapes(q, k, v, B, cu_seqlens, max_seqlen):
    _check(q, k, v, cu_seqlens=cu_seqlens)
    T, Hq, d = q.shape
    Hkv = k.shape[1]
    if cu_seqlens is None:
        B = 1 if B is None else int(B)
        if B < 1 or T % B != 0:
            raise ValueError("T must be a multiple of B for a fixed-length batch")
        return B, T // B, Hq, Hkv, d
    if max_seqlen is None:
        raise ValueError("max_seqlen is required with cu_seqlens")
    return cu_seqlens.numel() - 1, int(max_seqlen), Hq, Hkv, d


def workspace_bytes(B, max_seqlen, Hq, Hkv, d, gamma) -> int:
    return int(load_library().da_workspace_bytes(B, max_seqlen, Hq, Hkv, d, gamma))


def launch_plan(B, max_seqlen, Hq, Hkv, d, gamma, block_q=0) -> dict:
    """The library's tiling of a problem in full-size workgroups (da_launch_plan; host only)."""
    p = Plan()
    lib = load_library()
    rc = lib.da_launch_plan(B, max_seqlen, Hq, Hkv, d, gamma, block_q, ctypes.byref(p))
    if rc != 0:
        raise DeltaAttnError("da_launch_plan", rc)
    return p.as_dict()


def launch_workgroups(B, max_seqlen, Hq, Hkv, d, gamma, *, window=1, n_sink=0, block_q=0, mode=0,
                      packed=False) -> dict:
    """The workgroups that the launches of a problem take (da_launch_workgroups; host only)."""
    w = Workgroups()
    rc = load_library().da_launch_workgroups(B, max_seqlen, int(packed), Hq, Hkv, d, window, n_sink,
                                             gamma, block_q, mode, ctypes.byref(w))
    if rc != 0:
        raise DeltaAttnError("da_launch_workgroups", rc)
    return w.as_dict()


def fused_supported(Hq, Hkv, gamma) -> bool:
    """Whether delta_attn_prefill takes the fused schedule for these sizes."""
    return bool(load_library().da_fused_supported(Hq, Hkv, gamma))


def delta_attn_prefill(q, k, v, *, window, n_sink, gamma, B=None, cu_seqlens=None,
                       max_seqlen=None, out=None, workspace=None, stream=None):
    """Delta Attention prefill (Algorithm 1); returns ``out`` [T, Hq, d] bf16."""
    B_, N, Hq, Hkv, d = _shapes(q, k, v, B, cu_seqlens, max_seqlen)
    if out is None:
        out = torch.empty_like(q)
    if workspace is None:
        nbytes = workspace_bytes(B_, N, Hq, Hkv, d, gamma)
        workspace = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=q.device)
    _check_rest(q, k, v, out, workspace)
    wsz = workspace.numel() * workspace.element_size()
    st = _stream(q.device, stream)
    if cu_seqlens is None:
        _call("delta_attn_prefill", _ptr(q), _ptr(k), _ptr(v), _ptr(out), B_, Hq, Hkv, N, d,
              window, n_sink, gamma, _ptr(workspace), wsz, st)
    else:
        _call("delta_attn_prefill_varlen", _ptr(q), _ptr(k), _ptr(v), _ptr(out),
              _ptr(cu_seqlens), B_, N, Hq, Hkv, d, window, n_sink, gamma, _ptr(workspace),
              wsz, st)
    return out


def delta_attn_prefill_noalloc(q, k, v, *, window, n_sink, gamma, B=None, cu_seqlens=None,
                               max_seqlen=None, out=None, stream=None):
    """Delta Attention prefill whose workspace is the library's static device
    array (delta_attn_prefill_noalloc): the call allocates nothing on the
    device; pass ``out`` to allocate nothing here either."""
    B_, N, Hq, Hkv, d = _shapes(q, k, v, B, cu_seqlens, max_seqlen)
    if out is None:
        out = torch.empty_like(q)
    _check_rest(q, k, v, out)
    _call("delta_attn_prefill_noalloc", _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(cu_seqlens),
          B_, N, Hq, Hkv, d, window, n_sink, gamma, _stream(q.device, stream))
    return out


STEP_SPARSE, STEP_DENSE_ROWS, STEP_CORRECT, STEP_ALL, STEP_FUSED = 1, 2, 4, 7, 8
CORR_DELTA, CORR_RECOMPUTE, CORR_INTERP, CORR_EMA, CORR_ABG = 0, 1, 2, 3, 4


def delta_attn_prefill_correction(q, k, v, *, window, n_sink, gamma, mode,
                                  params=(0.0, 0.0, 0.0), B=None, cu_seqlens=None,
                                  max_seqlen=None, out=None, workspace=None, stream=None):
    """Algorithm 1 with the step-5 correction chosen by ``mode`` (CORR_*)."""
    B_, N, Hq, Hkv, d = _shapes(q, k, v, B, cu_seqlens, max_seqlen)
    if out is None:
        out = torch.empty_like(q)
    if workspace is None:
        nbytes = int(load_library().da_workspace_bytes_correction(B_, N, Hq, Hkv, d, gamma, mode))
        workspace = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=q.device)
    _check_rest(q, k, v, out, workspace)
    wsz = workspace.numel() * workspace.element_size()
    p = list(params) + [0.0] * (3 - len(params))
    _call("delta_attn_prefill_correction", _ptr(q), _ptr(k), _ptr(v), _ptr(out),
          _ptr(cu_seqlens), B_, N, Hq, Hkv, d, window, n_sink, gamma, mode, float(p[0]),
          float(p[1]), float(p[2]), _ptr(workspace), wsz, _stream(q.device, stream))
    return out


def delta_attn_prefill_steps(q, k, v, out, workspace, steps, *, window, n_sink, gamma, B=None,
                             cu_seqlens=None, max_seqlen=None, stream=None):
    """Run the given steps of Algorithm 1 (bit mask of STEP_*) on existing buffers."""
    B_, N, Hq, Hkv, d = _shapes(q, k, v, B, cu_seqlens, max_seqlen)
    _check_rest(q, k, v, out, workspace)
    wsz = workspace.numel() * workspace.element_size()
    _call("delta_attn_prefill_steps", _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(cu_seqlens),
          B_, N, Hq, Hkv, d, window, n_sink, gamma, _ptr(workspace), wsz,
          _stream(q.device, stream), steps)
    return out


def sparse_attn_prefill(q, k, v, *, window, n_sink, B=None, cu_seqlens=None, max_seqlen=None,
                        out=None, stream=None):
    """Sink + sliding-window attention for every row (the f* of the paper)."""
    B_, N, Hq, Hkv, d = _shapes(q, k, v, B, cu_seqlens, max_seqlen)
    if out is None:
        out = torch.empty_like(q)
    _check_rest(q, k, v, out)
    st = _stream(q.device, stream)
    if cu_seqlens is None:
        _call("sparse_attn_prefill", _ptr(q), _ptr(k), _ptr(v), _ptr(out), B_, Hq, Hkv, N, d,
              window, n_sink, st)
    else:
        _call("sparse_attn_prefill_varlen", _ptr(q), _ptr(k), _ptr(v), _ptr(out),
              _ptr(cu_seqlens), B_, N, Hq, Hkv, d, window, n_sink, st)
    return out


def dense_causal_attn_prefill(q, k, v, *, B=None, cu_seqlens=None, max_seqlen=None, out=None,
                              stream=None):
    """Dense causal attention for every row (the quadratic baseline f)."""
    B_, N, Hq, Hkv, d = _shapes(q, k, v, B, cu_seqlens, max_seqlen)
    if out is None:
        out = torch.empty_like(q)
    _check_rest(q, k, v, out)
    st = _stream(q.device, stream)
    if cu_seqlens is None:
        _call("dense_causal_attn_prefill", _ptr(q), _ptr(k), _ptr(v), _ptr(out), B_, Hq, Hkv,
              N, d, st)
    else:
        _call("dense_causal_attn_prefill_varlen", _ptr(q), _ptr(k), _ptr(v), _ptr(out),
              _ptr(cu_seqlens), B_, N, Hq, Hkv, d, st)
    return out


def fused_supported_blocksparse(Hq, Hkv, gamma, block_q) -> bool:
    """Whether the key-block-list path takes the fused schedule for these sizes."""
    return bool(load_library().da_fused_supported_blocksparse(Hq, Hkv, gamma, block_q))


def _blocks(block_ptr, block_idx, B, Hkv, N, block_q):
    """Pointers of the key-block lists after checking their device, dtype and
    that block_ptr holds [B, Hkv, ceil(N / block_q) + 1] offsets."""
    if block_q not in (64, 128, 256):
        raise ValueError("block_q must be 64, 128 or 256")
    nqb = -(-N // block_q)
    if block_ptr.numel() != B * Hkv * (nqb + 1):
        raise ValueError(f"block_ptr must hold B * Hkv * (ceil(N / block_q) + 1) = "
                         f"{B * Hkv * (nqb + 1)} offsets (got {block_ptr.numel()})")
    return _ptr(block_ptr), _ptr(block_idx)


def blocksparse_attn_prefill(q, k, v, *, block_q, block_ptr, block_idx, B=None,
                             cu_seqlens=None, max_seqlen=None, out=None, stream=None):
    """Sparse attention whose key sets come from key-block lists, for every row."""
    B_, N, Hq, Hkv, d = _shapes(q, k, v, B, cu_seqlens, max_seqlen)
    if out is None:
        out = torch.empty_like(q)
    _check_rest(q, k, v, out, block_ptr=block_ptr, block_idx=block_idx)
    _call("blocksparse_attn_prefill", _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(cu_seqlens),
          B_, N, Hq, Hkv, d, block_q, *_blocks(block_ptr, block_idx, B_, Hkv, N, block_q),
          _stream(q.device, stream))
    return out


def delta_attn_prefill_blocksparse(q, k, v, *, block_q, block_ptr, block_idx, gamma, B=None,
                                   cu_seqlens=None, max_seqlen=None, out=None, workspace=None,
                                   stream=None, steps=0):
    """Delta Attention with f* from key-block lists; ``steps`` 0 runs the whole path."""
    B_, N, Hq, Hkv, d = _shapes(q, k, v, B, cu_seqlens, max_seqlen)
    if out is None:
        out = torch.empty_like(q)
    if workspace is None:
        nbytes = workspace_bytes(B_, N, Hq, Hkv, d, gamma)
        workspace = torch.empty(max(nbytes, 1), dtype=torch.uint8, device=q.device)
    _check_rest(q, k, v, out, workspace, block_ptr, block_idx)
    wsz = workspace.numel() * workspace.element_size()
    _call("delta_attn_prefill_blocksparse", _ptr(q), _ptr(k), _ptr(v), _ptr(out),
          _ptr(cu_seqlens), B_, N, Hq, Hkv, d, block_q,
          *_blocks(block_ptr, block_idx, B_, Hkv, N, block_q), gamma,
          _ptr(workspace), wsz, _stream(q.device, stream), steps)
    return out


def check_inputs(*, max_seqlen, B=None, cu_seqlens=None, Hkv=None, block_q=None,
                 block_ptr=None, block_idx=None, stream=None):
    """Count violations of the rules cu_seqlens and key-block lists must follow
    (see da_check_inputs); synchronises the stream.  Returns the count."""
    import torch as _t
    dev = (cu_seqlens if cu_seqlens is not None else block_ptr).device
    if B is None:
        B = cu_seqlens.numel() - 1
    result = _t.zeros(1, dtype=_t.int32, device=dev)
    nnz = block_idx.numel() if block_idx is not None else 0
    lib = load_library()
    rc = lib.da_check_inputs(_ptr(cu_seqlens), B, max_seqlen, Hkv or 0, block_q or 0,
                             _ptr(block_ptr), _ptr(block_idx), nnz, _ptr(result),
                             _stream(dev, stream))
    if rc not in (0, 3):
        raise DeltaAttnError("da_check_inputs", rc, lib.da_last_hip_error())
    return int(result.item())



# ---------------------------------------------------------------------------------------------
# Serving after the prefill: the paged cache (see include/delta_attn.h for its layout and rules),
# the attention over it and the selection of key blocks.
#
# k_pages / v_pages are [P, Hkv, 64, d] bf16, or [layers, P, Hkv, 64, d] where a call moves the
# tokens of all layers; table int32 [S, M], lens int32 [S], refs int32 [P].  A batch of new tokens
# is packed like a prefill's: B sequences of T / B rows, or cu_seqlens and max_seqlen; sequence b
# is slot slots[b] (default b).  Calls run on the device of their tensors, whichever is current.

PAGE_TOKENS = 64

_entries = {}  # the library's entry points that have been called


class _On:
    """The device of a call and its stream: sets the device where another is current, and takes
    new tensors from that stream's memory."""
    __slots__ = ("dev", "raw", "stream", "other")

    def __init__(self, dev, stream):
        if dev.type != "cuda":
            raise ValueError(f"tensors must be on a GPU (got {dev})")
        self.dev = dev
        self.stream = stream
        self.raw = torch._C._cuda_getCurrentRawStream(dev.index) if stream is None else stream.cuda_stream
        self.other = dev.index != torch._C._cuda_getDevice()

    def call(self, name, *args):
        fn = _entries.get(name)
        if fn is None:
            fn = _entries[name] = getattr(load_library(), name)
        if self.other:
            with torch.cuda.device(self.dev):
                rc = fn(*args, self.raw)
        else:
            rc = fn(*args, self.raw)
        if rc != 0:
            raise DeltaAttnError(name, rc, load_library().da_last_hip_error())

    def empty(self, shape, dtype):
        if self.stream is None:
            return torch.empty(shape, dtype=dtype, device=self.dev)
        with torch.cuda.stream(self.stream):
            return torch.empty(shape, dtype=dtype, device=self.dev)

    def full(self, n, value, dtype):
        if self.stream is None:
            return torch.full((n,), value, dtype=dtype, device=self.dev)
        with torch.cuda.stream(self.stream):
            return torch.full((n,), value, dtype=dtype, device=self.dev)

    def like(self, t, shape=None):
        """A new tensor of t's type (and shape); t lies on the device (cheaper than `empty`)."""
        if self.stream is None:
            return torch.empty_like(t) if shape is None else t.new_empty(shape)
        with torch.cuda.stream(self.stream):
            return torch.empty_like(t) if shape is None else t.new_empty(shape)

    def workspace(self, given, nbytes):
        """(tensor, address, size) of the caller's workspace, or of one that lasts for this call."""
        if given is None:
            if not nbytes:
                return None, None, 0
            given = self.empty(nbytes, torch.uint8)
            return given, given.data_ptr(), nbytes
        _on_device("workspace", given, self.dev, None)
        return given, given.data_ptr(), given.numel() * given.element_size()


def _ints(name, t, dev, shape=None):
    """t is a contiguous int32 tensor on `dev`, of `shape` if given."""
    if t.dtype is not torch.int32 or t.device != dev or not t.is_contiguous():
        _on_device(name, t, dev, torch.int32)
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)} (got {list(t.shape)})")


def _table(table, lens, dev):
    _ints("table", table, dev)
    shape = table.shape
    if len(shape) != 2:
        raise ValueError("table must be [S, M]")
    _ints("lens", lens, dev, shape[:1])
    return shape


def _halves(name, t, dev):
    """t is a contiguous bf16 tensor on `dev`."""
    if t.dtype is not torch.bfloat16 or t.device != dev or not t.is_contiguous():
        _on_device(name, t, dev, torch.bfloat16)


def _pages(k_pages, v_pages, layered=False):
    """(dev, layers, P, Hkv, d) of a cache's pages."""
    dev, shape = k_pages.device, k_pages.shape
    _halves("k_pages", k_pages, dev)
    if v_pages is not None:
        _halves("v_pages", v_pages, dev)
        if v_pages.shape != shape:
            raise ValueError("k_pages and v_pages must have the same shape")
    n = len(shape)
    if n != 4 and not (layered and n == 5):
        raise ValueError("pages must be [P, Hkv, 64, d]" + (" or [layers, P, Hkv, 64, d]" if layered else ""))
    if shape[-2] != PAGE_TOKENS:
        raise ValueError(f"pages must hold {PAGE_TOKENS} tokens")
    return dev, (shape[0] if n == 5 else 1), shape[-4], shape[-3], shape[-1]


def _slots(slots, B, S, dev):
    if slots is None:
        if B > S:
            raise ValueError(f"{B} sequences without slots, but the table has {S}")
        return None
    _ints("slots", slots, dev, (B,))
    return slots.data_ptr()


def _new_rows(T, B, cu_seqlens, max_seqlen, dev):
    """(B, rows per sequence, at most) of a batch of T new rows."""
    if cu_seqlens is None:
        B = 1 if B is None else int(B)
        if B < 1 or T < 1 or T % B != 0:
            raise ValueError("the number of rows must be a multiple of B for a fixed-length batch")
        return B, T // B
    _ints("cu_seqlens", cu_seqlens, dev)
    if cu_seqlens.dim() != 1 or cu_seqlens.shape[0] < 2:
        raise ValueError("cu_seqlens must be 1-D with B + 1 >= 2 entries")
    if max_seqlen is None:
        raise ValueError("max_seqlen is required with cu_seqlens")
    return cu_seqlens.shape[0] - 1, int(max_seqlen)


def _requests(result, shape, ints, on):
    if result is None:
        return on.like(ints, shape)
    _ints("result", result, on.dev, shape)
    return result


def pages_fork(table, lens, refs, src, dst, *, result=None, stream=None):
    """Slots ``dst`` become copies of slots ``src`` that share their pages.  Returns ``result``
    int32 [n]: the lengths, -1 where a request was refused (da_pages_fork)."""
    on = _On(table.device, stream)
    S, M = _table(table, lens, on.dev)
    _ints("refs", refs, on.dev)
    n = src.numel()
    _ints("src", src, on.dev, (n,))
    _ints("dst", dst, on.dev, (n,))
    result = _requests(result, (n,), src, on)
    on.call("da_pages_fork", _ptr(table), _ptr(lens), _ptr(refs), S, M, refs.numel(), _ptr(src), _ptr(dst), n,
            _ptr(result))
    return result


def pages_resize(k_pages, v_pages, table, lens, refs, slots, new_lens=None, *, result=None, stream=None):
    """Slots get the lengths ``new_lens`` (None: 0, they are freed): pages are given back, taken,
    and copied where a shared one will be written.  Returns ``result`` int32 [n, 4], whose first
    column is the new length or -1 where a request was refused (da_pages_resize)."""
    dev, layers, P, Hkv, d = _pages(k_pages, v_pages, layered=True)
    on = _On(dev, stream)
    S, M = _table(table, lens, dev)
    _ints("refs", refs, dev, (P,))
    n = slots.numel()
    _ints("slots", slots, dev, (n,))
    if new_lens is not None:
        _ints("new_lens", new_lens, dev, (n,))
    result = _requests(result, (n, 4), slots, on)
    on.call("da_pages_resize", _ptr(k_pages), _ptr(v_pages), layers, Hkv, d, _ptr(table), _ptr(lens), _ptr(refs), S, M,
            P, _ptr(slots), _ptr(new_lens), n, _ptr(result))
    return result


def pages_append(k, v, k_pages, v_pages, table, lens, *, slots=None, B=None, cu_seqlens=None, max_seqlen=None,
                 new_lens=None, stream=None):
    """Writes the keys and values of new tokens, [T, Hkv, d] or [layers, T, Hkv, d], as the last
    ones of their sequences, which pages_resize has made room for (da_pages_append).  With
    ``new_lens`` [B], the lengths asked of pages_resize, a sequence that has another length stays as
    it is: a growth that was refused leaves old tokens where the new ones belong
    (da_pages_append_to).  A caller that does not look at pages_resize's result before passes it."""
    dev, layers, P, Hkv, d = _pages(k_pages, v_pages, layered=True)
    on = _On(dev, stream)
    S, M = _table(table, lens, dev)
    _halves("k", k, dev)
    _halves("v", v, dev)
    if k.dim() != k_pages.dim() - 1 or k.shape[-2:] != (Hkv, d) or (k.dim() == 4 and k.shape[0] != layers):
        raise ValueError("k must be [T, Hkv, d] for pages of one layer, [layers, T, Hkv, d] for more")
    if k.shape != v.shape:
        raise ValueError("k and v must have the same shape")
    T = k.shape[-3]
    B, N = _new_rows(T, B, cu_seqlens, max_seqlen, dev)
    args = (_ptr(k), _ptr(v), T, _ptr(k_pages), _ptr(v_pages), layers, Hkv, d, _ptr(table), _ptr(lens), S, M, P,
            _slots(slots, B, S, dev), _ptr(cu_seqlens), B, N)
    if new_lens is None:
        on.call("da_pages_append", *args)
    else:
        _ints("new_lens", new_lens, dev, (B,))
        on.call("da_pages_append_to", *args, _ptr(new_lens))


def pages_compact(k_pages, v_pages, table, lens, refs, slots, start, keep, cu_keep, *, result=None, stream=None):
    """Of the tokens of slots[i] from start[i] on, those at start[i] + keep[cu_keep[i]:cu_keep[i + 1]]
    move up to start[i]; the rest is dropped.  Returns ``result`` int32 [n, 4], whose first column is
    the number kept or -1 where a request was refused (da_pages_compact)."""
    dev, layers, P, Hkv, d = _pages(k_pages, v_pages, layered=True)
    on = _On(dev, stream)
    S, M = _table(table, lens, dev)
    _ints("refs", refs, dev, (P,))
    n = slots.numel()
    _ints("slots", slots, dev, (n,))
    _ints("start", start, dev, (n,))
    _ints("keep", keep, dev, (keep.numel(),))
    _ints("cu_keep", cu_keep, dev, (n + 1,))
    result = _requests(result, (n, 4), slots, on)
    if not keep.numel():  # (an empty tensor has no address; no place is read)
        keep = cu_keep
        n_keep = 0
    else:
        n_keep = keep.numel()
    on.call("da_pages_compact", _ptr(k_pages), _ptr(v_pages), layers, Hkv, d, _ptr(table), _ptr(lens), _ptr(refs), S, M,
            P, _ptr(slots), _ptr(start), _ptr(keep), n_keep, _ptr(cu_keep), n, _ptr(result))
    return result


def _queries(q, k_pages, v_pages, out, lse, Hkv, d, on):
    _halves("q", q, on.dev)
    if q.dim() != 3 or q.shape[2] != d or q.shape[1] % Hkv:
        raise ValueError(f"q must be [T, Hq, {d}] with Hq a multiple of {Hkv}")
    if out is None:
        out = on.like(q)
    else:
        _halves("out", out, on.dev)
        if out.shape != q.shape:
            raise ValueError(f"out must have the shape of q {tuple(q.shape)}")
        o0, o1 = _span(out)
        for name, t in (("q", q), ("k_pages", k_pages), ("v_pages", v_pages)):
            t0, t1 = _span(t)
            if o0 < t1 and t0 < o1:
                raise ValueError(f"out must not overlap {name}")
    if lse is not None:
        _on_device("lse", lse, on.dev, torch.float32)
        if tuple(lse.shape) != tuple(q.shape[:2]):
            raise ValueError("lse must be [T, Hq]")
    return out


@functools.lru_cache(maxsize=4096)
def paged_workspace_bytes(B, max_seqlen, Hq, Hkv, d, max_len, top_k=0) -> int:
    """Workspace of tree_attn_paged, or with top_k of selected_attn_paged (da_paged_workspace_bytes)."""
    return int(load_library().da_paged_workspace_bytes(B, max_seqlen, Hq, Hkv, d, max_len, top_k))


def tree_attn_paged(q, k_pages, v_pages, table, lens, *, mask=None, slots=None, B=None, cu_seqlens=None,
                    max_seqlen=None, max_len=None, out=None, lse=None, workspace=None, stream=None):
    """Attention of the last tokens of each sequence, whose keys and values are in the cache:
    single tokens or causal chunks, or trees of drafts where ``mask`` int64 [T, words] has a bit for
    each drafted token that a row sees.  ``max_len`` bounds the lengths (default: the table's room):
    the work is shared out as for sequences that long, which suits short ones in a table with far more
    room less well (8 of 500 tokens, room for 262144: 13.4 us, with max_len 500 11.5).  Returns ``out``
    [T, Hq, d] (tree_attn_paged)."""
    dev, _, P, Hkv, d = _pages(k_pages, v_pages)
    on = _On(dev, stream)
    S, M = _table(table, lens, dev)
    out = _queries(q, k_pages, v_pages, out, lse, Hkv, d, on)
    T, Hq = q.shape[:2]
    B, N = _new_rows(T, B, cu_seqlens, max_seqlen, dev)
    words = 0
    if mask is not None:
        _on_device("mask", mask, dev, torch.int64)
        if mask.dim() != 2 or mask.shape[0] != T or mask.shape[1] * 64 < N:
            raise ValueError("mask must be [T, words] with a bit for each of max_seqlen tokens")
        words = mask.shape[1]
    room = M * PAGE_TOKENS
    max_len = room if max_len is None else min(int(max_len), room)
    ws, ptr, size = on.workspace(workspace, paged_workspace_bytes(B, N, Hq, Hkv, d, max_len) if workspace is None else 0)
    on.call("tree_attn_paged", _ptr(q), _ptr(k_pages), _ptr(v_pages), _ptr(out), _ptr(lse), _ptr(table), _ptr(lens), S, M,
            P, _slots(slots, B, S, dev), _ptr(cu_seqlens), B, N, max_len, Hq, Hkv, d, _ptr(mask), words, ptr, size)
    return out


def selected_attn_paged(q, k_pages, v_pages, table, lens, pages, *, slots=None, B=None, cu_seqlens=None,
                        max_seqlen=None, out=None, lse=None, workspace=None, stream=None):
    """Attention of the last tokens of each sequence over the pages that ``pages`` [T, Hkv, top_k]
    lists for them (as select_pages does) and the page each of them is in.  Returns ``out``
    [T, Hq, d] (selected_attn_paged)."""
    dev, _, P, Hkv, d = _pages(k_pages, v_pages)
    on = _On(dev, stream)
    S, M = _table(table, lens, dev)
    out = _queries(q, k_pages, v_pages, out, lse, Hkv, d, on)
    T, Hq = q.shape[:2]
    B, N = _new_rows(T, B, cu_seqlens, max_seqlen, dev)
    _ints("pages", pages, dev)
    if pages.dim() != 3 or tuple(pages.shape[:2]) != (T, Hkv):
        raise ValueError("pages must be [T, Hkv, top_k]")
    top_k = pages.shape[2]
    ws, ptr, size = on.workspace(workspace, paged_workspace_bytes(B, N, Hq, Hkv, d, 1, top_k) if workspace is None else 0)
    on.call("selected_attn_paged", _ptr(q), _ptr(k_pages), _ptr(v_pages), _ptr(out), _ptr(lse), _ptr(table), _ptr(lens),
            S, M, P, _slots(slots, B, S, dev), _ptr(cu_seqlens), B, N, Hq, Hkv, d, _ptr(pages), top_k, ptr, size)
    return out


def _summaries(codes, scales, blocks, Hkv, d, dev):
    _on_device("codes", codes, dev, torch.int8)
    _on_device("scales", scales, dev, torch.float32)
    if codes.dim() != 3 or codes.shape[0] < blocks or tuple(codes.shape[1:]) != (Hkv, d):
        raise ValueError(f"codes must be [{blocks}, {Hkv}, {d}]")
    if tuple(scales.shape) != tuple(codes.shape[:2]):
        raise ValueError(f"scales must be [{codes.shape[0]}, {Hkv}]")


def key_summary(k, *, B=None, cu_seqlens=None, max_seqlen=None, codes=None, scales=None, stream=None):
    """8-bit summaries of the whole 64-key blocks of k [T, Hkv, d]: (codes int8 [blocks, Hkv, d],
    scales fp32 [blocks, Hkv]), for select_blocks (da_key_summary)."""
    on = _On(k.device, stream)
    _on_device("k", k, on.dev, torch.bfloat16)
    if k.dim() != 3:
        raise ValueError("k must be [T, Hkv, d]")
    T, Hkv, d = k.shape
    B, N = _new_rows(T, B, cu_seqlens, max_seqlen, on.dev)
    blocks = int(load_library().da_key_summary_blocks(T, B))
    if codes is None:
        codes = on.empty((blocks, Hkv, d), torch.int8)
    if scales is None:
        scales = on.empty((codes.shape[0], Hkv), torch.float32)
    _summaries(codes, scales, blocks, Hkv, d, on.dev)
    on.call("da_key_summary", _ptr(k), _ptr(cu_seqlens), B, N, Hkv, d, _ptr(codes), _ptr(scales))
    return codes, scales


def page_summary(k_pages, table, lens, codes, scales, *, slots=None, first=None, max_new=None, stream=None):
    """Updates the summaries codes int8 [P, Hkv, d] and scales fp32 [P, Hkv] of the whole pages of
    each sequence, those from token ``first`` [B] (default 0) on and at most ``max_new`` tokens
    further (default: all; a decoding step that has added n tokens passes the lengths before it and
    n) (da_page_summary)."""
    dev, _, P, Hkv, d = _pages(k_pages, None)
    on = _On(dev, stream)
    S, M = _table(table, lens, dev)
    _summaries(codes, scales, P, Hkv, d, dev)
    B = S if slots is None else slots.numel()
    if first is not None:
        _ints("first", first, dev, (B,))
    on.call("da_page_summary", _ptr(k_pages), Hkv, d, _ptr(table), _ptr(lens), S, M, P, _slots(slots, B, S, dev),
            _ptr(first), B, M * PAGE_TOKENS if max_new is None else int(max_new), _ptr(codes), _ptr(scales))


def select_blocks(q, codes, scales, *, top_k, block_q, n_sink=1, n_recent=1, B=None, cu_seqlens=None, max_seqlen=None,
                  block_ptr=None, block_idx=None, stream=None):
    """The key tiles that each query block of block_q rows attends to, by score against key_summary's
    summaries: (block_ptr, block_idx) for blocksparse_attn_prefill and delta_attn_prefill_blocksparse
    (da_select_blocks).  A prompt within one query block has no lists: block_idx is then one -1, as
    those calls take no empty tensor."""
    on = _On(q.device, stream)
    _on_device("q", q, on.dev, torch.bfloat16)
    if q.dim() != 3 or codes.dim() != 3:
        raise ValueError("q must be [T, Hq, d] and codes [blocks, Hkv, d]")
    T, Hq, d = q.shape
    Hkv = codes.shape[1]
    B, N = _new_rows(T, B, cu_seqlens, max_seqlen, on.dev)
    lib = load_library()
    _summaries(codes, scales, int(lib.da_key_summary_blocks(T, B)), Hkv, d, on.dev)
    if block_q not in (64, 128, 256):
        raise ValueError("block_q must be 64, 128 or 256")
    entries = int(lib.da_select_blocks_entries(B, N, Hkv, top_k, block_q))
    nqb = -(-N // block_q)
    if block_ptr is None:
        block_ptr = on.empty((B, Hkv, nqb + 1), torch.int32)
    if block_idx is None:
        block_idx = on.empty(entries, torch.int32) if entries else on.full(1, -1, torch.int32)
    _ints("block_ptr", block_ptr, on.dev, (B, Hkv, nqb + 1))
    _ints("block_idx", block_idx, on.dev)
    if block_idx.numel() < max(entries, 1):
        raise ValueError(f"block_idx must hold {max(entries, 1)} entries (got {block_idx.numel()})")
    on.call("da_select_blocks", _ptr(q), _ptr(codes), _ptr(scales), _ptr(cu_seqlens), B, N, Hq, Hkv, d, top_k, n_sink,
            n_recent, block_q, _ptr(block_ptr), _ptr(block_idx))
    return block_ptr, block_idx


def select_pages(q, codes, scales, table, lens, *, top_k, n_sink=1, n_recent=1, slots=None, B=None, cu_seqlens=None,
                 max_seqlen=None, max_len=None, pages=None, workspace=None, stream=None):
    """The pages that each of the last tokens of each sequence attends to, by score against
    page_summary's summaries: ``pages`` int32 [T, Hkv, top_k] for selected_attn_paged, ascending,
    -1 behind the last (da_select_pages)."""
    on = _On(q.device, stream)
    _on_device("q", q, on.dev, torch.bfloat16)
    if q.dim() != 3 or codes.dim() != 3:
        raise ValueError("q must be [T, Hq, d] and codes [P, Hkv, d]")
    T, Hq, d = q.shape
    P, Hkv = codes.shape[:2]
    _summaries(codes, scales, P, Hkv, d, on.dev)
    S, M = _table(table, lens, on.dev)
    B, N = _new_rows(T, B, cu_seqlens, max_seqlen, on.dev)
    room = M * PAGE_TOKENS
    max_len = room if max_len is None else min(int(max_len), room)
    if pages is None:
        pages = on.like(lens, (T, Hkv, top_k))
    _ints("pages", pages, on.dev, (T, Hkv, top_k))
    need = int(load_library().da_select_pages_workspace_bytes(B, N, Hkv, max_len)) if workspace is None else 0
    ws, ptr, size = on.workspace(workspace, need)
    on.call("da_select_pages", _ptr(q), _ptr(codes), _ptr(scales), _ptr(table), _ptr(lens), S, M, P,
            _slots(slots, B, S, on.dev), _ptr(cu_seqlens), B, N, max_len, Hq, Hkv, d, top_k, n_sink, n_recent, _ptr(pages),
            ptr, size)
    return pages


def tree_mask(parents, device="cpu"):
    """The mask of tree_attn_paged for draft trees: ``parents`` holds for each sequence the parent of
    each drafted token (an earlier one of the sequence, or -1 under the context); a row sees itself and
    its ancestors.  Returns int64 [T, words] on ``device``."""
    words = max(1, -(-max((len(p) for p in parents), default=1) // 64))
    rows = []
    for seq in parents:
        seen = []
        for i, p in enumerate(seq):
            if not -1 <= p < i:
                raise ValueError(f"the parent of token {i} must be an earlier one or -1 (got {p})")
            seen.append((seen[p] if p >= 0 else 0) | 1 << i)
        for x in seen:
            w = [(x >> 64 * k) & 0xFFFFFFFFFFFFFFFF for k in range(words)]
            rows.append([v - (1 << 64) if v >> 63 else v for v in w])
    return torch.tensor(rows, dtype=torch.int64).reshape(-1, words).to(device)
