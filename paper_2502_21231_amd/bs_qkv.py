"""Python binding of the entry points of bs_qkv.h in libbs_attn.so (argument marshalling only): norm
and rotation of queries and keys, appending to a paged key/value cache, attention over it.

As in bs_attn.py, each function has the name of the C entry point it calls, and every step of the
computation runs in the library's HIP kernels.  What stays the same from step to step (the rotation and
the norms' weights, the cache with its page table) is marshalled once, by `make_qk_params` and
`make_paged_cache`, and handed to the calls.
"""
from __future__ import annotations

import ctypes

import torch

from . import bs_attn as B

EXPORTS = ("bs_qk_norm_rope_fwd", "bs_qk_norm_rope_workspace_size", "bs_qk_norm_rope_bwd", "bs_kv_append",
           "bs_attn_paged_workspace_size", "bs_attn_paged_fwd")
BS_KERNEL_QK_ROPE, BS_KERNEL_KV_APPEND, BS_KERNEL_PAGED = 8, 9, 10


class bs_qk_params(ctypes.Structure):
    _fields_ = [("inv_freq", ctypes.c_void_p), ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("weight_dtype", ctypes.c_int32),
                ("eps", ctypes.c_float)]


class bs_paged_cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("num_pages", ctypes.c_int64),
                ("page_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("block_table", ctypes.c_void_p), ("table_stride", ctypes.c_int64), ("max_pages", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("kv_lens", ctypes.c_void_p)]


_LIB = None


def _library() -> ctypes.CDLL:
    global _LIB
    if _LIB is None:
        lib = B.load_library()
        P, I32, I64, F, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
        DIMS, PAR, CACHE = (ctypes.POINTER(t) for t in (B.bs_dims, bs_qk_params, bs_paged_cache))
        sig = {
            "bs_qk_norm_rope_fwd": (ctypes.c_int, [DIMS, PAR, P, I64, P, I64, P, P, P, P]),
            "bs_qk_norm_rope_workspace_size": (SZ, [DIMS]),
            "bs_qk_norm_rope_bwd": (ctypes.c_int, [DIMS, PAR, P, I64, P, I64, P, P, P, P, I64, P, I64, P, P, P, SZ, P]),
            "bs_kv_append": (ctypes.c_int, [DIMS, PAR, CACHE, P, I32, P, I64, P, I64, P, I64, P, P]),
            "bs_attn_paged_workspace_size": (SZ, [DIMS, I32, I32]),
            "bs_attn_paged_fwd": (ctypes.c_int, [DIMS, P, CACHE, P, I32, I32, ctypes.c_int, F, P, P, P, SZ, P]),
        }
        for name, (res, args) in sig.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _LIB = lib
    return _LIB


_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _call(t, fn, *args) -> None:
    """fn(*args, stream) with the device of `t` current (a launch on the default stream goes to the
    current device, whatever memory it is given)."""
    if t.get_device() == _current_device():
        B._check(fn(*args, B._stream(t)))
        return
    with torch.cuda.device(t.device):
        B._check(fn(*args, B._stream(t)))


def _heads(t, name, dtype=None) -> int:
    """Checks a [T, heads, d] tensor on the GPU whose heads are contiguous; elements from token to token."""
    if isinstance(t, torch.Tensor) and t.is_cuda and t.dim() == 3 and (dtype is None or t.dtype is dtype):
        T, h, d = t.shape
        s = t.stride()
        if (s[2] == 1 or d == 1) and (s[1] == d or h == 1):
            return s[0] if T > 1 else h * d
        raise ValueError(f"{name}: the heads of a token must be contiguous (strides {s})")
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on the GPU (got {t.device})")
    if dtype is not None and t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype} (got {t.dtype})")
    raise ValueError(f"{name} must have 3 dimensions (got {t.dim()})")


def _dims(q_shape, hq, hkv, dtype) -> B.bs_dims:
    return B.bs_dims(q_shape[0], 0, hq, hkv, q_shape[2], dtype)


def _same_device(device, **tensors):
    for name, t in tensors.items():
        if t is not None and t.device != device:
            raise ValueError(f"{name} is on {t.device}, not on {device}")


class QkParams:
    """Rotation and norm of queries and keys (see `make_qk_params`)."""

    def __init__(self, struct, tensors, head_dim, device):
        self.struct, self.tensors, self.head_dim, self.device = struct, tensors, head_dim, device
        self.ref = ctypes.byref(struct)

    def check(self, t):
        if self.head_dim is not None and t.shape[2] != self.head_dim:
            raise ValueError(f"the weights have {self.head_dim} elements, a head {t.shape[2]}")
        if self.device is not None and t.device != self.device:
            raise ValueError(f"params are on {self.device}, the tokens on {t.device}")


def make_qk_params(inv_freq=None, interleaved: bool = False, q_weight=None, k_weight=None,
                   eps: float = 1e-6) -> QkParams:
    """What is done to queries and keys: with weights ([head_dim], bf16 or float32) a norm of each head,
    with `inv_freq` (float32 [rot_dim / 2]) the rotation of the first rot_dim elements by position *
    inv_freq, of pairs (i, i + rot_dim / 2), or (2i, 2i + 1) if interleaved."""
    given = [t for t in (inv_freq, q_weight, k_weight) if t is not None]
    if inv_freq is not None:
        B._need(inv_freq, "inv_freq", torch.float32, 1)
    head_dim, wdtype = None, B.BS_F32
    for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
        if w is not None:
            B._need(w, name, None, 1)
            if head_dim is not None and (w.numel() != head_dim or B._dtype_code(w) != wdtype):
                raise ValueError("q_weight and k_weight must have the same dtype and length")
            head_dim, wdtype = w.numel(), B._dtype_code(w)
    device = given[0].device if given else None
    for t in given:
        if t.device != device:
            raise ValueError("inv_freq and the weights must be on one device")
    s = bs_qk_params(B._ptr(inv_freq), 0 if inv_freq is None else 2 * inv_freq.numel(), int(bool(interleaved)),
                     B._ptr(q_weight), B._ptr(k_weight), wdtype, float(eps))
    return QkParams(s, (inv_freq, q_weight, k_weight), head_dim, device)


class PagedCache:
    """A paged cache with its table and lengths (see `make_paged_cache`)."""

    def __init__(self, struct, k, v, block_table, kv_lens):
        self.struct, self.k, self.v, self.block_table, self.kv_lens = struct, k, v, block_table, kv_lens
        self.ref = ctypes.byref(struct)
        self.hkv, self.head_dim, self.dtype = k.shape[2], k.shape[3], k.dtype
        self.num_seqs, self.device = kv_lens.numel(), k.device

    def check(self, t, cu_seqlens_q) -> int:
        """The number of sequences, for tokens t [T, heads, d]."""
        if t.dtype is not self.dtype or t.shape[2] != self.head_dim or t.device != self.device:
            raise ValueError(f"the cache holds {self.dtype} heads of {self.head_dim} elements on {self.device}")
        B._need(cu_seqlens_q, "cu_seqlens_q", torch.int32, 1)
        n = cu_seqlens_q.numel() - 1
        if n != self.num_seqs or cu_seqlens_q.device != self.device:
            raise ValueError(f"cu_seqlens_q must have {self.num_seqs + 1} entries on {self.device}")
        return n


def make_paged_cache(k, v, block_table, kv_lens) -> PagedCache:
    """A cache whose pages are k, v [num_pages, page_size, hkv, head_dim], strided alike in any order of
    memory with contiguous heads (pages stored as [num_pages, hkv, page_size, head_dim]: permute(0, 2, 1,
    3)).  block_table int32 [num_seqs, max_pages], -1 (or any number that is no page) where a sequence has
    none; kv_lens int32 [num_seqs].  The tensors are held, not copied: a step fills the table and lengths in
    place."""
    for t, name in ((k, "k"), (v, "v")):
        if not isinstance(t, torch.Tensor) or t.dim() != 4:
            raise ValueError(f"{name} must be a tensor [num_pages, page_size, hkv, head_dim]")
        if not t.is_cuda:
            raise ValueError(f"{name} must be on the GPU (got {t.device})")
    if k.shape != v.shape or k.dtype != v.dtype or k.stride() != v.stride():
        raise ValueError("k and v must have the same shape, dtype and strides")
    B._dtype_code(k)
    if k.shape[3] > 1 and k.stride(3) != 1:
        raise ValueError("the elements of a head must follow one another")
    if not isinstance(block_table, torch.Tensor) or block_table.dim() != 2 or block_table.dtype != torch.int32:
        raise TypeError("block_table must be an int32 tensor [num_seqs, max_pages]")
    if block_table.shape[1] > 1 and block_table.stride(1) != 1:
        raise ValueError("the entries of a row of block_table must follow one another")
    B._need(kv_lens, "kv_lens", torch.int32, 1)
    if kv_lens.numel() != block_table.shape[0]:
        raise ValueError("block_table and kv_lens must have one entry per sequence")
    _same_device(k.device, v=v, block_table=block_table, kv_lens=kv_lens)
    pages, page_size, hkv, d = k.shape
    # a dimension of one element may have any stride; the library wants one it could use
    unit = d
    ps, ts, hs = (k.stride(i) if k.shape[i] > 1 else unit for i in range(3))
    rows = block_table.shape[0]
    s = bs_paged_cache(B._ptr(k), B._ptr(v), pages, ps, ts, hs, B._ptr(block_table),
                       block_table.stride(0) if rows > 1 else block_table.shape[1], block_table.shape[1], page_size,
                       B._ptr(kv_lens))
    return PagedCache(s, k, v, block_table, kv_lens)


def _qk(q, k, params):
    qs, ks = _heads(q, "q"), _heads(k, "k", q.dtype)
    if q.shape[0] != k.shape[0] or q.shape[2] != k.shape[2]:
        raise ValueError(f"shape mismatch q {tuple(q.shape)} k {tuple(k.shape)}")
    params.check(q)
    return qs, ks


def _out(t, like, name):
    """`t`, or a new contiguous tensor of the shape of `like`."""
    if t is None:
        return torch.empty(like.shape, dtype=like.dtype, device=like.device)
    B._need(t, name, like.dtype, 3)
    if t.shape != like.shape:
        raise ValueError(f"{name} must have the shape {tuple(like.shape)}")
    return t


def _positions(positions, q):
    B._need(positions, "positions", torch.int64, 1)
    if positions.numel() != q.shape[0]:
        raise ValueError("one position per token")


def bs_qk_norm_rope_fwd(q, k, positions, params: QkParams, q_out=None, k_out=None):
    """Norm and rotation of q [T, hq, d] and k [T, hkv, d] (contiguous heads, any stride from token to
    token: parts of a fused projection's output will do) at `positions` (int64 [T]).  Returns contiguous
    (q_out, k_out) for the attention; they may be q and k themselves."""
    qs, ks = _qk(q, k, params)
    _positions(positions, q)
    q_out, k_out = _out(q_out, q, "q_out"), _out(k_out, k, "k_out")
    dims = _dims(q.shape, q.shape[1], k.shape[1], B._dtype_code(q))
    _call(q, _library().bs_qk_norm_rope_fwd, ctypes.byref(dims), params.ref, B._ptr(q), qs, B._ptr(k), ks,
          B._ptr(positions), B._ptr(q_out), B._ptr(k_out))
    return q_out, k_out


def bs_qk_norm_rope_workspace_size(dims: B.bs_dims) -> int:
    n = _library().bs_qk_norm_rope_workspace_size(ctypes.byref(dims))
    if n == 0:
        raise B.BsError(B.BS_ERR_INVALID_ARG, B.bs_last_error())
    return int(n)


def alloc_qk_workspace(q, k) -> torch.Tensor:
    """Workspace of bs_qk_norm_rope_bwd for tokens like these."""
    dims = _dims(q.shape, q.shape[1], k.shape[1], B._dtype_code(q))
    return torch.empty(bs_qk_norm_rope_workspace_size(dims), dtype=torch.uint8, device=q.device)


def bs_qk_norm_rope_bwd(q, k, positions, params: QkParams, dq_out, dk_out, dq=None, dk=None, dq_weight=None,
                        dk_weight=None, workspace=None):
    """Gradients of bs_qk_norm_rope_fwd's inputs from those of its outputs (contiguous).  q, k: the forward's
    inputs.  dq, dk may be strided like q and k (parts of the projection's gradient), or dq_out and dk_out
    themselves.  Returns (dq, dk, dq_weight, dk_weight); the weights' are float32 [d], None without weights."""
    qs, ks = _qk(q, k, params)
    _positions(positions, q)
    B._need(dq_out, "dq_out", q.dtype, 3)
    B._need(dk_out, "dk_out", q.dtype, 3)
    if dq_out.shape != q.shape or dk_out.shape != k.shape:
        raise ValueError("dq_out and dk_out must have the shapes of q and k")
    if dq is None:
        dq = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    if dk is None:
        dk = torch.empty(k.shape, dtype=k.dtype, device=k.device)
    dqs, dks = _heads(dq, "dq", q.dtype), _heads(dk, "dk", k.dtype)
    if dq.shape != q.shape or dk.shape != k.shape:
        raise ValueError("dq and dk must have the shapes of q and k")
    _, wq, wk = params.tensors
    d = q.shape[2]
    if wq is None and dq_weight is not None or wk is None and dk_weight is not None:
        raise ValueError("the gradient of a weight that the params do not have")
    if wq is not None and dq_weight is None:
        dq_weight = torch.empty(d, dtype=torch.float32, device=q.device)
    if wk is not None and dk_weight is None:
        dk_weight = torch.empty(d, dtype=torch.float32, device=q.device)
    for w, name in ((dq_weight, "dq_weight"), (dk_weight, "dk_weight")):
        if w is not None:
            B._need(w, name, torch.float32, 1)
            if w.numel() != d:
                raise ValueError(f"{name} must have {d} elements")
    if workspace is None and (wq is not None or wk is not None):
        workspace = alloc_qk_workspace(q, k)
    dims = _dims(q.shape, q.shape[1], k.shape[1], B._dtype_code(q))
    _call(q, _library().bs_qk_norm_rope_bwd, ctypes.byref(dims), params.ref, B._ptr(q), qs, B._ptr(k), ks,
          B._ptr(positions), B._ptr(dq_out), B._ptr(dk_out), B._ptr(dq), dqs, B._ptr(dk), dks, B._ptr(dq_weight),
          B._ptr(dk_weight), B._ptr(workspace), 0 if workspace is None else workspace.numel())
    return dq, dk, dq_weight, dk_weight


def bs_kv_append(q, k, v, cache: PagedCache, cu_seqlens_q, params: QkParams | None = None, q_out=None):
    """Appends the new tokens of a step to the cache: rows cu_seqlens_q[b] .. cu_seqlens_q[b+1]-1 of k, v
    [T, hkv, d] are the last tokens of sequence b, whose cache.kv_lens[b] counts them already.  Keys go
    through `params` at their position; so do the queries q [T, hq, d] (or None), into q_out, which is
    returned.  Rows behind the last sequence are left alone (an own q_out then holds whatever its memory did)."""
    ks, vs = _heads(k, "k"), _heads(v, "v", k.dtype)
    if k.shape != v.shape or k.shape[1] != cache.hkv:
        raise ValueError(f"k {tuple(k.shape)} and v {tuple(v.shape)} must have the cache's {cache.hkv} heads")
    nseq = cache.check(k, cu_seqlens_q)
    if params is not None:
        params.check(k)
    qs, hq = 0, cache.hkv
    if q is not None:
        qs, hq = _heads(q, "q", k.dtype), q.shape[1]
        if q.shape[0] != k.shape[0] or q.shape[2] != k.shape[2] or q.device != k.device:
            raise ValueError(f"shape mismatch q {tuple(q.shape)} k {tuple(k.shape)}")
        q_out = _out(q_out, q, "q_out")
    dims = _dims(k.shape, hq, cache.hkv, B._dtype_code(k))
    _call(k, _library().bs_kv_append, ctypes.byref(dims), None if params is None else params.ref, cache.ref,
          B._ptr(cu_seqlens_q), nseq, B._ptr(q), qs, B._ptr(k), ks, B._ptr(v), vs,
          B._ptr(q_out) if q is not None else None)
    return q_out if q is not None else None


def bs_attn_paged_workspace_size(dims: B.bs_dims, num_seqs: int, max_seqlen_k: int) -> int:
    n = _library().bs_attn_paged_workspace_size(ctypes.byref(dims), num_seqs, max_seqlen_k)
    if n == 0:
        raise B.BsError(B.BS_ERR_INVALID_ARG, B.bs_last_error())
    return int(n)


def alloc_paged_workspace(q, cache: PagedCache, max_seqlen_k: int) -> torch.Tensor:
    """Workspace of bs_attn_paged_fwd for queries like these over this cache."""
    dims = _dims(q.shape, q.shape[1], cache.hkv, B._dtype_code(q))
    return torch.empty(bs_attn_paged_workspace_size(dims, cache.num_seqs, int(max_seqlen_k)), dtype=torch.uint8,
                       device=q.device)


def bs_attn_paged_fwd(q, cache: PagedCache, cu_seqlens_q, max_seqlen_k: int, causal: bool = True,
                      scale: float | None = None, out=None, lse=None, workspace=None):
    """Attention of the new tokens q [T, hq, d] of each sequence over its cached keys (row i of n sees key j
    iff j <= i + kv_len - n, with causal).  Returns (out [T, hq, d], lse float32 [hq, T]); rows behind the last
    sequence are left as they were."""
    B._need(q, "q", None, 3)
    nseq = cache.check(q, cu_seqlens_q)
    T, hq, d = q.shape
    out = _out(out, q, "out")
    if lse is None:
        lse = torch.empty(hq, T, dtype=torch.float32, device=q.device)
    else:
        B._need(lse, "lse", torch.float32, 2)
        if lse.shape != (hq, T):
            raise ValueError(f"lse must have the shape {(hq, T)}")
    if workspace is None:
        workspace = alloc_paged_workspace(q, cache, max_seqlen_k)
    dims = _dims(q.shape, hq, cache.hkv, B._dtype_code(q))
    _call(q, _library().bs_attn_paged_fwd, ctypes.byref(dims), B._ptr(q), cache.ref, B._ptr(cu_seqlens_q), nseq,
          int(max_seqlen_k), int(bool(causal)), B._scale(scale, d), B._ptr(out), B._ptr(lse), B._ptr(workspace),
          workspace.numel())
    return out, lse
