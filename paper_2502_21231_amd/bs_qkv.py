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


# Small calls are bound by this module's own time: the checks pass their common case with few attribute reads.


def _heads(t, name, dtype=None):
    """Checks a [T, heads, d] tensor on the GPU whose heads are contiguous; (elements from token to token, shape)."""
    if isinstance(t, torch.Tensor) and t.is_cuda and (dtype is None or t.dtype is dtype):
        shape = t.shape
        if len(shape) == 3:
            T, h, d = shape
            s0, s1, s2 = t.stride()
            if (s2 == 1 or d == 1) and (s1 == d or h == 1):
                return (s0 if T > 1 else h * d), shape
            raise ValueError(f"{name}: the heads of a token must be contiguous (strides {t.stride()})")
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on the GPU (got {t.device})")
    if dtype is not None and t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype} (got {t.dtype})")
    raise ValueError(f"{name} must have 3 dimensions (got {t.dim()})")


def _same_device(device, **tensors):
    for name, t in tensors.items():
        if t is not None and t.device != device:
            raise ValueError(f"{name} is on {t.device}, not on {device}")


def _one_device(index, *tensors):
    """Refuses tensors (or None) that are not on the GPU `index`; a workspace in host memory is one."""
    for t in tensors:
        if t is not None and t.get_device() != index:
            raise ValueError(f"a tensor is on {t.device}, the tokens are on cuda:{index}")


class QkParams:
    """Rotation and norm of queries and keys (see `make_qk_params`)."""

    def __init__(self, struct, tensors, head_dim, device):
        self.struct, self.tensors, self.head_dim, self.device = struct, tensors, head_dim, device
        self.ref = ctypes.byref(struct)
        self.index = None if device is None else device.index

    def check(self, t, d):
        if self.head_dim != d and self.head_dim is not None:
            raise ValueError(f"the weights have {self.head_dim} elements, a head {d}")
        if self.index != t.get_device() and self.index is not None:
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
        self.num_seqs, self.device, self.index = kv_lens.numel(), k.device, k.device.index

    def check(self, t, d, cu_seqlens_q) -> int:
        """The number of sequences, for tokens t [T, heads, d]."""
        if t.dtype is not self.dtype or d != self.head_dim or t.get_device() != self.index:
            raise ValueError(f"the cache holds {self.dtype} heads of {self.head_dim} elements on {self.device}")
        B._need(cu_seqlens_q, "cu_seqlens_q", torch.int32, 1)
        n = self.num_seqs
        if cu_seqlens_q.numel() != n + 1 or cu_seqlens_q.get_device() != self.index:
            raise ValueError(f"cu_seqlens_q must have {n + 1} entries on {self.device}")
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


def _qk(q, k, positions, params):
    """Strides of q and k, and the sizes (T, hq, hkv, d)."""
    qs, (T, hq, d) = _heads(q, "q")
    ks, (Tk, hkv, dk) = _heads(k, "k", q.dtype)
    if T != Tk or d != dk:
        raise ValueError(f"shape mismatch q {tuple(q.shape)} k {tuple(k.shape)}")
    params.check(q, d)
    B._need(positions, "positions", torch.int64, 1)
    if positions.shape[0] != T:
        raise ValueError("one position per token")
    return qs, ks, T, hq, hkv, d


def _out(t, like, name):
    """`t`, or a new contiguous tensor of the shape of `like`."""
    if t is None:
        return torch.empty_like(like, memory_format=torch.contiguous_format)
    B._need(t, name, like.dtype, 3)
    if t.shape != like.shape:
        raise ValueError(f"{name} must have the shape {tuple(like.shape)}")
    return t


def bs_qk_norm_rope_fwd(q, k, positions, params: QkParams, q_out=None, k_out=None):
    """Norm and rotation of q [T, hq, d] and k [T, hkv, d] (contiguous heads, any stride from token to
    token: parts of a fused projection's output will do) at `positions` (int64 [T]).  Returns contiguous
    (q_out, k_out) for the attention; they may be q and k themselves."""
    qs, ks, T, hq, hkv, d = _qk(q, k, positions, params)
    q_out, k_out = _out(q_out, q, "q_out"), _out(k_out, k, "k_out")
    _one_device(q.get_device(), k, positions, q_out, k_out)
    dims = B.bs_dims(T, 0, hq, hkv, d, B._dtype_code(q))
    p = B._ptr
    _call(q, _library().bs_qk_norm_rope_fwd, ctypes.byref(dims), params.ref, p(q), qs, p(k), ks, p(positions),
          p(q_out), p(k_out))
    return q_out, k_out


def bs_qk_norm_rope_workspace_size(dims: B.bs_dims) -> int:
    n = _library().bs_qk_norm_rope_workspace_size(ctypes.byref(dims))
    if n == 0:
        raise B.BsError(B.BS_ERR_INVALID_ARG, B.bs_last_error())
    return int(n)


def alloc_qk_workspace(q, k) -> torch.Tensor:
    """Workspace of bs_qk_norm_rope_bwd for tokens like these."""
    dims = B.bs_dims(q.shape[0], 0, q.shape[1], k.shape[1], q.shape[2], B._dtype_code(q))
    return torch.empty(bs_qk_norm_rope_workspace_size(dims), dtype=torch.uint8, device=q.device)


def _dweight(given, w, name, d):
    if w is None:
        if given is not None:
            raise ValueError(f"{name}: the gradient of a weight that the params do not have")
        return None
    if given is None:
        return torch.empty_like(w, dtype=torch.float32)
    B._need(given, name, torch.float32, 1)
    if given.shape[0] != d:
        raise ValueError(f"{name} must have {d} elements")
    return given


def bs_qk_norm_rope_bwd(q, k, positions, params: QkParams, dq_out, dk_out, dq=None, dk=None, dq_weight=None,
                        dk_weight=None, workspace=None):
    """Gradients of bs_qk_norm_rope_fwd's inputs from those of its outputs (contiguous).  q, k: the forward's
    inputs.  dq, dk may be strided like q and k (parts of the projection's gradient), or dq_out and dk_out
    themselves.  Returns (dq, dk, dq_weight, dk_weight); the weights' are float32 [d], None without weights."""
    qs, ks, T, hq, hkv, d = _qk(q, k, positions, params)
    dt = q.dtype
    B._need(dq_out, "dq_out", dt, 3)
    B._need(dk_out, "dk_out", dt, 3)
    if dq is None:
        dq = torch.empty_like(dq_out)
    if dk is None:
        dk = torch.empty_like(dk_out)
    dqs, q_shape = _heads(dq, "dq", dt)
    dks, k_shape = _heads(dk, "dk", dt)
    if q_shape != (T, hq, d) or k_shape != (T, hkv, d) or dq_out.shape != q_shape or dk_out.shape != k_shape:
        raise ValueError("dq_out, dk_out, dq and dk must have the shapes of q and k")
    _, wq, wk = params.tensors
    dq_weight = _dweight(dq_weight, wq, "dq_weight", d)
    dk_weight = _dweight(dk_weight, wk, "dk_weight", d)
    if workspace is None and (wq is not None or wk is not None):
        workspace = alloc_qk_workspace(q, k)
    _one_device(q.get_device(), k, positions, dq_out, dk_out, dq, dk, dq_weight, dk_weight, workspace)
    dims = B.bs_dims(T, 0, hq, hkv, d, B._dtype_code(q))
    p = B._ptr
    _call(q, _library().bs_qk_norm_rope_bwd, ctypes.byref(dims), params.ref, p(q), qs, p(k), ks, p(positions),
          p(dq_out), p(dk_out), p(dq), dqs, p(dk), dks, p(dq_weight), p(dk_weight), p(workspace),
          0 if workspace is None else workspace.numel())
    return dq, dk, dq_weight, dk_weight


def bs_kv_append(q, k, v, cache: PagedCache, cu_seqlens_q, params: QkParams | None = None, q_out=None):
    """Appends the new tokens of a step to the cache: rows cu_seqlens_q[b] .. cu_seqlens_q[b+1]-1 of k, v
    [T, hkv, d] are the last tokens of sequence b, whose cache.kv_lens[b] counts them already.  Keys go
    through `params` at their position; so do the queries q [T, hq, d] (or None), into q_out, which is
    returned.  Rows behind the last sequence are left alone (an own q_out then holds whatever its memory did)."""
    ks, k_shape = _heads(k, "k")
    vs, v_shape = _heads(v, "v", k.dtype)
    T, hkv, d = k_shape
    if k_shape != v_shape or hkv != cache.hkv:
        raise ValueError(f"k {tuple(k_shape)} and v {tuple(v_shape)} must have the cache's {cache.hkv} heads")
    nseq = cache.check(k, d, cu_seqlens_q)
    if params is not None:
        params.check(k, d)
    qs, hq = 0, hkv
    if q is not None:
        qs, (Tq, hq, dq) = _heads(q, "q", k.dtype)
        if Tq != T or dq != d:
            raise ValueError(f"shape mismatch q {tuple(q.shape)} k {tuple(k_shape)}")
        q_out = _out(q_out, q, "q_out")
    else:
        q_out = None
    _one_device(cache.index, q, v, q_out)
    dims = B.bs_dims(T, 0, hq, hkv, d, B._dtype_code(k))
    p = B._ptr
    _call(k, _library().bs_kv_append, ctypes.byref(dims), None if params is None else params.ref, cache.ref,
          p(cu_seqlens_q), nseq, p(q), qs, p(k), ks, p(v), vs, p(q_out))
    return q_out


def bs_attn_paged_workspace_size(dims: B.bs_dims, num_seqs: int, max_seqlen_k: int) -> int:
    n = _library().bs_attn_paged_workspace_size(ctypes.byref(dims), num_seqs, max_seqlen_k)
    if n == 0:
        raise B.BsError(B.BS_ERR_INVALID_ARG, B.bs_last_error())
    return int(n)


def alloc_paged_workspace(q, cache: PagedCache, max_seqlen_k: int) -> torch.Tensor:
    """Workspace of bs_attn_paged_fwd for queries like these over this cache (66 MiB are enough for any)."""
    dims = B.bs_dims(q.shape[0], 0, q.shape[1], cache.hkv, q.shape[2], B._dtype_code(q))
    return torch.empty(bs_attn_paged_workspace_size(dims, cache.num_seqs, int(max_seqlen_k)), dtype=torch.uint8,
                       device=q.device)


def bs_attn_paged_fwd(q, cache: PagedCache, cu_seqlens_q, max_seqlen_k: int, causal: bool = True,
                      scale: float | None = None, out=None, lse=None, workspace=None):
    """Attention of the new tokens q [T, hq, d] of each sequence over its cached keys (row i of n sees key j
    iff j <= i + kv_len - n, with causal).  Returns (out [T, hq, d], lse float32 [hq, T]); rows behind the last
    sequence are left as they were."""
    B._need(q, "q", None, 3)
    T, hq, d = q.shape
    nseq = cache.check(q, d, cu_seqlens_q)
    out = _out(out, q, "out")
    if lse is None:
        lse = torch.empty(hq, T, dtype=torch.float32, device=q.device)
    else:
        B._need(lse, "lse", torch.float32, 2)
        if lse.shape != (hq, T):
            raise ValueError(f"lse must have the shape {(hq, T)}")
    if workspace is None:
        workspace = alloc_paged_workspace(q, cache, max_seqlen_k)
    _one_device(cache.index, out, lse, workspace)
    dims = B.bs_dims(T, 0, hq, cache.hkv, d, B._dtype_code(q))
    p = B._ptr
    _call(q, _library().bs_attn_paged_fwd, ctypes.byref(dims), p(q), cache.ref, p(cu_seqlens_q), nseq,
          int(max_seqlen_k), int(bool(causal)), B._scale(scale, d), p(out), p(lse), p(workspace), workspace.numel())
    return out, lse
