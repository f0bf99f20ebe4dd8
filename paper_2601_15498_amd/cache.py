"""Binding of the paged 4-bit cache (include/mars_cache.h) -- argument marshalling only.

The functions mirror the header name for name and take the cache's tensors: ``pool`` [layers, pages, heads, bytes] uint8, ``page_table``
[sequences, width], ``lens``, ``held`` [sequences] and ``refs`` [pages], all int32 (``KVCache`` makes them).  Every call enqueues on the
current torch stream and returns without synchronising; there is no CPU fallback.  bf16 rows may be given as ``torch.bfloat16`` or as
``torch.uint16``/``int16`` bit patterns.

A regular call -- plain tensors of the right types and shapes, outputs and workspace given -- goes through csrc/cache_marshal.cpp
(``_cache_marshal.so``); anything else through ctypes here, with the checks that say what is wrong.
"""
import ctypes
import math
import warnings

import torch

from . import binding
from .binding import MARS_BF16, MARS_F32, MarsError, _DTYPE_CODES, _check, _dtype_code, _ptr, _stream  # noqa: F401

MARS_KV_OK, MARS_KV_NO_PAGES, MARS_KV_TOO_LONG, MARS_KV_BAD_SEQUENCE, MARS_KV_BAD_PATH, MARS_KV_NOT_EMPTY = range(6)
MARS_KV_MAX_REQUESTS = 4096
HEAD_DIMS = (64, 128, 256)


class CacheStruct(ctypes.Structure):
    """struct mars_kv_cache (a host struct holding device pointers)."""
    _fields_ = ([(n, ctypes.c_void_p) for n in ("pool", "page_table", "lens", "held", "refs")]
                + [(n, ctypes.c_int32) for n in ("layers", "pages", "heads", "dim", "page", "sequences", "width")])


class RowsStruct(ctypes.Structure):
    """struct mars_kv_rows."""
    _fields_ = [("data", ctypes.c_void_p), ("request", ctypes.c_int64), ("node", ctypes.c_int64), ("head", ctypes.c_int64)]


_lib = None
_native = None  # csrc/cache_marshal.cpp, once the library is loaded


class _NoNative:
    """In place of csrc/cache_marshal.cpp: no call is a regular one."""
    append = read = tree_mask = attention = commit = reserve = fork = release = staticmethod(lambda *args: None)


def _load_native(L):
    try:
        from . import _cache_marshal
        if _cache_marshal.torch_version != torch.__version__:
            raise ImportError(f"built with PyTorch {_cache_marshal.torch_version}, not {torch.__version__}")
    except ImportError as e:
        warnings.warn(f"_cache_marshal.so is missing or does not load ({e}): calls go through ctypes, which costs some 6 us each; "
                      "build it with `python -m paper_2601_15498_amd.build`", RuntimeWarning, stacklevel=3)
        return _NoNative
    _cache_marshal.bind(*(ctypes.cast(f, ctypes.c_void_p).value for f in
                          (L.mars_kv_append, L.mars_kv_read, L.mars_tree_mask, L.mars_kv_attention, L.mars_kv_commit, L.mars_kv_reserve,
                           L.mars_kv_fork, L.mars_kv_release)), True)
    return _cache_marshal


def _calls():
    lib()
    return _native


def lib():
    global _lib, _native
    if _lib is None:
        L = binding.lib()
        p, i, n = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
        cache, rows = ctypes.POINTER(CacheStruct), ctypes.POINTER(RowsStruct)
        for name, result, arguments in (
                ("mars_kv_head_bytes", n, [i, i]),
                ("mars_kv_append", i, [cache, i, p, rows, rows, i, p, i, i, p, p]),
                ("mars_kv_read", i, [cache, i, p, p, rows, rows, i, i, i, p]),
                ("mars_tree_mask", i, [p, p, i, i, p, p, p]),
                ("mars_kv_attention_workspace_bytes", n, [i] * 6),
                ("mars_kv_attention", i, [cache, i, p, rows, i, i, p, p, ctypes.c_float, i, rows, p, i, i, p, n, p]),
                ("mars_kv_commit", i, [cache, p, p, p, i, i, p, p, p]),
                ("mars_kv_reserve_workspace_bytes", n, [i, i]),
                ("mars_kv_reserve", i, [cache, p, p, i, i, p, p, n, p]),
                ("mars_kv_fork", i, [cache, p, p, i, p, p]),
                ("mars_kv_release", i, [cache, p, i, p, p]),
                ("mars_kv_copy_pages", i, [cache, p, p, i, p])):
            f = getattr(L, name)
            f.restype, f.argtypes = result, arguments
        _native = _load_native(L)   # (before _lib: whoever sees the library has the calls)
        _lib = L
    return _lib


class KVCache:
    """The tensors of an empty cache."""

    def __init__(self, layers: int, pages: int, heads: int, head_dim: int, page_size: int, sequences: int, max_len: int, device="cuda"):
        self.head_dim, self.page_size = head_dim, page_size
        self.pool = torch.empty((layers, pages, heads, mars_kv_head_bytes(head_dim, page_size)), dtype=torch.uint8, device=device)
        self.page_table = torch.full((sequences, -(-max_len // page_size)), -1, dtype=torch.int32, device=device)
        self.lens = torch.zeros(sequences, dtype=torch.int32, device=device)
        self.held = torch.zeros(sequences, dtype=torch.int32, device=device)
        self.refs = torch.zeros(pages, dtype=torch.int32, device=device)


def mars_kv_head_bytes(head_dim: int, page_size: int) -> int:
    """Bytes of a head in a page; raises where the library does not support the sizes."""
    n = int(lib().mars_kv_head_bytes(head_dim, page_size))
    if n == 0:
        raise MarsError(f"head_dim {head_dim} (64, 128 or 256) and page_size {page_size} (a power of two, 8 to 256) are not supported together")
    return n


def _page_size(pool, head_dim):
    return pool.shape[3] * 16 // (17 * head_dim)


def _table(t, shape, what):
    if t is None:
        return None
    assert t.dtype == torch.int32 and t.shape == shape and t.is_contiguous(), what
    assert t.is_cuda, what + ": not on the GPU"
    return t.data_ptr()


def _cache(pool, page_table, lens, held=None, refs=None, head_dim=0, page_size=0):
    """The struct of a call; without a pool (the calls that move no rows) its part of the sizes is made up."""
    sequences, width = page_table.shape
    if pool is None:
        layers, pages, heads, head_dim = 1, refs.numel(), 1, 64
    else:
        layers, pages, heads, blk = pool.shape
        assert pool.dtype == torch.uint8 and pool.is_contiguous() and pool.is_cuda, "pool"
        if not head_dim:
            head_dim = blk * 16 // (17 * page_size)
        assert page_size * (head_dim + head_dim // 16) == blk, "pool: the bytes of a head are not those of these sizes"
    return CacheStruct(_ptr(pool), _table(page_table, (sequences, width), "page_table"), _table(lens, (sequences,), "lens"),
                       _table(held, (sequences,), "held"), _table(refs, (pages,), "refs"), layers, pages, heads, head_dim, page_size,
                       sequences, width)


def _rows(t, what):
    assert t.dim() == 4 and t.stride(3) == 1 and t.is_cuda, what
    return RowsStruct(t.data_ptr(), t.stride(0), t.stride(1), t.stride(2))


def _batch(seqs, lens, B):
    assert seqs is not None or B <= lens.shape[0], "more requests than sequences"
    return _table(seqs, (B,), "seqs")


def mars_kv_append(pool: torch.Tensor, page_table: torch.Tensor, lens: torch.Tensor, k: torch.Tensor, v: torch.Tensor, *, layer: int = 0,
                   seqs: torch.Tensor = None, n_new: torch.Tensor = None, status: torch.Tensor = None) -> None:
    """Keys and values [B, N, heads, head_dim] of new tokens into the cache, behind the committed ones.  Any strides that are multiples of 16
    bytes, the last one 1."""
    rc = (_native or _calls()).append(pool, page_table, lens, k, v, layer, seqs, n_new, status, _stream)
    if rc is not None:
        return _check(rc)
    B, N, heads, D = k.shape
    assert v.shape == k.shape and v.dtype == k.dtype and heads == pool.shape[2]
    c = _cache(pool, page_table, lens, head_dim=D, page_size=_page_size(pool, D))
    kr, vr = _rows(k, "k"), _rows(v, "v")
    _check(lib().mars_kv_append(c, layer, _batch(seqs, lens, B), kr, vr, _dtype_code(k), _table(n_new, (B,), "n_new"), B, N,
                                _table(status, (B,), "status"), _stream()))


def mars_kv_read(pool: torch.Tensor, page_table: torch.Tensor, held: torch.Tensor = None, *, layer: int = 0, seqs: torch.Tensor = None,
                 first: torch.Tensor = None, out=None, B: int = None, N: int = None, head_dim: int = None, dtype=torch.bfloat16):
    """Keys and values [B, N, heads, head_dim] of positions first[b] .. first[b] + N - 1, into ``out`` (a pair) if given."""
    if out is not None:
        rc = (_native or _calls()).read(pool, page_table, held, *out, layer, seqs, first, _stream)
        if rc is not None:
            _check(rc)
            return out
    if out is None:
        B = B if B is not None else seqs.numel() if seqs is not None else page_table.shape[0]
        out = tuple(torch.empty((B, N, pool.shape[2], head_dim), dtype=dtype, device=pool.device) for _ in range(2))
    k, v = out
    B, N, heads, D = k.shape
    assert v.shape == k.shape and v.dtype == k.dtype and heads == pool.shape[2]
    c = _cache(pool, page_table, None, held, head_dim=D, page_size=_page_size(pool, D))
    _check(lib().mars_kv_read(c, layer, _batch(seqs, page_table, B), _table(first, (B,), "first"), _rows(k, "k"), _rows(v, "v"),
                              _dtype_code(k), B, N, _stream()))
    return k, v


def mars_tree_mask(tree_parent: torch.Tensor, *, n_new: torch.Tensor = None, mask: torch.Tensor = None,
                   status: torch.Tensor = None) -> torch.Tensor:
    """[B, N, (N + 63) // 64] int64: bit j of row i is set iff node j is node i or an ancestor."""
    rc = (_native or _calls()).tree_mask(tree_parent, n_new, mask, status, _stream)
    if rc is not None:
        _check(rc)
        return mask
    B, N = tree_parent.shape
    if mask is None:
        mask = torch.empty((B, N, (N + 63) // 64), dtype=torch.int64, device=tree_parent.device)
    assert mask.dtype == torch.int64 and mask.shape == (B, N, (N + 63) // 64) and mask.is_contiguous() and mask.is_cuda
    _check(lib().mars_tree_mask(_table(tree_parent, (B, N), "tree_parent"), _table(n_new, (B,), "n_new"), B, N, mask.data_ptr(),
                                _table(status, (B,), "status"), _stream()))
    return mask


def alloc_attention_workspace(pool: torch.Tensor, page_table: torch.Tensor, q: torch.Tensor) -> torch.Tensor:
    """Workspace of mars_kv_attention for queries of this shape; serves calls on any layer, one after the other."""
    B, N, q_heads, D = q.shape
    n = int(lib().mars_kv_attention_workspace_bytes(B, N, q_heads, pool.shape[2], D, _dtype_code(q)))
    if n == 0:
        raise MarsError(f"sizes out of range: B={B} N={N} q_heads={q_heads} heads={pool.shape[2]} head_dim={D}")
    return torch.empty(n, dtype=torch.uint8, device=pool.device)


def mars_kv_attention(pool: torch.Tensor, page_table: torch.Tensor, lens: torch.Tensor, q: torch.Tensor, *, layer: int = 0,
                      seqs: torch.Tensor = None, n_new: torch.Tensor = None, mask: torch.Tensor = None, scale: float = None,
                      max_len: int = 0, out: torch.Tensor = None, lse: torch.Tensor = None, workspace: torch.Tensor = None):
    """Attention of queries [B, N, q_heads, head_dim] over the committed tokens and the nodes they see.  Returns (out, lse); lse is only
    formed where a tensor [B, N, q_heads] fp32 is given for it."""
    rc = (_native or _calls()).attention(pool, page_table, lens, q, layer, seqs, n_new, mask, scale, max_len, out, lse, workspace, _stream)
    if rc is not None:
        _check(rc)
        return out, lse
    B, N, q_heads, D = q.shape
    c = _cache(pool, page_table, lens, head_dim=D, page_size=_page_size(pool, D))
    if out is None:
        out = torch.empty((B, N, q_heads, D), dtype=q.dtype, device=q.device)
    assert out.shape == q.shape and out.dtype == q.dtype
    if lse is not None:
        assert lse.dtype == torch.float32 and lse.shape == (B, N, q_heads) and lse.is_contiguous() and lse.is_cuda
    if mask is not None:
        assert mask.dtype == torch.int64 and mask.shape == (B, N, (N + 63) // 64) and mask.is_contiguous() and mask.is_cuda
    if workspace is None:
        workspace = alloc_attention_workspace(pool, page_table, q)
    _check(lib().mars_kv_attention(c, layer, _batch(seqs, lens, B), _rows(q, "q"), _dtype_code(q), q_heads, _table(n_new, (B,), "n_new"),
                                   _ptr(mask), 1.0 / math.sqrt(D) if scale is None else scale, max_len, _rows(out, "out"), _ptr(lse), B, N,
                                   workspace.data_ptr(), workspace.numel(), _stream()))
    return out, lse


def mars_kv_commit(pool: torch.Tensor, page_table: torch.Tensor, lens: torch.Tensor, accept_len: torch.Tensor, path_idx: torch.Tensor, *,
                   page_size: int, seqs: torch.Tensor = None, new_lens: torch.Tensor = None, status: torch.Tensor = None) -> torch.Tensor:
    """The accepted nodes' rows move up behind the committed tokens in every layer; returns the new lengths (``lens`` itself, updated, where no
    other tensor is given for them)."""
    if new_lens is None:
        new_lens = lens
    rc = (_native or _calls()).commit(pool, page_table, lens, accept_len, path_idx, page_size, seqs, new_lens, status, _stream)
    if rc is not None:
        _check(rc)
        return new_lens
    B, N = path_idx.shape
    c = _cache(pool, page_table, lens, page_size=page_size)
    _check(lib().mars_kv_commit(c, _batch(seqs, lens, B), _table(accept_len, (B,), "accept_len"), _table(path_idx, (B, N), "path_idx"), B, N,
                                _table(new_lens, lens.shape, "new_lens"), _table(status, (B,), "status"), _stream()))
    return new_lens


def alloc_reserve_workspace(pool: torch.Tensor, B: int) -> torch.Tensor:
    n = int(lib().mars_kv_reserve_workspace_bytes(pool.shape[1], B))
    if n == 0:
        raise MarsError(f"sizes out of range: pages={pool.shape[1]} B={B}")
    return torch.empty(n, dtype=torch.uint8, device=pool.device)


def mars_kv_reserve(pool: torch.Tensor, page_table: torch.Tensor, lens: torch.Tensor, held: torch.Tensor, refs: torch.Tensor, n, *,
                    page_size: int, seqs: torch.Tensor = None, status: torch.Tensor = None, workspace: torch.Tensor = None) -> torch.Tensor:
    """Room for n tokens (an int for all requests, or [B] int32) behind the committed ones; pages that others hold too are replaced where
    they would be written, by copies as far as committed tokens are in them.  Returns the status of every request."""
    rc = (_native or _calls()).reserve(pool, page_table, lens, held, refs, n, page_size, seqs, status, workspace, _stream)
    if rc is not None:
        _check(rc)
        return status
    n_new = n if isinstance(n, torch.Tensor) else None
    B = seqs.numel() if seqs is not None else n_new.numel() if n_new is not None else lens.numel()
    if status is None:
        status = torch.empty(B, dtype=torch.int32, device=lens.device)
    if workspace is None:
        workspace = alloc_reserve_workspace(pool, B)
    c = _cache(pool, page_table, lens, held, refs, page_size=page_size)
    _check(lib().mars_kv_reserve(c, _batch(seqs, lens, B), _table(n_new, (B,), "n"), B, (1 << 24) if n_new is not None else int(n),
                                 _table(status, (B,), "status"), workspace.data_ptr(), workspace.numel(), _stream()))
    return status


def mars_kv_fork(page_table: torch.Tensor, lens: torch.Tensor, held: torch.Tensor, refs: torch.Tensor, src: torch.Tensor, dst: torch.Tensor, *,
                 page_size: int, status: torch.Tensor = None) -> None:
    """Empty sequences dst[b] become copies of src[b] that share the pages of the committed tokens."""
    rc = (_native or _calls()).fork(page_table, lens, held, refs, src, dst, page_size, status, _stream)
    if rc is not None:
        return _check(rc)
    B = src.numel()
    c = _cache(None, page_table, lens, held, refs, page_size=page_size)
    _check(lib().mars_kv_fork(c, _table(src, (B,), "src"), _table(dst, (B,), "dst"), B, _table(status, (B,), "status"), _stream()))


def mars_kv_release(page_table: torch.Tensor, lens: torch.Tensor, held: torch.Tensor, refs: torch.Tensor, seqs: torch.Tensor, *,
                    status: torch.Tensor = None) -> None:
    """The sequences give their pages back."""
    rc = (_native or _calls()).release(page_table, lens, held, refs, seqs, status, _stream)
    if rc is not None:
        return _check(rc)
    B = seqs.numel()
    c = _cache(None, page_table, lens, held, refs, page_size=8)
    _check(lib().mars_kv_release(c, _table(seqs, (B,), "seqs"), B, _table(status, (B,), "status"), _stream()))


def mars_kv_copy_pages(pool: torch.Tensor, src: torch.Tensor, dst: torch.Tensor) -> None:
    """Pages src[i] into pages dst[i], in all layers."""
    n = src.numel()
    layers, pages, heads, blk = pool.shape
    assert pool.dtype == torch.uint8 and pool.is_contiguous() and pool.is_cuda
    D, P = next(((d, p) for d in HEAD_DIMS for p in (8, 16, 32, 64, 128, 256) if p * (d + d // 16) == blk), (0, 0))
    c = CacheStruct(_ptr(pool), None, None, None, None, layers, pages, heads, D, P, 1, 1)
    _check(lib().mars_kv_copy_pages(c, _table(src, (n,), "src"), _table(dst, (n,), "dst"), n, _stream()))
