"""Binding of libcobs.so's cache operators (include/cobs_cache.h): attention of several
query tokens a row (a draft's tree), accumulated attention weights, eviction and the
compaction of the cache.

Argument marshalling only, in the manner of ``cobs``, whose Config describes the
problem; its record fields are not read here.  The work runs on the current stream of
the tensors' GPU unless one is passed, also where another GPU is the current one.
"""

import ctypes

import torch

from . import cobs
from .cobs import CobsError, _KV, _check, _fits, _gpu, _kv, _kv_fits, _need, _opt, _ptr, _same_gpu, _stream, _units, _ws

MAX_QUERIES = 64           # per row and call (the bits of a tree mask word)

_P, _I, _Z = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
_SIGS = {
    "cobs_tree_workspace_bytes": (_Z, [_P, _I]),
    "cobs_tree_decode": (ctypes.c_int, [_P, _P, ctypes.c_int, _I, _P, _P, _P, _P, _I, _P, _P, _P, _P, _Z, _P]),
    "cobs_attention_weights": (ctypes.c_int, [_P, _P, ctypes.c_int, _I, _P, _P, _P, _P, _I, _P, _P, _P, _P, _P]),
    "cobs_evict_workspace_bytes": (_Z, [_P]),
    "cobs_evict": (ctypes.c_int, [_P, _P, _P, _I, _I, _I, _P, _P, _P, _Z, _P]),
    "cobs_compact_cache": (ctypes.c_int, [_P, _P, _P, _I, _I, _P, _P, _P, _I, _P, _P, _P]),
}
EXPORTS = tuple(_SIGS)

_IO = {torch.float32: cobs.F32, torch.bfloat16: cobs.BF16}
_lib = None


def lib():
    """The loaded library with the cache operators' signatures (raises if it has not been built)."""
    global _lib
    if _lib is None:
        h = cobs.lib()
        for name, (res, args) in _SIGS.items():
            fn = getattr(h, name)
            fn.restype = res
            fn.argtypes = args
        _lib = h
    return _lib


# (a tensor on a GPU has initialised torch's side, which torch.cuda.current_device looks after once more each time)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _call(fn, t, *args):
    """The C call on the GPU of tensor `t`, which becomes the current one for it where it is not."""
    if t.get_device() == _current_device():
        return _check(fn(*args))
    with torch.cuda.device(t.device):
        return _check(fn(*args))


def _struct(cfg):
    return cfg.marshalled()[0]


# As in ``cobs``, a call looks its arguments over in one pass; only when something does
# not fit do the separate checks run, which name the fault, or find that there is none.

def _cache_fits(cfg, dtype, dev, k, v, block_table, num_pages):
    """The C view of a cache on GPU `dev`, or None if anything does not fit."""
    if block_table is None:
        return _kv_fits(cfg, dtype, dev, k, v)
    shape = k.shape
    if (not _fits(dev, (k, dtype, 0), (v, dtype, 0), (block_table, torch.int32, cfg.batch * cfg.num_blocks)) or
            v.shape != shape or shape[1:] != (cfg.num_kv_heads, cfg.block_size, cfg.head_dim) or
            type(num_pages) is not int or not 1 <= num_pages <= shape[0]):
        return None
    return _KV(k.data_ptr(), v.data_ptr(), 0, 0, 0, block_table.data_ptr(), num_pages)


def _queries_alone_fit(cfg, q, seq_lens, draft_lens, tree_mask, sel, *more):
    """Whether the arguments of a call with queries fit, but for the cache; `more` as for _fits."""
    if (draft_lens is None) != (tree_mask is None):
        return False
    dev, shape = _gpu(q), q.shape
    if (len(shape) != 4 or shape[0] != cfg.batch or shape[2] != cfg.num_q_heads or shape[3] != cfg.head_dim or
            not 1 <= shape[1] <= MAX_QUERIES or q.dtype not in _IO or (tree_mask is not None and tree_mask.shape != shape[:2])):
        return False
    return _fits(dev, (q, q.dtype, 0), (seq_lens, torch.int32, cfg.batch), (draft_lens, torch.int32, cfg.batch),
                 (tree_mask, torch.int64, 0), (sel, torch.int32, _units(cfg) * cfg.budget), *more)


def _queries_fit(cfg, dtype, q, k, v, seq_lens, draft_lens, tree_mask, sel, block_table, num_pages, *more):
    """The C view of the cache if every argument of a call with queries fits, else None; `more` as for _fits."""
    if q is None or k is None or v is None or seq_lens is None:
        return None
    if not _queries_alone_fit(cfg, q, seq_lens, draft_lens, tree_mask, sel, *more):
        return None
    return _cache_fits(cfg, dtype, _gpu(q), k, v, block_table, num_pages)


def tree_workspace_bytes(cfg, num_queries):
    return int(lib().cobs_tree_workspace_bytes(ctypes.byref(_struct(cfg)), int(num_queries)))


def evict_workspace_bytes(cfg):
    return int(lib().cobs_evict_workspace_bytes(ctypes.byref(_struct(cfg))))


def new_tree_workspace(cfg, num_queries, device):
    return torch.empty(max(tree_workspace_bytes(cfg, num_queries), 256), dtype=torch.uint8, device=device)


def new_evict_workspace(cfg, device):
    return torch.empty(max(evict_workspace_bytes(cfg), 256), dtype=torch.uint8, device=device)


def _queries(cfg, q, seq_lens, draft_lens, tree_mask, sel):
    """Checks of what cobs_tree_decode and cobs_attention_weights share; the number of queries a row."""
    if q is None or q.dtype not in _IO:
        raise CobsError("q must be torch.float32 or torch.bfloat16")
    if q.dim() != 4 or q.shape[0] != cfg.batch or tuple(q.shape[2:]) != (cfg.num_q_heads, cfg.head_dim):
        raise CobsError(f"q must have shape [{cfg.batch}, N, {cfg.num_q_heads}, {cfg.head_dim}], got {list(q.shape)}")
    n = q.shape[1]
    if not 1 <= n <= MAX_QUERIES:
        raise CobsError(f"q must hold 1 to {MAX_QUERIES} queries a row, got {n}")
    _need("q", q, q.dtype, q.numel())
    _need("seq_lens", seq_lens, torch.int32, cfg.batch)
    if (draft_lens is None) != (tree_mask is None):
        raise CobsError("draft_lens and tree_mask go together")
    if tree_mask is not None:
        _need("draft_lens", draft_lens, torch.int32, cfg.batch)
        _need("tree_mask", tree_mask, torch.int64, cfg.batch * n)
        if tuple(tree_mask.shape) != (cfg.batch, n):
            raise CobsError(f"tree_mask must have shape [{cfg.batch}, {n}], got {list(tree_mask.shape)}")
    if sel is not None:
        _need("sel", sel, torch.int32, _units(cfg) * cfg.budget)
    return n


def cobs_tree_decode(cfg, q, k, v, seq_lens, draft_lens, tree_mask, out, ws, sel=None, lse=None, block_table=None,
                     num_pages=0, stream=None):
    """Attention of the N queries q [B, N, Hq, d] of each row over the cached context (sel None: all of it; else
    the selected blocks and the window) and the drafted tokens that tree_mask [B, N] (bit j: token j) lets them see."""
    c, _, kvt = cfg.marshalled()
    kv = None
    if out is not None and ws is not None:
        nq = q.numel() if isinstance(q, torch.Tensor) else 0
        kv = _queries_fit(cfg, kvt, q, k, v, seq_lens, draft_lens, tree_mask, sel, block_table, num_pages,
                          (out, getattr(q, "dtype", None), nq), (lse, torch.float32, nq // cfg.head_dim),
                          (ws, ws.dtype, 0))
    if kv is None:
        n = _queries(cfg, q, seq_lens, draft_lens, tree_mask, sel)
        _need("out", out, q.dtype, q.numel())
        _opt("lse", lse, torch.float32, cfg.batch * n * cfg.num_q_heads)
        kv = _kv(cfg, k, v, block_table, num_pages)
        _ws(ws)
        _same_gpu(q=q, k=k, v=v, seq_lens=seq_lens, draft_lens=draft_lens, tree_mask=tree_mask, sel=sel, out=out,
                  lse=lse, ws=ws, block_table=block_table)
    _call(lib().cobs_tree_decode, q, ctypes.byref(c), q.data_ptr(), _IO[q.dtype], q.shape[1], ctypes.byref(kv),
          seq_lens.data_ptr(), _ptr(draft_lens), _ptr(tree_mask), sel is not None, _ptr(sel) or None, out.data_ptr(),
          _ptr(lse), ws.data_ptr(), ws.numel() * ws.element_size(), _stream(stream, q))


def cobs_attention_weights(cfg, q, k, v, seq_lens, draft_lens, tree_mask, lse, weights, prev=None, sel=None,
                           block_table=None, num_pages=0, stream=None):
    """weights [B, Hkv, T_max] = prev + the attention weights that the queries give each cached token; lse
    [B, N, Hq] as the queries' attention returned it.  prev None: zeros; it may be `weights`."""
    c, _, kvt = cfg.marshalled()
    kv, nw = None, _units(cfg) * cfg.max_seq_len
    if lse is not None and weights is not None:
        nq = q.numel() if isinstance(q, torch.Tensor) else 0
        kv = _queries_fit(cfg, kvt, q, k, v, seq_lens, draft_lens, tree_mask, sel, block_table, num_pages,
                          (lse, torch.float32, nq // cfg.head_dim), (weights, torch.float32, nw),
                          (prev, torch.float32, nw))
    if kv is None:
        n = _queries(cfg, q, seq_lens, draft_lens, tree_mask, sel)
        _need("lse", lse, torch.float32, cfg.batch * n * cfg.num_q_heads)
        _need("weights", weights, torch.float32, nw)
        _opt("prev", prev, torch.float32, nw)
        kv = _kv(cfg, k, v, block_table, num_pages)
        _same_gpu(q=q, k=k, v=v, seq_lens=seq_lens, draft_lens=draft_lens, tree_mask=tree_mask, sel=sel, lse=lse,
                  weights=weights, prev=prev, block_table=block_table)
    _call(lib().cobs_attention_weights, q, ctypes.byref(c), q.data_ptr(), _IO[q.dtype], q.shape[1], ctypes.byref(kv),
          seq_lens.data_ptr(), _ptr(draft_lens), _ptr(tree_mask), sel is not None, _ptr(sel) or None, lse.data_ptr(),
          _ptr(prev), weights.data_ptr(), _stream(stream, q))


def cobs_evict(cfg, weights, seq_lens, kept, ws, sinks=0, recent=0, new_lens=None, stream=None):
    """The positions that each (batch row, KV head) keeps, kept [B, Hkv, keep]: the first `sinks`, the last
    `recent` and the heaviest between, ascending, then -1; new_lens [B]: how many."""
    c = _struct(cfg)
    nw = _units(cfg) * cfg.max_seq_len
    if (kept is None or weights is None or seq_lens is None or ws is None or
            kept.shape[:-1] != (cfg.batch, cfg.num_kv_heads) or
            not _fits(_gpu(kept), (kept, torch.int32, 0), (weights, torch.float32, nw), (seq_lens, torch.int32, cfg.batch),
                      (new_lens, torch.int32, cfg.batch), (ws, ws.dtype, 0))):
        if kept is None or kept.dim() != 3 or tuple(kept.shape[:2]) != (cfg.batch, cfg.num_kv_heads):
            raise CobsError(f"kept must have shape [{cfg.batch}, {cfg.num_kv_heads}, keep]")
        _need("kept", kept, torch.int32, kept.numel())
        _need("weights", weights, torch.float32, nw)
        _need("seq_lens", seq_lens, torch.int32, cfg.batch)
        _opt("new_lens", new_lens, torch.int32, cfg.batch)
        _ws(ws)
        _same_gpu(weights=weights, seq_lens=seq_lens, kept=kept, new_lens=new_lens, ws=ws)
    _call(lib().cobs_evict, kept, ctypes.byref(c), weights.data_ptr(), seq_lens.data_ptr(), kept.shape[2], int(sinks),
          int(recent), kept.data_ptr(), _ptr(new_lens), ws.data_ptr(), ws.numel() * ws.element_size(),
          _stream(stream, kept))


def _destination(cfg, k, k_out, v_out, table, num_pages):
    """C view and capacity of another cache that kept tokens move to."""
    for name, t in (("k_out", k_out), ("v_out", v_out)):
        if t is None or t.dtype != k.dtype or t.dim() != 4 or t.shape[-1] != cfg.head_dim or t.stride(-1) != 1:
            raise CobsError(f"{name} must be a 4-D {k.dtype} tensor with a dense head dimension of {cfg.head_dim}")
    if table is not None:
        for name, t in (("k_out", k_out), ("v_out", v_out)):
            if tuple(t.shape[1:]) != (cfg.num_kv_heads, cfg.block_size, cfg.head_dim) or not t.is_contiguous():
                raise CobsError(f"paged {name} must be a contiguous [pages, Hkv, L, d] pool")
            if not 1 <= int(num_pages) <= t.shape[0]:
                raise CobsError(f"out_num_pages must lie in [1, {t.shape[0]}]")
        if table.dim() != 2 or table.shape[0] != cfg.batch:
            raise CobsError(f"out_block_table must have shape [{cfg.batch}, blocks]")
        _need("out_block_table", table, torch.int32, table.numel())
        return (_KV(k_out.data_ptr(), v_out.data_ptr(), 0, 0, 0, table.data_ptr(), int(num_pages)),
                table.shape[1] * cfg.block_size)
    if k_out.stride() != v_out.stride() or k_out.shape != v_out.shape:
        raise CobsError("k_out and v_out must share shape and strides")
    if k_out.shape[0] < cfg.batch or k_out.shape[1] < cfg.num_kv_heads:
        raise CobsError(f"k_out of shape {tuple(k_out.shape)} is smaller than [{cfg.batch}, {cfg.num_kv_heads}, ...]")
    return (_KV(k_out.data_ptr(), v_out.data_ptr(), k_out.stride(0), k_out.stride(1), k_out.stride(2), None, 0),
            k_out.shape[2] // cfg.block_size * cfg.block_size)


def cobs_compact_cache(cfg, k, v, kept, seq_lens, first=None, k_out=None, v_out=None, weights=None, weights_out=None,
                       block_table=None, num_pages=0, out_block_table=None, out_num_pages=0, stream=None):
    """Move the tokens kept [B, Hkv, n] (or [B, n], one list for all heads) of each row to the positions
    first[b] + 0, 1, ...: in place, or into another cache k_out, v_out (contiguous or pages).  weights
    [B, Hkv, T_max] move to weights_out (in place: to themselves) and are 0 from the last moved token to seq_lens."""
    c, _, kvt = cfg.marshalled()
    kv = dst = None
    capacity, nw = cfg.max_seq_len, _units(cfg) * cfg.max_seq_len
    if kept is not None and k is not None and v is not None and seq_lens is not None and weights_out is not None:
        # another cache, with weights, everything in place
        dev, shape = _gpu(kept), kept.shape
        if (k_out is not None and v_out is not None and weights is not None and len(weights_out.shape) == 3 and
                (shape[:-1] == (cfg.batch, cfg.num_kv_heads) or shape[:-1] == (cfg.batch,)) and
                _fits(dev, (kept, torch.int32, 0), (seq_lens, torch.int32, cfg.batch), (first, torch.int32, cfg.batch),
                      (weights, torch.float32, nw), (weights_out, torch.float32, 0))):
            view = _out_fits(cfg, kvt, dev, k_out, v_out, out_block_table, out_num_pages)
            if view is not None and weights_out.shape == (cfg.batch, cfg.num_kv_heads, view[1]):
                kv = _cache_fits(cfg, kvt, dev, k, v, block_table, num_pages)
                if kv is not None:
                    dst, capacity = view
    if kv is None:
        kv, dst, capacity, weights_out = _compaction(cfg, k, v, kept, seq_lens, first, k_out, v_out, weights,
                                                     weights_out, block_table, num_pages, out_block_table, out_num_pages)
    _call(lib().cobs_compact_cache, kept, ctypes.byref(c), ctypes.byref(kv), _ptr(kept) or None, kept.dim() == 3,
          kept.shape[-1], seq_lens.data_ptr(), _ptr(first), None if dst is None else ctypes.byref(dst), capacity,
          _ptr(weights), _ptr(weights_out), _stream(stream, kept))


def _out_fits(cfg, dtype, dev, k_out, v_out, table, num_pages):
    """C view and capacity of another cache that kept tokens move to, or None if anything does not fit."""
    shape = k_out.shape
    if (k_out.dtype is not dtype or v_out.dtype is not dtype or len(shape) != 4 or v_out.shape != shape or
            k_out.get_device() != dev or v_out.get_device() != dev or shape[3] != cfg.head_dim):
        return None
    if table is None:
        stride = k_out.stride()
        if stride[3] != 1 or v_out.stride() != stride or shape[0] < cfg.batch or shape[1] < cfg.num_kv_heads:
            return None
        return (_KV(k_out.data_ptr(), v_out.data_ptr(), stride[0], stride[1], stride[2], None, 0),
                shape[2] // cfg.block_size * cfg.block_size)
    if (shape[1:] != (cfg.num_kv_heads, cfg.block_size, cfg.head_dim) or not k_out.is_contiguous() or
            not v_out.is_contiguous() or type(num_pages) is not int or not 1 <= num_pages <= shape[0] or
            len(table.shape) != 2 or table.shape[0] != cfg.batch or not _fits(dev, (table, torch.int32, 0))):
        return None
    return (_KV(k_out.data_ptr(), v_out.data_ptr(), 0, 0, 0, table.data_ptr(), num_pages),
            table.shape[1] * cfg.block_size)


def _compaction(cfg, k, v, kept, seq_lens, first, k_out, v_out, weights, weights_out, block_table, num_pages,
                out_block_table, out_num_pages):
    """The separate checks of cobs_compact_cache: C views, capacity and the weights' destination."""
    if kept is None or kept.dim() not in (2, 3) or tuple(kept.shape[:-1]) != (cfg.batch, cfg.num_kv_heads)[:kept.dim() - 1]:
        raise CobsError(f"kept must have shape [{cfg.batch}, {cfg.num_kv_heads}, n] or [{cfg.batch}, n]")
    _need("kept", kept, torch.int32, kept.numel())
    _need("seq_lens", seq_lens, torch.int32, cfg.batch)
    _opt("first", first, torch.int32, cfg.batch)
    kv = _kv(cfg, k, v, block_table, num_pages)
    if (k_out is None) != (v_out is None):
        raise CobsError("k_out and v_out go together")
    dst, capacity = None, cfg.max_seq_len
    if k_out is not None:
        dst, capacity = _destination(cfg, k, k_out, v_out, out_block_table, out_num_pages)
    elif out_block_table is not None:
        raise CobsError("out_block_table needs k_out and v_out")
    _opt("weights", weights, torch.float32, _units(cfg) * cfg.max_seq_len)
    if weights is None:
        if weights_out is not None:
            raise CobsError("weights_out needs weights")
    elif dst is None:
        if weights_out is not None and weights_out.data_ptr() != weights.data_ptr():
            raise CobsError("in place, weights move to themselves")
        weights_out = weights
    else:
        _need("weights_out", weights_out, torch.float32, _units(cfg) * capacity)
        if weights_out.dim() != 3 or weights_out.shape[2] != capacity:
            raise CobsError(f"weights_out must have shape [{cfg.batch}, {cfg.num_kv_heads}, {capacity}]")
    _same_gpu(kept=kept, k=k, v=v, seq_lens=seq_lens, first=first, k_out=k_out, v_out=v_out, weights=weights,
              weights_out=weights_out, block_table=block_table, out_block_table=out_block_table)
    return kv, dst, capacity, weights_out
