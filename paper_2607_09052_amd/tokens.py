"""Binding of libcobs.so's token operators (include/cobs_tokens.h): rotary positions, the append of
new tokens to a cache, and the cache of 8-bit floats with its append, attention and unpacking.

Argument marshalling only, in the manner of ``cobs`` and ``cache``.  Queries, keys and values of new
tokens are [B, N, heads, d] tensors of any strides with a dense head dimension, so the parts of one
projection's output go in as they are.
"""

import ctypes
import math
from typing import NamedTuple

import torch

from . import cobs
from .cache import _IO, _call, _queries, _struct
from .cobs import CobsError, _fits, _gpu, _kv, _need, _opt, _ptr, _same_gpu, _stream, _ws

E4M3 = torch.float8_e4m3fn


class _Heads(ctypes.Structure):
    _fields_ = [("p", ctypes.c_void_p), ("stride_b", ctypes.c_int64), ("stride_n", ctypes.c_int64),
                ("stride_h", ctypes.c_int64)]


class _Rope(ctypes.Structure):
    _fields_ = [("inv_freq", ctypes.c_void_p), ("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("scale", ctypes.c_float)]


class _KV8(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64), ("stride_t", ctypes.c_int64),
                ("block_table", ctypes.c_void_p), ("num_pages", ctypes.c_int64)]


_P, _I, _Z, _E = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t, ctypes.c_int
_APPEND = [_P, _P, _P, _E, _I, _P, _P, _P, _P, _P, _P, _P, _E, _P, _P]
_SIGS = {
    "cobs_rotate": (_E, [_P, _E, _I, _I, _I, _I, _P, _P, _P, _E, _P]),
    "cobs_append": (_E, _APPEND),
    "cobs_append8": (_E, _APPEND),
    "cobs_decode8_workspace_bytes": (_Z, [_P, _I]),
    "cobs_decode8": (_E, [_P, _P, _E, _I, _P, _P, _P, _P, _I, _P, _P, _P, _P, _Z, _P]),
    "cobs_unpack8": (_E, [_P, _P, _P, _I, _I, _P, _P]),
}
EXPORTS = tuple(_SIGS)
_lib = None


def lib():
    """The loaded library with the token operators' signatures (raises if it has not been built)."""
    global _lib
    if _lib is None:
        h = cobs.lib()
        for name, (res, args) in _SIGS.items():
            fn = getattr(h, name)
            fn.restype = res
            fn.argtypes = args
        _lib = h
    return _lib


class Rope(NamedTuple):
    """Rotary positions (cobs_rope_t): frequencies fp32 [r / 2] on the GPU, pairs side by side (interleaved) or half
    a rotated part apart, a factor on the rotated elements."""
    inv_freq: torch.Tensor
    interleaved: bool = False
    scale: float = 1.0


class Cache8(NamedTuple):
    """An 8-bit cache (cobs_kv8_t): codes float8_e4m3fn (or uint8) [>=B, >=Hkv, >=T_max, d] with a dense head dimension, scales fp32
    [B, Hkv, T_max / L]; or pages: codes [pages, Hkv, L, d], scales [pages, Hkv]."""
    k: torch.Tensor
    v: torch.Tensor
    k_scale: torch.Tensor
    v_scale: torch.Tensor


def rope_frequencies(rotary_dim, base=10000.0, factor=1.0, original_len=None, slow=1.0, fast=32.0, device=None):
    """Frequencies base^(-2p / r) of the pairs p < r / 2, scaled for contexts `factor` times as long: all divided by it,
    or, with the original context length, by parts: pairs of at most `slow` turns over it are divided, those of `fast`
    turns and more are kept, and a linear ramp over the turns lies between."""
    f = float(base) ** (-torch.arange(rotary_dim // 2, dtype=torch.float64) * 2.0 / rotary_dim)
    keep = torch.zeros_like(f)
    if original_len is not None:
        keep = ((original_len * f / (2.0 * math.pi) - slow) / (fast - slow)).clamp(0.0, 1.0)
    return (f * (keep + (1.0 - keep) / factor)).float().to(device or "cpu")


def new_cache8(cfg, device, num_pages=0):
    """A zero-filled 8-bit cache of the configuration: contiguous, or a pool of pages."""
    if num_pages:
        shape, scales = (num_pages, cfg.num_kv_heads, cfg.block_size, cfg.head_dim), (num_pages, cfg.num_kv_heads)
    else:
        shape = (cfg.batch, cfg.num_kv_heads, cfg.max_seq_len, cfg.head_dim)
        scales = (cfg.batch, cfg.num_kv_heads, cfg.num_blocks)
    k, v = (torch.zeros(shape, dtype=torch.uint8, device=device).view(E4M3) for _ in range(2))
    return Cache8(k, v, *(torch.zeros(scales, dtype=torch.float32, device=device) for _ in range(2)))


def decode8_workspace_bytes(cfg, num_queries):
    return int(lib().cobs_decode8_workspace_bytes(ctypes.byref(_struct(cfg)), int(num_queries)))


def new_decode8_workspace(cfg, num_queries, device):
    return torch.empty(max(decode8_workspace_bytes(cfg, num_queries), 256), dtype=torch.uint8, device=device)


# As in ``cobs``, a call looks its arguments over in one pass; only when something does
# not fit do the separate checks run, which name the fault, or find that there is none.

def _heads_fit(t, dtype, dev, shape):
    """The C view of heads [B, N, H, d] on GPU `dev`, or None if anything does not fit."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev:
        return None
    s = t.stride()
    if s[3] != 1:
        return None
    return _Heads(t.data_ptr(), s[0] if shape[0] > 1 else 0, s[1] if shape[1] > 1 else 0, s[2] if shape[2] > 1 else 0)


def _heads(name, t, dtype, shape):
    if t is None or t.dtype not in _IO or (dtype is not None and t.dtype != dtype):
        raise CobsError(f"{name} must be {dtype or 'torch.float32 or torch.bfloat16'}")
    if t.dim() != 4 or tuple(t.shape) != tuple(shape) or t.stride(-1) != 1:
        raise CobsError(f"{name} must have shape {list(shape)} with a dense head dimension, got {list(t.shape)}")
    return _Heads(t.data_ptr(), *(s if n > 1 else 0 for s, n in zip(t.stride()[:3], t.shape[:3])))


def _rope(rope, positions, tokens):
    """The C form of a rotation whose tensors fit, and its tensors."""
    if not isinstance(rope, Rope):
        raise CobsError("rope must be a tokens.Rope")
    _need("inv_freq", rope.inv_freq, torch.float32, 1)
    if positions is not None:
        _need("positions", positions, torch.int32, tokens)
    return _Rope(rope.inv_freq.data_ptr(), 2 * rope.inv_freq.numel(), bool(rope.interleaved), float(rope.scale))


def cobs_rotate(x, rope, positions, out, stream=None):
    """out [B, N, H, d] = x with the rotary positions `positions` [B, N] applied; out may be x."""
    if x is None or x.dim() != 4:
        raise CobsError("x must have shape [B, N, H, d]")
    shape = tuple(x.shape)
    hx = _heads("x", x, None, shape)
    hy = _heads("out", out, None, shape)
    if positions is None:
        raise CobsError("positions is required")
    r = _rope(rope, positions, shape[0] * shape[1])
    if tuple(positions.shape) != shape[:2]:
        raise CobsError(f"positions must have shape {list(shape[:2])}, got {list(positions.shape)}")
    _same_gpu(x=x, out=out, positions=positions, inv_freq=rope.inv_freq)
    _call(lib().cobs_rotate, x, ctypes.byref(hx), _IO[x.dtype], *shape, ctypes.byref(r), positions.data_ptr(),
          ctypes.byref(hy), _IO[out.dtype], _stream(stream, x))


def _append(fn, cfg, c, view, k_new, v_new, tensors, seq_lens, new_lens, rope, positions, q, q_out, new_seq_lens, stream):
    """The call of cobs_append and cobs_append8 into the cache of C form `view` and of `tensors`."""
    if k_new is None or v_new is None or k_new.dim() != 4:
        raise CobsError(f"k_new must have shape [{cfg.batch}, N, {cfg.num_kv_heads}, {cfg.head_dim}]")
    B, N, d = cfg.batch, k_new.shape[1], cfg.head_dim
    hk = _heads("k_new", k_new, None, (B, N, cfg.num_kv_heads, d))
    hv = _heads("v_new", v_new, k_new.dtype, (B, N, cfg.num_kv_heads, d))
    hq = hy = r = None
    if (q is None) != (q_out is None):
        raise CobsError("q and q_out go together")
    if q is not None:
        hq = _heads("q", q, k_new.dtype, (B, N, cfg.num_q_heads, d))
        hy = _heads("q_out", q_out, None, (B, N, cfg.num_q_heads, d))
    if rope is not None:
        r = _rope(rope, positions, B * N)
        if positions is not None and tuple(positions.shape) != (B, N):
            raise CobsError(f"positions must have shape [{B}, {N}], got {list(positions.shape)}")
    elif positions is not None:
        raise CobsError("positions needs rope")
    dev = _gpu(k_new)
    if not _fits(dev, (seq_lens, torch.int32, B), (new_lens, torch.int32, B), (new_seq_lens, torch.int32, B)) or seq_lens is None:
        _need("seq_lens", seq_lens, torch.int32, B)
        _opt("new_lens", new_lens, torch.int32, B)
        _opt("new_seq_lens", new_seq_lens, torch.int32, B)
    _same_gpu(k_new=k_new, v_new=v_new, seq_lens=seq_lens, new_lens=new_lens, new_seq_lens=new_seq_lens, q=q, q_out=q_out,
              positions=positions, inv_freq=None if rope is None else rope.inv_freq, **tensors)
    _call(fn, k_new, ctypes.byref(c), ctypes.byref(hk), ctypes.byref(hv), _IO[k_new.dtype], N, ctypes.byref(view),
          seq_lens.data_ptr(), _ptr(new_lens), None if r is None else ctypes.byref(r), _ptr(positions),
          None if hq is None else ctypes.byref(hq), None if hy is None else ctypes.byref(hy),
          0 if q_out is None else _IO[q_out.dtype], _ptr(new_seq_lens), _stream(stream, k_new))


def cobs_append(cfg, k_new, v_new, k, v, seq_lens, new_lens=None, rope=None, positions=None, q=None, q_out=None,
                new_seq_lens=None, block_table=None, num_pages=0, stream=None):
    """Tokens k_new, v_new [B, N, Hkv, d] behind the cache's seq_lens [B] tokens (new_lens [B] of the N; None: all), keys rotated;
    their queries q [B, N, Hq, d], rotated, to q_out; new_seq_lens [B]: the lengths after."""
    c = _struct(cfg)
    _append(lib().cobs_append, cfg, c, _kv(cfg, k, v, block_table, num_pages), k_new, v_new,
            dict(k=k, v=v, block_table=block_table), seq_lens, new_lens, rope, positions, q, q_out, new_seq_lens, stream)


def _cache8(cfg, cache8, block_table, num_pages):
    """Validated C view of an 8-bit cache."""
    if not isinstance(cache8, Cache8):
        raise CobsError("cache8 must be a tokens.Cache8")
    k, v, ks, vs = cache8
    for name, t in (("k", k), ("v", v)):
        if t is None or t.dtype not in (E4M3, torch.uint8):
            raise CobsError(f"8-bit {name} must be {E4M3} or torch.uint8")
        if t.dim() != 4 or t.shape[-1] != cfg.head_dim or t.stride(-1) != 1:
            raise CobsError(f"8-bit {name} must be 4-D with a dense head dimension of {cfg.head_dim}")
    if block_table is not None:
        for name, t in (("k", k), ("v", v)):
            if tuple(t.shape[1:]) != (cfg.num_kv_heads, cfg.block_size, cfg.head_dim) or not t.is_contiguous():
                raise CobsError(f"paged 8-bit {name} must be a contiguous [pages, Hkv, L, d] pool")
            if not 1 <= int(num_pages) <= t.shape[0]:
                raise CobsError(f"num_pages must lie in [1, {t.shape[0]}]")
        _need("block_table", block_table, torch.int32, cfg.batch * cfg.num_blocks)
        want = (int(num_pages), cfg.num_kv_heads)
    else:
        if k.stride() != v.stride() or k.shape != v.shape:
            raise CobsError("8-bit K and V must share shape and strides")
        if k.shape[0] < cfg.batch or k.shape[1] < cfg.num_kv_heads or k.shape[2] < cfg.max_seq_len:
            raise CobsError(f"8-bit K/V of shape {tuple(k.shape)} is smaller than "
                            f"[{cfg.batch}, {cfg.num_kv_heads}, {cfg.max_seq_len}, {cfg.head_dim}]")
        want = (cfg.batch, cfg.num_kv_heads, cfg.num_blocks)
    for name, t in (("k_scale", ks), ("v_scale", vs)):
        _need(name, t, torch.float32, math.prod(want))
        if t.dim() != len(want) or tuple(t.shape[1:]) != want[1:]:
            raise CobsError(f"{name} must have shape {list(want)}, got {list(t.shape)}")
    if block_table is not None:
        return _KV8(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), 0, 0, 0, block_table.data_ptr(), int(num_pages))
    return _KV8(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), k.stride(0), k.stride(1), k.stride(2), None, 0)


def _of8(cache8, block_table):
    return dict(k=cache8.k, v=cache8.v, k_scale=cache8.k_scale, v_scale=cache8.v_scale, block_table=block_table)


def cobs_append8(cfg, k_new, v_new, cache8, seq_lens, new_lens=None, rope=None, positions=None, q=None, q_out=None,
                 new_seq_lens=None, block_table=None, num_pages=0, stream=None):
    """cobs_append into an 8-bit cache; a block whose scale grows has its earlier codes written anew."""
    c = _struct(cfg)
    view = _cache8(cfg, cache8, block_table, num_pages)
    _append(lib().cobs_append8, cfg, c, view, k_new, v_new, _of8(cache8, block_table), seq_lens, new_lens, rope, positions,
            q, q_out, new_seq_lens, stream)


def cobs_decode8(cfg, q, cache8, seq_lens, draft_lens, tree_mask, out, ws, sel=None, lse=None, block_table=None,
                 num_pages=0, stream=None):
    """Attention of the N queries q [B, N, Hq, d] of each row over an 8-bit cache; arguments as for cache.cobs_tree_decode."""
    c = _struct(cfg)
    n = _queries(cfg, q, seq_lens, draft_lens, tree_mask, sel)
    _need("out", out, q.dtype, q.numel())
    _opt("lse", lse, torch.float32, cfg.batch * n * cfg.num_q_heads)
    view = _cache8(cfg, cache8, block_table, num_pages)
    nws = _ws(ws)
    _same_gpu(q=q, seq_lens=seq_lens, draft_lens=draft_lens, tree_mask=tree_mask, sel=sel, out=out, lse=lse, ws=ws,
              **_of8(cache8, block_table))
    _call(lib().cobs_decode8, q, ctypes.byref(c), q.data_ptr(), _IO[q.dtype], n, ctypes.byref(view), seq_lens.data_ptr(),
          _ptr(draft_lens), _ptr(tree_mask), sel is not None, _ptr(sel) or None, out.data_ptr(), _ptr(lse), ws.data_ptr(), nws,
          _stream(stream, q))


def cobs_unpack8(cfg, cache8, seq_lens, k_out, v_out, first_block=0, num_blocks=None, last=None, block_table=None,
                 num_pages=0, out_block_table=None, out_num_pages=0, stream=None):
    """Blocks of an 8-bit cache as bf16 or fp32 (cfg.kv_dtype) in the same places of the cache k_out, v_out: num_blocks
    from first_block on (None: all), or the `last` blocks of each row."""
    c = _struct(cfg)
    view = _cache8(cfg, cache8, block_table, num_pages)
    dst = _kv(cfg, k_out, v_out, out_block_table, out_num_pages)
    _need("seq_lens", seq_lens, torch.int32, cfg.batch)
    if last is not None:
        if first_block != 0 or num_blocks is not None:
            raise CobsError("last stands for itself, without first_block and num_blocks")
        if last < 0:
            raise CobsError("last must not be negative")
        first_block, num_blocks = -1, min(int(last), cfg.num_blocks)
    elif first_block < 0:
        raise CobsError("first_block must not be negative")
    elif num_blocks is None:
        num_blocks = cfg.num_blocks - first_block
    _same_gpu(seq_lens=seq_lens, k_out=k_out, v_out=v_out, out_block_table=out_block_table, **_of8(cache8, block_table))
    _call(lib().cobs_unpack8, seq_lens, ctypes.byref(c), ctypes.byref(view), seq_lens.data_ptr(), int(first_block),
          int(num_blocks), ctypes.byref(dst), _stream(stream, seq_lens))
