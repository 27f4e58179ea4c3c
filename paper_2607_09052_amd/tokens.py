"""Binding of libcobs.so's token operators (include/cobs_tokens.h): rotary positions, the append of
new tokens to a cache, and the cache of 8-bit floats with its append, attention and unpacking.

Argument marshalling only, in the manner of ``cobs`` and ``cache``.  Queries, keys and values of new
tokens are [B, N, heads, d] tensors of any strides with a dense head dimension, so the parts of one
projection's output go in as they are.
"""

import ctypes
import math
import struct
from typing import NamedTuple

import torch

from . import cobs
from .cache import _IO, _cache_fits, _call, _queries, _queries_alone_fit, _struct
from .cobs import CobsError, _fits, _gpu, _kv, _need, _opt, _ptr, _same_gpu, _stream, _ws

E4M3 = torch.float8_e4m3fn


# The C structs cobs_heads_t, cobs_rope_t and cobs_kv8_t, packed (a third of the time of a ctypes.Structure's making).
_pack_heads = struct.Struct("@Pqqq").pack
_pack_rope = struct.Struct("@Piif4x").pack
_pack_kv8 = struct.Struct("@PPPPqqqPq").pack

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
    """Zero-filled workspace of cobs_decode8 (the library requires zeros before first use)."""
    return torch.zeros(max(decode8_workspace_bytes(cfg, num_queries), 256), dtype=torch.uint8, device=device)


# As in ``cobs``, a call looks its arguments over in one pass; only when something does
# not fit do the separate checks run, which name the fault, or find that there is none.

def _heads_fit(t, dtype, dev, shape):
    """The C view of heads [B, N, H, d] on GPU `dev`, or None if anything does not fit."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev:
        return None
    b, n, h, e = t.stride()
    return _pack_heads(t.data_ptr(), b, n, h) if e == 1 else None


def _heads(name, t, dtype, shape):
    if t is None or t.dtype not in _IO or (dtype is not None and t.dtype != dtype):
        raise CobsError(f"{name} must be {dtype or 'torch.float32 or torch.bfloat16'}")
    if t.dim() != 4 or tuple(t.shape) != tuple(shape) or t.stride(-1) != 1:
        raise CobsError(f"{name} must have shape {list(shape)} with a dense head dimension, got {list(t.shape)}")
    return _pack_heads(t.data_ptr(), *t.stride()[:3])


def _rope_form(rope):
    freq, interleaved, scale = rope
    return _pack_rope(freq.data_ptr(), 2 * freq.numel(), bool(interleaved), float(scale))


def _rope(rope, positions, shape):
    """Checks of a rotation and its positions."""
    if not isinstance(rope, Rope):
        raise CobsError("rope must be a tokens.Rope")
    _need("inv_freq", rope.inv_freq, torch.float32, 1)
    if positions is not None:
        _need("positions", positions, torch.int32, shape[0] * shape[1])
        if tuple(positions.shape) != tuple(shape):
            raise CobsError(f"positions must have shape {list(shape)}, got {list(positions.shape)}")


def cobs_rotate(x, rope, positions, out, stream=None):
    """out [B, N, H, d] = x with the rotary positions `positions` [B, N] applied; out may be x."""
    hx = hy = None
    if x is not None and out is not None and positions is not None and type(rope) is Rope and len(x.shape) == 4:
        dev, shape = _gpu(x), x.shape
        if (x.dtype in _IO and out.dtype in _IO and positions.shape == shape[:2] and
                _fits(dev, (positions, torch.int32, 0), (rope[0], torch.float32, 1))):
            hx, hy = _heads_fit(x, x.dtype, dev, shape), _heads_fit(out, out.dtype, dev, shape)
    if hx is None or hy is None:
        if x is None or x.dim() != 4:
            raise CobsError("x must have shape [B, N, H, d]")
        shape = tuple(x.shape)
        hx, hy = _heads("x", x, None, shape), _heads("out", out, None, shape)
        if positions is None:
            raise CobsError("positions is required")
        _rope(rope, positions, shape[:2])
        _same_gpu(x=x, out=out, positions=positions, inv_freq=rope.inv_freq)
    _call(lib().cobs_rotate, x, hx, _IO[x.dtype], *shape, _rope_form(rope), positions.data_ptr(), hy, _IO[out.dtype],
          _stream(stream, x))


def _new_fit(cfg, dev, k_new, v_new, seq_lens, new_lens, rope, positions, q, q_out, new_seq_lens):
    """The C views (k_new, v_new, q, q_out, rope) of an append's arguments, or None if anything does not fit."""
    B, N, H, d = k_new.shape
    t = k_new.dtype
    if (t not in _IO or B != cfg.batch or H != cfg.num_kv_heads or d != cfg.head_dim or
            not _fits(dev, (seq_lens, torch.int32, B), (new_lens, torch.int32, B), (new_seq_lens, torch.int32, B),
                      (positions, torch.int32, 0))):
        return None
    r = hq = hy = None
    if rope is not None:
        if type(rope) is not Rope or not _fits(dev, (rope[0], torch.float32, 1)):
            return None
        r = _rope_form(rope)
    if positions is not None and (r is None or positions.shape != (B, N)):
        return None
    if q is not None or q_out is not None:
        if q is None or q_out is None or q_out.dtype not in _IO:
            return None
        shape = (B, N, cfg.num_q_heads, d)
        hq, hy = _heads_fit(q, t, dev, shape), _heads_fit(q_out, q_out.dtype, dev, shape)
        if hq is None or hy is None:
            return None
    hk, hv = _heads_fit(k_new, t, dev, k_new.shape), _heads_fit(v_new, t, dev, k_new.shape)
    return None if hk is None or hv is None else (hk, hv, hq, hy, r)


def _new(cfg, k_new, v_new, seq_lens, new_lens, rope, positions, q, q_out, new_seq_lens):
    """The separate checks of an append's arguments: their C views."""
    if k_new is None or k_new.dim() != 4:
        raise CobsError(f"k_new must have shape [{cfg.batch}, N, {cfg.num_kv_heads}, {cfg.head_dim}]")
    B, N, d = cfg.batch, k_new.shape[1], cfg.head_dim
    hk = _heads("k_new", k_new, None, (B, N, cfg.num_kv_heads, d))
    hv = _heads("v_new", v_new, k_new.dtype, (B, N, cfg.num_kv_heads, d))
    hq = hy = None
    if (q is None) != (q_out is None):
        raise CobsError("q and q_out go together")
    if q is not None:
        hq = _heads("q", q, k_new.dtype, (B, N, cfg.num_q_heads, d))
        hy = _heads("q_out", q_out, None, (B, N, cfg.num_q_heads, d))
    if rope is not None:
        _rope(rope, positions, (B, N))
    elif positions is not None:
        raise CobsError("positions needs rope")
    _need("seq_lens", seq_lens, torch.int32, B)
    _opt("new_lens", new_lens, torch.int32, B)
    _opt("new_seq_lens", new_seq_lens, torch.int32, B)
    return hk, hv, hq, hy, None if rope is None else _rope_form(rope)


def _append(fn, c, view, k_new, views, seq_lens, new_lens, positions, q_out, new_seq_lens, stream):
    hk, hv, hq, hy, r = views
    _call(fn, k_new, ctypes.byref(c), hk, hv, _IO[k_new.dtype], k_new.shape[1], view, seq_lens.data_ptr(), _ptr(new_lens), r,
          _ptr(positions), hq, hy, 0 if q_out is None else _IO[q_out.dtype], _ptr(new_seq_lens), _stream(stream, k_new))


def cobs_append(cfg, k_new, v_new, k, v, seq_lens, new_lens=None, rope=None, positions=None, q=None, q_out=None,
                new_seq_lens=None, block_table=None, num_pages=0, stream=None):
    """Tokens k_new, v_new [B, N, Hkv, d] behind the cache's seq_lens [B] tokens (new_lens [B] of the N; None: all), keys rotated;
    their queries q [B, N, Hq, d], rotated, to q_out; new_seq_lens [B]: the lengths after."""
    c, _, kvt = cfg.marshalled()
    kv = views = None
    if k_new is not None and v_new is not None and k is not None and v is not None and seq_lens is not None and len(k_new.shape) == 4:
        dev = _gpu(k_new)
        views = _new_fit(cfg, dev, k_new, v_new, seq_lens, new_lens, rope, positions, q, q_out, new_seq_lens)
        if views is not None:
            kv = _cache_fits(cfg, kvt, dev, k, v, block_table, num_pages)
    if kv is None:
        views = _new(cfg, k_new, v_new, seq_lens, new_lens, rope, positions, q, q_out, new_seq_lens)
        kv = _kv(cfg, k, v, block_table, num_pages)
        _same_gpu(k_new=k_new, v_new=v_new, seq_lens=seq_lens, new_lens=new_lens, new_seq_lens=new_seq_lens, q=q, q_out=q_out,
                  positions=positions, inv_freq=None if rope is None else rope.inv_freq, k=k, v=v, block_table=block_table)
    _append(lib().cobs_append, c, ctypes.byref(kv), k_new, views, seq_lens, new_lens, positions, q_out, new_seq_lens, stream)


def _cache8_fits(cfg, dev, cache8, block_table, num_pages):
    """The C view of an 8-bit cache on GPU `dev`, or None if anything does not fit."""
    if type(cache8) is not Cache8:
        return None
    k, v, ks, vs = cache8
    if k is None or v is None or ks is None or vs is None:
        return None
    shape, stride, t = k.shape, k.stride(), k.dtype
    if ((t is not E4M3 and t is not torch.uint8) or v.dtype is not t or len(shape) != 4 or v.shape != shape or
            v.stride() != stride or stride[3] != 1 or k.get_device() != dev or v.get_device() != dev or
            not _fits(dev, (ks, torch.float32, 0), (vs, torch.float32, 0))):
        return None
    H, L, d = cfg.num_kv_heads, cfg.block_size, cfg.head_dim
    if block_table is None:
        if (shape[0] < cfg.batch or shape[1] < H or shape[2] < cfg.max_seq_len or shape[3] != d or
                not ks.shape == vs.shape == (cfg.batch, H, cfg.max_seq_len // L)):
            return None
        return _pack_kv8(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), stride[0], stride[1], stride[2], 0, 0)
    if (shape != (shape[0], H, L, d) or not k.is_contiguous() or type(num_pages) is not int or not 1 <= num_pages <= shape[0] or
            not ks.shape == vs.shape == (shape[0], H) or not _fits(dev, (block_table, torch.int32, cfg.batch * cfg.num_blocks))):
        return None
    return _pack_kv8(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr(), 0, 0, 0, block_table.data_ptr(), num_pages)


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
    at = (k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr())
    if block_table is not None:
        return _pack_kv8(*at, 0, 0, 0, block_table.data_ptr(), int(num_pages))
    return _pack_kv8(*at, *k.stride()[:3], 0, 0)


def _of8(cache8, block_table):
    return dict(k=cache8.k, v=cache8.v, k_scale=cache8.k_scale, v_scale=cache8.v_scale, block_table=block_table)


def cobs_append8(cfg, k_new, v_new, cache8, seq_lens, new_lens=None, rope=None, positions=None, q=None, q_out=None,
                 new_seq_lens=None, block_table=None, num_pages=0, stream=None):
    """cobs_append into an 8-bit cache; a block whose scale grows has its earlier codes written anew."""
    c = _struct(cfg)
    view = views = None
    if k_new is not None and v_new is not None and seq_lens is not None and len(k_new.shape) == 4:
        dev = _gpu(k_new)
        views = _new_fit(cfg, dev, k_new, v_new, seq_lens, new_lens, rope, positions, q, q_out, new_seq_lens)
        if views is not None:
            view = _cache8_fits(cfg, dev, cache8, block_table, num_pages)
    if view is None:
        view = _cache8(cfg, cache8, block_table, num_pages)
        views = _new(cfg, k_new, v_new, seq_lens, new_lens, rope, positions, q, q_out, new_seq_lens)
        _same_gpu(k_new=k_new, v_new=v_new, seq_lens=seq_lens, new_lens=new_lens, new_seq_lens=new_seq_lens, q=q, q_out=q_out,
                  positions=positions, inv_freq=None if rope is None else rope.inv_freq, **_of8(cache8, block_table))
    _append(lib().cobs_append8, c, view, k_new, views, seq_lens, new_lens, positions, q_out, new_seq_lens, stream)


def cobs_decode8(cfg, q, cache8, seq_lens, draft_lens, tree_mask, out, ws, sel=None, lse=None, block_table=None,
                 num_pages=0, stream=None):
    """Attention of the N queries q [B, N, Hq, d] of each row over an 8-bit cache; arguments as for cache.cobs_tree_decode."""
    c = _struct(cfg)
    view = None
    if q is not None and out is not None and ws is not None and seq_lens is not None:
        nq, t = q.numel(), q.dtype
        if _queries_alone_fit(cfg, q, seq_lens, draft_lens, tree_mask, sel, (out, t, nq), (lse, torch.float32, nq // cfg.head_dim),
                        (ws, ws.dtype, 0)):
            view = _cache8_fits(cfg, _gpu(q), cache8, block_table, num_pages)
    if view is None:
        n = _queries(cfg, q, seq_lens, draft_lens, tree_mask, sel)
        _need("out", out, q.dtype, q.numel())
        _opt("lse", lse, torch.float32, cfg.batch * n * cfg.num_q_heads)
        view = _cache8(cfg, cache8, block_table, num_pages)
        _ws(ws)
        _same_gpu(q=q, seq_lens=seq_lens, draft_lens=draft_lens, tree_mask=tree_mask, sel=sel, out=out, lse=lse, ws=ws,
                  **_of8(cache8, block_table))
    _call(lib().cobs_decode8, q, ctypes.byref(c), q.data_ptr(), _IO[q.dtype], q.shape[1], view, seq_lens.data_ptr(),
          _ptr(draft_lens), _ptr(tree_mask), sel is not None, _ptr(sel) or None, out.data_ptr(), _ptr(lse), ws.data_ptr(),
          ws.numel() * ws.element_size(), _stream(stream, q))


def cobs_unpack8(cfg, cache8, seq_lens, k_out, v_out, first_block=0, num_blocks=None, last=None, block_table=None,
                 num_pages=0, out_block_table=None, out_num_pages=0, stream=None):
    """Blocks of an 8-bit cache as bf16 or fp32 (cfg.kv_dtype) in the same places of the cache k_out, v_out: num_blocks
    from first_block on (None: all), or the `last` blocks of each row."""
    c, _, kvt = cfg.marshalled()
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
    dst = view = None
    if seq_lens is not None and k_out is not None and v_out is not None and _fits(_gpu(seq_lens), (seq_lens, torch.int32, cfg.batch)):
        dev = _gpu(seq_lens)
        view = _cache8_fits(cfg, dev, cache8, block_table, num_pages)
        if view is not None:
            dst = _cache_fits(cfg, kvt, dev, k_out, v_out, out_block_table, out_num_pages)
    if dst is None:
        view = _cache8(cfg, cache8, block_table, num_pages)
        dst = _kv(cfg, k_out, v_out, out_block_table, out_num_pages)
        _need("seq_lens", seq_lens, torch.int32, cfg.batch)
        _same_gpu(seq_lens=seq_lens, k_out=k_out, v_out=v_out, out_block_table=out_block_table, **_of8(cache8, block_table))
    _call(lib().cobs_unpack8, seq_lens, ctypes.byref(c), view, seq_lens.data_ptr(), int(first_block), int(num_blocks),
          ctypes.byref(dst), _stream(stream, seq_lens))
