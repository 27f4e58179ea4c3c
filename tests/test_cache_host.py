"""The cache operators without a GPU: the oracle's identities, and the refusals of the C entry points and
of the binding, which come before any launch."""

import ctypes
import os
import re

import numpy as np
import pytest
import torch

from oracle import cache as O
from oracle import method as M
from paper_2607_09052_amd import cache, cobs

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# ------------------------------------------------------------------ oracle --
def _random(N=3, G=2, d=8, T=40, n=3, seed=0):
    r = np.random.default_rng(seed)
    return r.normal(size=(N, G, d)), r.normal(size=(T + n, d)), r.normal(size=(T + n, d))


def test_one_query_without_a_draft_is_the_decode_attention():
    q, K, V = _random(N=1, T=200, n=0, d=16)
    sel = [0, 2]
    see = O.visible(200, 0, 1, 32, 50, sel)
    out, lse = O.tree_attention(q, K, V, see, 0.25)
    want, wl = M.sparse_attention(q[0], K, V, M.union_tokens(200, 32, 50, sel), 0.25)
    assert np.allclose(out[0], want, atol=1e-12) and np.allclose(lse[0], wl, atol=1e-12)


def test_a_chain_draft_is_causal_attention():
    q, K, V = _random(N=3, T=5, n=3)
    out, lse = O.tree_attention(q, K, V, O.visible(5, 3, 3, 32, 0, None, [1, 3, 7]), 0.3)
    for i in range(3):
        want, wl = M.sparse_attention(q[i], K, V, range(5 + i + 1), 0.3)
        assert np.allclose(out[i], want, atol=1e-12) and np.allclose(lse[i], wl, atol=1e-12)


def test_weights_of_a_softmax_sum_to_one_per_query_head():
    q, K, V = _random(N=4, T=30, n=4)
    see = O.visible(30, 4, 4, 32, 0, None, [1, 3, 5, 0])
    _, lse = O.tree_attention(q, K, V, see, 0.3)
    w = O.attention_weights(q, K, see, lse, 0.3)
    assert abs(w.sum() - 4 * 2) < 1e-12
    lse[2] = np.inf                                  # a query left out
    assert abs(O.attention_weights(q, K, see, lse, 0.3).sum() - 3 * 2) < 1e-12


def test_values_that_a_query_does_not_see_do_not_reach_it():
    q, K, V = _random(N=2, T=3, n=2)
    K[4], V[4] = np.nan, np.inf
    see = O.visible(3, 2, 2, 32, 0, None, [1, 1])
    out, lse = O.tree_attention(q, K, V, see, 0.3)
    assert np.isfinite(out).all() and np.isfinite(lse).all()


def test_eviction_keeps_ends_and_the_heaviest():
    w = [5.0, 1.0, 2.0, 2.0, np.nan, 2.0, 0.0, 9.0]
    assert O.evict(w, 8, 8, 0, 0) == list(range(8))
    assert O.evict(w, 8, 4, 1, 1) == [0, 2, 3, 7]    # ties to the lower position
    assert O.evict(w, 8, 7, 0, 0) == [0, 1, 2, 3, 5, 6, 7]
    assert O.evict(w, 8, 3, 1, 2) == [0, 6, 7]
    assert O.compact_weights(w, list(w), [0, 2, 3], 8, 1)[1:] == [5.0, 2.0, 2.0, 0.0, 0.0, 0.0, 0.0]


# ---------------------------------------------------------------- refusals --
def test_library_exports_what_the_header_declares():
    with open(os.path.join(ROOT, "include", "cobs_cache.h")) as f:
        declared = sorted(set(re.findall(r"^\s*(?:size_t|cobs_status_t)\s+(cobs_\w+)\s*\(", f.read(), re.M)))
    assert declared == sorted(cache.EXPORTS)
    for name in declared:
        assert hasattr(cobs.lib(), name)


def _cfg(**over):
    base = dict(batch=2, num_q_heads=8, num_kv_heads=2, head_dim=128, max_seq_len=4096, rank=0, budget=8, window=128)
    base.update(over)
    return cobs.Config(**base)


FAKE, OTHER = 1 << 20, 1 << 24


def _kv(**over):
    base = dict(k=FAKE, v=FAKE + 4096, stride_b=1 << 20, stride_h=1 << 19, stride_t=128, block_table=None, num_pages=0)
    base.update(over)
    return cobs._KV(*base.values())


def _tree(cfg=None, kv=None, **over):
    cfg = _cfg().c_struct() if cfg is None else cfg
    kv = _kv() if kv is None else kv
    a = dict(q=FAKE, io=0, N=8, seq=FAKE, drafts=FAKE, mask=FAKE, sparse=1, sel=FAKE, out=OTHER, lse=FAKE, ws=FAKE,
             nws=1 << 40)
    a.update(over)
    return cache.lib().cobs_tree_decode(
        ctypes.byref(cfg), a["q"], a["io"], a["N"], ctypes.byref(kv), a["seq"], a["drafts"], a["mask"], a["sparse"],
        a["sel"], a["out"], a["lse"], a["ws"], a["nws"], None)


def _weights(cfg=None, kv=None, **over):
    cfg = _cfg().c_struct() if cfg is None else cfg
    kv = _kv() if kv is None else kv
    a = dict(q=FAKE, io=0, N=8, seq=FAKE, drafts=FAKE, mask=FAKE, sparse=1, sel=FAKE, lse=FAKE, prev=None, w=OTHER)
    a.update(over)
    return cache.lib().cobs_attention_weights(
        ctypes.byref(cfg), a["q"], a["io"], a["N"], ctypes.byref(kv), a["seq"], a["drafts"], a["mask"], a["sparse"],
        a["sel"], a["lse"], a["prev"], a["w"], None)


SHARED = [
    (dict(q=None), 1), (dict(q=FAKE + 4), 1), (dict(seq=None), 1),
    (dict(drafts=None), 1), (dict(mask=None), 1), (dict(mask=FAKE + 4), 1),
    (dict(sel=None), 1),                       # sparse with a budget
    (dict(sparse=0), 1),                       # a selection without sparse
    (dict(sparse=2), 1),
    (dict(io=2), 1), (dict(io=7), 1),
    (dict(N=0), 1), (dict(N=-1), 1), (dict(N=65), 2),
]


@pytest.mark.parametrize("edit,code", SHARED + [
    (dict(out=None), 1), (dict(out=OTHER + 8), 1), (dict(out=FAKE), 1),
    (dict(ws=None), 3), (dict(ws=FAKE + 64), 3), (dict(nws=0), 3),
])
def test_tree_decode_refuses(edit, code):
    assert _tree(**edit) == code


@pytest.mark.parametrize("edit,code", SHARED + [(dict(lse=None), 1), (dict(w=None), 1)])
def test_attention_weights_refuse(edit, code):
    assert _weights(**edit) == code


BAD_CONFIGS = [
    (dict(batch=0), 1), (dict(num_q_heads=7), 1), (dict(num_kv_heads=0), 1), (dict(max_seq_len=100), 1),
    (dict(budget=-1), 1), (dict(window=-1), 1), (dict(softmax_scale=-1.0), 1), (dict(softmax_scale=float("nan")), 1),
    (dict(num_q_heads=6), 2), (dict(head_dim=96), 2), (dict(block_size=16), 2),
    (dict(max_seq_len=64 * 8193), 2), (dict(batch=65536), 2), (dict(batch=65535, num_q_heads=128, num_kv_heads=8), 2),
]


@pytest.mark.parametrize("edit,code", BAD_CONFIGS)
def test_configs_are_refused(edit, code):
    cfg = _cfg().c_struct()
    for k, v in edit.items():
        setattr(cfg, k, v)
    lib = cache.lib()
    kv, w = _kv(), ctypes.c_void_p(FAKE)
    assert _tree(cfg) == code and _weights(cfg) == code
    assert lib.cobs_evict(ctypes.byref(cfg), w, w, 8, 0, 0, w, None, w, 1 << 40, None) == code
    assert lib.cobs_compact_cache(ctypes.byref(cfg), ctypes.byref(kv), w, 1, 8, w, None, None, cfg.max_seq_len, None,
                                  None, None) == code
    assert lib.cobs_tree_workspace_bytes(ctypes.byref(cfg), 8) == 0
    assert lib.cobs_evict_workspace_bytes(ctypes.byref(cfg)) == 0


@pytest.mark.parametrize("edit,code", [
    (dict(k=None), 1), (dict(v=None), 1), (dict(k=FAKE + 8), 1), (dict(v=FAKE + 4), 1),
    (dict(stride_t=64), 1), (dict(stride_t=132), 1), (dict(stride_h=-8), 1), (dict(stride_b=4), 1),
    (dict(stride_t=(1 << 22) + 8), 2), (dict(block_table=FAKE, num_pages=0), 1),
])
def test_caches_are_refused(edit, code):
    kv, lib, w, cfg = _kv(**edit), cache.lib(), ctypes.c_void_p(FAKE), _cfg().c_struct()
    assert _tree(kv=kv) == code and _weights(kv=kv) == code
    good = _kv(k=OTHER, v=OTHER + 4096)
    for a, b in ((kv, None), (kv, good), (good, kv)):
        assert lib.cobs_compact_cache(ctypes.byref(cfg), ctypes.byref(a), w, 1, 8, w, None, b and ctypes.byref(b), 4096,
                                      None, None, None) == code


@pytest.mark.parametrize("edit", [
    dict(weights=None), dict(seq=None), dict(kept=None), dict(new=FAKE), dict(keep=0), dict(keep=4097), dict(sinks=-1),
    dict(recent=-1), dict(sinks=9), dict(recent=9), dict(sinks=5, recent=4), dict(sinks=2 ** 31 - 1, recent=2 ** 31 - 1),
])
def test_evict_refuses(edit):
    a = dict(weights=OTHER, seq=FAKE, keep=8, sinks=1, recent=2, kept=OTHER, new=None)
    a.update(edit)
    cfg = _cfg().c_struct()
    assert cache.lib().cobs_evict(ctypes.byref(cfg), a["weights"], a["seq"], a["keep"], a["sinks"], a["recent"],
                                  a["kept"], a["new"], FAKE, 1 << 40, None) == 1


@pytest.mark.parametrize("edit,code", [
    (dict(kept=None), 1), (dict(seq=None), 1), (dict(n=-1), 1), (dict(n=4097), 1), (dict(per_head=2), 1),
    (dict(cap=0), 1), (dict(cap=4095), 1), (dict(cap=64 * 8193), 2),
    (dict(dst=None, cap=64), 1),                       # in place the capacity is the cache's
    (dict(dst=_kv()), 1), (dict(dst=_kv(v=OTHER)), 1),  # the same memory as another cache
    (dict(dst=_kv(k=FAKE + 4096, v=OTHER)), 1),
    (dict(dst=_kv(block_table=FAKE, num_pages=4)), 1),  # the same pool, the source not in pages
    (dict(dst=_kv(k=OTHER, v=OTHER + 4096, stride_b=0)), 1), (dict(dst=_kv(k=OTHER, v=OTHER + 4096, stride_h=0)), 1),
    (dict(w=FAKE), 1), (dict(wo=FAKE), 1), (dict(w=FAKE, wo=FAKE), 1), (dict(dst=None, w=FAKE, wo=OTHER), 1),
])
def test_compact_refuses(edit, code):
    a = dict(kept=FAKE, per_head=1, n=8, seq=FAKE, first=None, dst=_kv(k=OTHER, v=OTHER + 4096), cap=4096, w=None, wo=None)
    a.update(edit)
    cfg, kv = _cfg().c_struct(), _kv()
    assert cache.lib().cobs_compact_cache(
        ctypes.byref(cfg), ctypes.byref(kv), a["kept"], a["per_head"], a["n"], a["seq"], a["first"],
        None if a["dst"] is None else ctypes.byref(a["dst"]), a["cap"], a["w"], a["wo"], None) == code


def test_compaction_in_place_refuses_rows_that_share_memory_and_one_table_for_both():
    cfg, lib, w = _cfg().c_struct(), cache.lib(), ctypes.c_void_p(FAKE)
    for kv in (_kv(stride_b=0), _kv(stride_h=0)):
        assert lib.cobs_compact_cache(ctypes.byref(cfg), ctypes.byref(kv), w, 1, 8, w, None, None, 4096, None, None, None) == 1
    kv, dst = (_kv(block_table=FAKE, num_pages=9) for _ in range(2))
    assert lib.cobs_compact_cache(ctypes.byref(cfg), ctypes.byref(kv), w, 1, 8, w, None, ctypes.byref(dst), 4096, None, None,
                                  None) == 1


# ----------------------------------------------------------------- binding --
def _tensors(B=2, N=3, Hkv=2, G=4, d=128, T=128):
    t = dict(q=torch.zeros(B, N, Hkv * G, d), k=torch.zeros(B, Hkv, T, d, dtype=torch.bfloat16),
             v=torch.zeros(B, Hkv, T, d, dtype=torch.bfloat16), seq_lens=torch.zeros(B, dtype=torch.int32),
             draft_lens=torch.zeros(B, dtype=torch.int32), tree_mask=torch.zeros(B, N, dtype=torch.int64),
             out=torch.zeros(B, N, Hkv * G, d), ws=torch.zeros(1 << 20, dtype=torch.uint8))
    return _cfg(max_seq_len=T), t


@pytest.mark.parametrize("edit,text", [
    (dict(q=torch.zeros(2, 3, 8, 128, dtype=torch.float16)), "q must be"), (dict(q=torch.zeros(2, 3, 8, 64)), "shape"),
    (dict(q=torch.zeros(3, 3, 8, 128)), "shape"), (dict(q=torch.zeros(2, 8, 3, 128).transpose(1, 2)), "contiguous"),
    (dict(tree_mask=None), "go together"), (dict(draft_lens=None), "go together"),
    (dict(tree_mask=torch.zeros(2, 4, dtype=torch.int64)), "tree_mask must have shape"),
    (dict(tree_mask=torch.zeros(2, 3, dtype=torch.int32)), "tree_mask must be"),
    (dict(out=torch.zeros(2, 3, 8, 128, dtype=torch.bfloat16)), "out must be"), (dict(out=None), "out is required"),
    (dict(sel=torch.zeros(2, 2, 7, dtype=torch.int32)), "sel holds"), (dict(lse=torch.zeros(2, 3, 7)), "lse holds"),
    (dict(ws=None), "ws is required"), (dict(k=torch.zeros(2, 2, 128, 128)), "k must be"),
    (dict(seq_lens=torch.zeros(2, dtype=torch.int64)), "seq_lens must be"), (dict(), "must be on a GPU"),
])
def test_binding_names_the_wrong_argument_of_a_tree_call(edit, text):
    cfg, t = _tensors()
    t.update(edit)
    with pytest.raises(cobs.CobsError, match=text):
        cache.cobs_tree_decode(cfg, **t)


@pytest.mark.parametrize("edit,text", [
    (dict(kept=torch.zeros(2, 4, dtype=torch.int64)), "kept must be"), (dict(kept=torch.zeros(3, 4, dtype=torch.int32)), "shape"),
    (dict(kept=torch.zeros(2, 3, 4, dtype=torch.int32)), "shape"), (dict(k_out=torch.zeros(2, 2, 64, 128)), "go together"),
    (dict(k_out=torch.zeros(2, 2, 64, 128), v_out=torch.zeros(2, 2, 64, 128)), "k_out must be"),
    (dict(weights_out=torch.zeros(2, 2, 128)), "needs weights"),
    (dict(weights=torch.zeros(2, 2, 128), weights_out=torch.zeros(2, 2, 128)), "to themselves"),
    (dict(k_out=torch.zeros(2, 2, 64, 128, dtype=torch.bfloat16), v_out=torch.zeros(2, 2, 64, 128, dtype=torch.bfloat16),
          weights=torch.zeros(2, 2, 128), weights_out=torch.zeros(2, 2, 128)), "weights_out must have shape"),
    (dict(out_block_table=torch.zeros(2, 2, dtype=torch.int32)), "needs k_out"), (dict(), "must be on a GPU"),
])
def test_binding_names_the_wrong_argument_of_a_compaction(edit, text):
    cfg, t = _tensors()
    a = dict(k=t["k"], v=t["v"], kept=torch.zeros(2, 4, dtype=torch.int32), seq_lens=t["seq_lens"])
    a.update(edit)
    with pytest.raises(cobs.CobsError, match=text):
        cache.cobs_compact_cache(cfg, **a)


@pytest.mark.parametrize("edit,text", [
    (dict(kept=torch.zeros(2, 8, dtype=torch.int32)), "kept must have shape"),
    (dict(kept=torch.zeros(2, 3, 8, dtype=torch.int32)), "kept must have shape"),
    (dict(weights=torch.zeros(2, 2, 64)), "weights holds"), (dict(new_lens=torch.zeros(1, dtype=torch.int32)), "new_lens"),
    (dict(ws=None), "ws is required"), (dict(), "must be on a GPU"),
])
def test_binding_names_the_wrong_argument_of_an_eviction(edit, text):
    cfg, t = _tensors()
    a = dict(weights=torch.zeros(2, 2, 128), seq_lens=t["seq_lens"], kept=torch.zeros(2, 2, 8, dtype=torch.int32), ws=t["ws"])
    a.update(edit)
    with pytest.raises(cobs.CobsError, match=text):
        cache.cobs_evict(cfg, **a)
