"""The cache operators against fp64: attention of several query tokens a row, accumulated attention
weights, eviction, compaction, and all of them in turn as a serving program runs them.  Tolerances are
derived in tests/cache_util.py."""

import numpy as np
import pytest
import torch

from oracle import cache as O
from paper_2607_09052_amd import cache, cobs
from tests.cache_util import Problem, run_tree, run_weights, to_mask
from tests.gpu_util import DEV, f64, say, sync

pytestmark = pytest.mark.gpu

SHAPES = [
    # one token, one query: the smallest call
    dict(B=1, Hkv=1, G=1, d=64, L=32, T=1, N=1),
    dict(B=1, Hkv=1, G=1, d=64, L=32, T=0, N=1),                       # the draft alone
    dict(B=2, Hkv=2, G=4, d=128, T=(300, 77), N=8),
    dict(B=3, Hkv=1, G=16, d=128, T=(31, 32, 33), N=5, L=32),
    dict(B=2, Hkv=3, G=2, d=64, T=(129, 1000), N=3, L=128),
    dict(B=2, Hkv=2, G=8, d=128, T=(700, 0), N=64),                    # the longest draft; a row without a context
    dict(B=2, Hkv=1, G=16, d=64, T=(1500, 64), N=64, L=64),
    dict(B=1, Hkv=2, G=4, d=128, T=3001, N=17, c=0.25),
    dict(B=4, Hkv=2, G=4, d=128, T=(200, 90, 0, 511), N=9, drafts=(9, 0, 4, 1)),   # padded drafts, an empty row
    dict(B=2, Hkv=2, G=4, d=128, T=(900, 333), N=6, s=3, w=100),
    dict(B=2, Hkv=2, G=8, d=128, T=(900, 20), N=33, s=5, w=70, L=32),
    dict(B=2, Hkv=1, G=2, d=64, T=(2000, 640), N=12, s=40, w=0, L=128),   # a budget over the candidates, no window
    dict(B=1, Hkv=2, G=4, d=128, T=700, N=4, s=0, w=65),               # the window alone
    dict(B=2, Hkv=2, G=1, d=128, T=(450, 7), N=40, s=2, w=5000),       # a window over everything
    dict(B=2, Hkv=2, G=4, d=128, T=(257, 64), N=7, draft=False),       # queries without a draft
    dict(B=1, Hkv=2, G=8, d=64, T=1200, N=1, draft=False, s=4, w=33),
]


def _ids(x):
    return "-".join(f"{k}{v}" for k, v in x.items()) if isinstance(x, dict) else str(x)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=_ids)
def test_tree_decode_matches_fp64(shape, kv, io):
    say(f"tree {shape} {kv} {io}")
    p = Problem(DEV, kv=kv, io=io, **shape).upload()
    out, lse = run_tree(p)
    sync()
    say(f"worst error / tolerance {p.check_tree(out, lse):.3f}")


# Many rows over a long cache (of which little may be filled): tiles of 256 rows
MANY_ROWS = [
    dict(B=2, Hkv=8, G=16, T=(300, 77), N=64, extra=8192),
    dict(B=2, Hkv=8, G=16, T=(1100, 0), N=64, drafts=(64, 40), extra=7200, layout="pages"),
    dict(B=2, Hkv=8, G=16, T=(500, 33), N=44, drafts=(31, 44), extra=11000, layout="strided"),   # 704 rows, 31 of 44 queries
    dict(B=2, Hkv=8, G=16, T=(1900, 700), N=64, s=128, w=100, extra=6400),
    dict(B=2, Hkv=8, G=16, T=(129, 96), N=64, draft=False, L=32, extra=8192, c=0.3),
    dict(B=1, Hkv=8, G=16, T=0, N=64, drafts=(0,), extra=16448),
]


@pytest.mark.parametrize("shape", MANY_ROWS, ids=_ids)
def test_tree_decode_of_many_rows_matches_fp64(shape):
    say(f"tree, many rows {shape}")
    p = Problem(DEV, io="bf16", **shape).upload()
    out, lse = run_tree(p)
    sync()
    say(f"worst error / tolerance {p.check_tree(out, lse):.3f}")


@pytest.mark.parametrize("kv,io", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("shape", [
    dict(B=8, Hkv=8, G=4, T=(8100, 0, 33, 700, 2500, 1, 64, 4000), N=5, drafts=(5, 2, 0, 5, 3, 5, 1, 4), extra=700),   # 8 parts a row
    dict(B=16, Hkv=8, G=2, T=(31, 4000, 0, 5) + (0,) * 11 + (100,), N=3, layout="pages", extra=700),           # 4 of them
    dict(B=5, Hkv=2, G=8, T=(13000, 12000, 300, 12500, 5), N=12, draft=False, extra=45000),                    # 51
], ids=_ids)
def test_parts_by_the_rows_lengths(shape, kv, io):
    """Contexts of very different lengths, which share the parts of the longest by their lengths."""
    say(f"uneven rows {shape} {kv} {io}")
    p = Problem(DEV, kv=kv, io=io, d=64, **shape).upload()
    out, lse = run_tree(p)
    sync()
    say(f"worst error / tolerance {p.check_tree(out, lse):.3f}")
    before = torch.rand((p.B, p.Hkv, p.cap), generator=torch.Generator().manual_seed(1)).to(DEV)
    weights = run_weights(p, lse, before.clone())
    sync()
    p.check_weights(weights, lse, None, f64(before))


def test_many_rows_over_one_long_context():
    """64 (row, KV head) pairs that share one cache of 17024 tokens by strides of 0: one part of 532 frames each."""
    p = Problem(DEV, B=1, Hkv=1, G=16, T=16960, N=64, io="bf16", seed=8).upload()
    B, H = 4, 16
    cfg = cobs.Config(batch=B, num_q_heads=H * 16, num_kv_heads=H, head_dim=128, max_seq_len=p.cap, rank=0, budget=0, window=0)
    q = torch.randn((B, 64, H, 16, 128), generator=torch.Generator().manual_seed(9)).to(torch.bfloat16).to(DEV)
    q[3, :, 15] = p.qd[0]
    out, lse = torch.empty((B, 64, H * 16, 128), dtype=torch.bfloat16, device=DEV), torch.empty((B, 64, H * 16), device=DEV)
    cache.cobs_tree_decode(cfg, q.view(B, 64, H * 16, 128), p.kd.expand(B, H, p.cap, 128), p.vd.expand(B, H, p.cap, 128),
                           p.seq.expand(B).contiguous(), p.drafts.expand(B).contiguous(), p.mask.expand(B, 64).contiguous(),
                           out, cache.new_tree_workspace(cfg, 64, DEV), lse=lse)
    sync()
    p.check_tree(out[3:, :, 240:].contiguous(), lse[3:, :, 240:].contiguous())


def test_many_rows_do_not_see_what_others_see():
    """As below, with tiles of 256 rows: values of drafted tokens that are not finite, NaN where no query looks."""
    N, drafts, T = 64, (64, 50), (90, 0)
    bits = [[1 << i for i in range(N)] for _ in range(2)]
    a = dict(B=2, Hkv=8, G=16, T=T, N=N, drafts=drafts, bits=bits, io="bf16", extra=8192)
    p, clean = Problem(DEV, **a), Problem(DEV, **a)
    for b in range(2):
        p.k[b, :, T[b] + drafts[b]:] = float("nan")
        p.v[b, :, T[b] + drafts[b]:] = float("inf")
        p.v[b, :, T[b] + 5, 3:6] = torch.tensor([float("inf"), float("nan"), -float("inf")], dtype=p.v.dtype)
    p.upload(), clean.upload()
    (out, lse), (want, wl) = run_tree(p), run_tree(clean)
    sync()
    got5 = out[:, 5].float()
    for e, f in ((3, torch.isposinf), (4, torch.isnan), (5, torch.isneginf)):
        assert bool(f(got5[..., e]).all()), (e, got5[..., e])
    out[:, 5, :, 3:6] = want[:, 5, :, 3:6]
    assert torch.equal(out, want) and torch.equal(lse, wl)


def test_many_rows_on_pages_out_of_range():
    """A page id out of range leaves its tokens out, as if another selection had (both by tiles of 256 rows)."""
    p = Problem(DEV, B=1, Hkv=16, G=16, T=300, N=64, io="bf16", layout="pages", extra=8192).upload()
    gone = Problem(DEV, B=1, Hkv=16, G=16, T=300, N=64, io="bf16", layout="pages", extra=8192, s=160, w=0)
    for h in range(16):                                                    # blocks 0, 2, 3, 4 of 0 .. 4
        gone.sel[0, h, :] = -1
        gone.sel[0, h, :4] = (0, 2, 3, 4)
    gone.upload()
    gone.check_tree(*run_tree(gone))
    for bad in (-1, p.pages["num_pages"]):
        p.pages["block_table"][0, 1] = bad
        out, lse = run_tree(p)
        sync()
        gone.check_tree(out, lse)


@pytest.mark.parametrize("layout", ["pages", "strided"])
@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [SHAPES[i] for i in (2, 5, 8, 9, 10, 14)], ids=_ids)
def test_layouts_do_not_change_a_bit(shape, kv, layout):
    say(f"layout {layout} {shape} {kv}")
    for io in ("f32", "bf16"):
        p = Problem(DEV, kv=kv, io=io, **shape).upload()
        x = Problem(DEV, kv=kv, io=io, layout=layout, **shape).upload()
        (o1, l1), (o2, l2) = run_tree(p), run_tree(x)
        w1, w2 = (run_weights(y, l1, torch.zeros((p.B, p.Hkv, p.cap), device=DEV)) for y in (p, x))
        assert torch.equal(o1, o2) and torch.equal(l1, l2) and torch.equal(w1, w2)


@pytest.mark.parametrize("kv", ["bf16", "f32"])
def test_one_query_is_the_sparse_decode(kv):
    """The same attention by cobs_sparse_decode: both are within their errors of the exact one, here the sum of the
    tree's (checked above against fp64) and the decode's documented 2e-3 (bf16) / 1e-5 (fp32) relative."""
    p = Problem(DEV, B=2, Hkv=2, G=4, T=(900, 333), N=1, s=3, w=100, kv=kv, draft=False).upload()
    out, lse = run_tree(p)
    want, wl = torch.empty((2, 8, 128), device=DEV), torch.empty((2, 8), device=DEV)
    ws = cobs.new_workspace(p.cfg, cobs.OP_DECODE, DEV)
    cobs.cobs_sparse_decode(p.cfg, p.qd[:, 0].contiguous(), p.kd, p.vd, p.seq, p.sel_d, want, ws, lse=wl)
    p.check_tree(out, lse)
    assert float((out[:, 0] - want).norm() / want.norm()) < (2e-3 if kv == "bf16" else 1e-5)
    assert float((lse[:, 0] - wl).abs().max()) < 1e-4


@pytest.mark.parametrize("kv,io", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32")])
def test_what_a_query_does_not_see_does_not_reach_it(kv, io):
    """NaN, infinities and the type's lowest value behind the rows, in unselected blocks and in drafted tokens that
    no query or only others see; masks with no bit and with bits past the draft."""
    say(f"unseen {kv} {io}")
    T, N, drafts = (200, 64, 0), 40, (40, 33, 2)
    bits = []
    for b in range(3):
        rows = [(1 << i) for i in range(N)]
        rows[1] = 0                                            # sees no draft (row 2: nothing at all)
        rows[0] |= (1 << 63) | (1 << drafts[b] if drafts[b] < 63 else 0)
        bits.append(rows)
    for s, w in ((-1, 0), (1, 30)):
        p = Problem(DEV, B=3, T=T, N=N, drafts=drafts, bits=bits, kv=kv, io=io, s=s, w=w, L=32, extra=64)
        bad = torch.tensor([float("nan"), float("inf"), -float("inf"), torch.finfo(p.k.dtype).min], dtype=p.k.dtype)
        clean = Problem(DEV, B=3, T=T, N=N, drafts=drafts, bits=bits, kv=kv, io=io, s=s, w=w, L=32, extra=64)
        for b in range(3):
            for h in range(2):
                seen = p.see(b, h).any(0)
                for t in range(p.cap):
                    if t >= len(seen) or not seen[t]:
                        p.k[b, h, t] = bad[(t + h) % 4]
                        p.v[b, h, t] = bad[(t + h + 1) % 4]
                # drafted token 5 is seen by query 5 alone: its value is not finite, nor is that query's output
                if drafts[b] > 5:
                    p.v[b, h, T[b] + 5, 3:6] = torch.tensor([float("inf"), float("nan"), -float("inf")], dtype=p.k.dtype)
        p.upload(), clean.upload()
        out, lse = run_tree(p)
        want, wl = run_tree(clean)
        sync()
        clean.check_tree(want, wl)
        only5 = [b for b in range(3) if drafts[b] > 5]
        got5 = out[only5, 5].float()
        for e, f in ((3, torch.isposinf), (4, torch.isnan), (5, torch.isneginf)):
            assert bool(f(got5[..., e]).all()), (e, got5[..., e])
        out[only5, 5, :, 3:6] = want[only5, 5, :, 3:6]
        assert torch.equal(out, want) and torch.equal(lse, wl)
        zero = torch.zeros((3, 2, p.cap), device=DEV)
        assert torch.equal(run_weights(p, wl, zero.clone())[:, :, :], run_weights(clean, wl, zero.clone()))


@pytest.mark.parametrize("kv", ["bf16", "f32"])
def test_pages_out_of_range_are_left_out(kv):
    p = Problem(DEV, B=2, T=(300, 200), N=4, kv=kv, layout="pages").upload()
    full = Problem(DEV, B=2, T=(300, 200), N=4, kv=kv).upload()
    _, l0 = run_tree(full)
    p.pages["block_table"][0, 1] = p.pages["num_pages"]
    p.pages["block_table"][1, 0] = -5
    out, lse = run_tree(p)
    weights = run_weights(p, l0, torch.zeros((2, 2, p.cap), device=DEV))
    sync()
    q = f64(p.q).reshape(2, 4, 2, 4, 128)
    for b, gone in ((0, 1), (1, 0)):
        for h in range(2):
            see = p.see(b, h)
            see[:, 64 * gone:64 * gone + 64] = False
            E = p.T[b] + 4
            want, wl = O.tree_attention(q[b, :, h], f64(p.k)[b, h, :E], f64(p.v)[b, h, :E], see, p.cfg.scale)
            # as in check_tree, loosely bounded: scores within 388 half steps of c sum |q||k| (< 15 here), 4e-4
            assert np.abs(f64(out)[b, :, 4 * h:4 * h + 4] - want).max() < 1e-3
            assert np.abs(f64(lse)[b, :, 4 * h:4 * h + 4] - wl).max() < 1e-3
            assert bool((weights[b, h, 64 * gone:64 * gone + 64] == 0).all())


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("kv", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=_ids)
def test_attention_weights_match_fp64(shape, kv, io):
    say(f"weights {shape} {kv} {io}")
    p = Problem(DEV, kv=kv, io=io, **shape).upload()
    _, lse = run_tree(p)
    lse[:, p.N // 2:p.N // 2 + 1, 0] = float("inf")              # a query head left out
    g = torch.Generator().manual_seed(3)
    before = torch.randn((p.B, p.Hkv, p.cap), generator=g).to(DEV)
    prev = torch.rand((p.B, p.Hkv, p.cap), generator=g).to(DEV) * 0.01
    for pv in (None, prev):
        weights = run_weights(p, lse, before.clone(), pv)
        sync()
        p.check_weights(weights, lse, None if pv is None else f64(pv), f64(before))
    same = prev.clone()
    run_weights(p, lse, same, same)                             # prev in place
    E = torch.arange(p.cap, device=DEV).view(1, 1, -1) < (p.seq + (p.drafts if p.draft else 0)).view(-1, 1, 1)
    assert torch.equal(same, torch.where(E, weights, prev))


def test_weights_add_up_to_the_queries():
    """All of the context's and the draft's weights: one per live query head, within the terms' errors (2^-12 of
    them is far above what check_weights allows each)."""
    p = Problem(DEV, B=2, T=(5000, 1234), N=10, drafts=(10, 3), G=8).upload()
    _, lse = run_tree(p)
    w = run_weights(p, lse, torch.zeros((2, 2, p.cap), device=DEV))
    got = w.double().sum(-1).cpu()
    assert torch.allclose(got, torch.tensor([[80.0, 80.0], [24.0, 24.0]], dtype=torch.float64), rtol=2.0 ** -12)


EVICT = [
    dict(T=(1,), keep=1), dict(T=(5, 4, 0), keep=4, sinks=1, recent=1), dict(T=(2000, 64, 65), keep=64, sinks=4, recent=16),
    dict(T=(4093,), keep=1024, sinks=0, recent=0), dict(T=(4096, 1), keep=4095, sinks=8, recent=8),
    dict(T=(3000, 2999), keep=100, sinks=60, recent=40), dict(T=(70000, 30011), keep=5000, sinks=4, recent=64),
    dict(T=(131072,), keep=32768, sinks=4, recent=1024), dict(T=(50000,), keep=1), dict(T=(20000,), keep=19999, recent=19998),
    # (chunks of 8192 so far; of 16384 and of 32768: more rows)
    dict(T=(39990, 17, 33000, 40001) * 8, keep=700, sinks=3, recent=20), dict(T=(33001, 32769, 5) * 24, keep=900, sinks=3, recent=20),
]


@pytest.mark.parametrize("law", ["heavy", "ties", "zeros", "specials", "close"])
@pytest.mark.parametrize("shape", EVICT, ids=_ids)
def test_evict_matches_the_definition(shape, law):
    say(f"evict {shape} {law}")
    T, keep = shape["T"], shape["keep"]
    B, Hkv, cap = len(T), 2, max(64, -(-max(T) // 64) * 64)
    g = np.random.default_rng(7)
    w = np.exp(2 * g.standard_normal((B, Hkv, cap))).astype(np.float32)
    if law == "ties":
        w = np.round(np.minimum(w, 8)).astype(np.float32)
    elif law == "zeros":
        w[g.random(w.shape) < 0.97] = 0.0
        w[g.random(w.shape) < 0.3] *= -0.0
    elif law == "specials":
        w *= g.choice([-1, 1], w.shape)
        w[g.random(w.shape) < 0.3] = np.inf
        w[g.random(w.shape) < 0.3] = -np.inf
        w[g.random(w.shape) < 0.3] = np.nan
        w[g.random(w.shape) < 0.1] = np.finfo(np.float32).min
        w[g.random(w.shape) < 0.1] = 1e-45
    elif law == "close":
        w = (np.float32(0.3).view(np.int32) + g.integers(0, 40, w.shape)).astype(np.int32).view(np.float32)
    cfg = cobs.Config(batch=B, num_q_heads=Hkv, num_kv_heads=Hkv, head_dim=64, max_seq_len=cap, rank=0, budget=0, window=0)
    seq = torch.tensor(T, dtype=torch.int32, device=DEV)
    ws = cache.new_evict_workspace(cfg, DEV)
    kept = torch.full((B, Hkv, keep), -7, dtype=torch.int32, device=DEV)
    lens = torch.empty(B, dtype=torch.int32, device=DEV)
    wd = torch.from_numpy(w).to(DEV)
    for _ in range(2):                     # twice on one workspace
        kept.fill_(-7)
        cache.cobs_evict(cfg, wd, seq, kept, ws, sinks=shape.get("sinks", 0), recent=shape.get("recent", 0), new_lens=lens)
        sync()
        assert lens.tolist() == [min(t, keep) for t in T]
        got = kept.cpu().numpy()
        for b in range(B):
            for h in range(Hkv):
                want = O.evict(w[b, h], T[b], keep, shape.get("sinks", 0), shape.get("recent", 0))
                assert got[b, h].tolist() == want + [-1] * (keep - len(want)), (b, h)


def _cache_of(kv, B, Hkv, cap, d, L, layout, seed):
    """A random cache in a layout, and the function that reads it as [B, Hkv, cap, d]."""
    g = torch.Generator().manual_seed(seed)
    t = torch.float32 if kv == "f32" else torch.bfloat16
    if layout == "pages":
        nb = cap // L
        table = torch.randperm(B * nb + 2, generator=g)[:B * nb].to(torch.int32).view(B, nb).to(DEV)
        k, v = (torch.randn((B * nb + 2, Hkv, L, d), generator=g).to(t).to(DEV) for _ in range(2))
        return k, v, table, lambda x: x[table.long()].permute(0, 2, 1, 3, 4).reshape(B, Hkv, cap, d)
    if layout == "strided":
        k, v = (torch.randn((B, cap, Hkv, d + 8), generator=g).to(t).to(DEV)[..., :d].permute(0, 2, 1, 3) for _ in range(2))
        return k, v, None, lambda x: x
    k, v = (torch.randn((B, Hkv, cap, d), generator=g).to(t).to(DEV) for _ in range(2))
    return k, v, None, lambda x: x


@pytest.mark.parametrize("kv,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("src,dst", [("contiguous", None), ("pages", None), ("strided", None),
                                     ("contiguous", "contiguous"), ("pages", "pages"), ("strided", "pages"),
                                     ("pages", "strided")])
@pytest.mark.parametrize("T,num,per_head,first", [
    ((1500, 200), 900, True, None), ((1500, 200, 0, 640), 7, False, (1400, 190, 0, 633)), ((3000,), 2999, True, None),
    ((64, 65), 1, True, (10, 64)), ((5000, 4000), 1300, True, (100, 0)), ((33,), 0, True, None),
])
def test_compaction_moves_rows_and_weights(kv, d, src, dst, T, num, per_head, first):
    say(f"compact {kv} {d} {src} {dst} {T} {num} {per_head} {first}")
    B, Hkv, L = len(T), 2, 64
    cap = -(-max(T) // L) * L
    dcap = cap if dst is None else -(-max(num + (max(first) if first else 0), 1) // L) * L
    if dst == "strided":
        dcap = max(L, dcap - L)                 # entries behind the capacity are dropped
    rng = np.random.default_rng(5)
    kept = np.full((B, Hkv, num), -1, dtype=np.int32)
    for b in range(B):
        f = first[b] if first else 0
        for h in range(Hkv):
            if per_head or h == 0:
                m = min(num, max(T[b] - f, 0))
                kept[b, h, :m] = np.sort(rng.choice(max(T[b] - f, 1), m, replace=False)) + f
            else:
                kept[b, h] = kept[b, 0]
            if num > 20:
                kept[b, h, num - 9] = T[b] + 3      # no such token: moves nothing
    cfg = cobs.Config(batch=B, num_q_heads=Hkv, num_kv_heads=Hkv, head_dim=d, max_seq_len=cap, rank=0, budget=0, window=0,
                      kv_dtype=kv)
    k, v, table, read = _cache_of(kv, B, Hkv, cap, d, L, src, 1)
    weights = torch.rand((B, Hkv, cap), device=DEV)
    k0, v0, w0 = read(k).cpu().clone(), read(v).cpu().clone(), weights.cpu().clone()
    ko = vo = wo = otable = None
    back, wback = read, weights
    e_k, e_v, e_w = k0.clone(), v0.clone(), w0.clone()
    if dst is not None:
        ko, vo, otable, back = _cache_of(kv, B, Hkv, dcap, d, L, dst, 2)
        wo = torch.rand((B, Hkv, dcap), device=DEV)
        e_k, e_v, e_w, wback = back(ko).cpu().clone(), back(vo).cpu().clone(), wo.cpu().clone(), wo
    pages = dict(block_table=table, num_pages=k.shape[0]) if table is not None else {}
    if otable is not None:
        pages.update(out_block_table=otable, out_num_pages=ko.shape[0])
    kd = torch.from_numpy(kept if per_head else kept[:, 0].copy()).to(DEV)
    cache.cobs_compact_cache(cfg, k, v, kd, torch.tensor(T, dtype=torch.int32, device=DEV),
                             first=None if first is None else torch.tensor(first, dtype=torch.int32, device=DEV),
                             k_out=ko, v_out=vo, weights=weights, weights_out=wo, **pages)
    sync()
    for b in range(B):
        f = first[b] if first else 0
        for h in range(Hkv):
            O.compact(k0[b, h].view(torch.int16 if kv == "bf16" else torch.int32).numpy(),
                      e_k[b, h].view(torch.int16 if kv == "bf16" else torch.int32).numpy(), kept[b, h].tolist(), T[b], f)
            O.compact(v0[b, h].view(torch.int16 if kv == "bf16" else torch.int32).numpy(),
                      e_v[b, h].view(torch.int16 if kv == "bf16" else torch.int32).numpy(), kept[b, h].tolist(), T[b], f)
            O.compact_weights(w0[b, h].numpy(), e_w[b, h].numpy(), kept[b, h].tolist(), T[b], f)
    assert torch.equal(back(ko if dst else k).cpu(), e_k)
    assert torch.equal(back(vo if dst else v).cpu(), e_v)
    assert torch.equal(wback.cpu(), e_w)


@pytest.mark.parametrize("kv,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("src", ["contiguous", "pages", "strided"])
def test_compaction_in_place_of_many_rows(kv, d, src):
    """Enough (row, KV head) pairs for the wider slices, and entries for several of their batches."""
    test_compaction_moves_rows_and_weights(kv, d, src, None, (2300, 200) * 16, 1700, True, None)


def test_compaction_leaves_pages_out_of_range_alone():
    B, Hkv, L, d, cap = 1, 1, 64, 64, 256
    cfg = cobs.Config(batch=B, num_q_heads=1, num_kv_heads=1, head_dim=d, max_seq_len=cap, rank=0, budget=0, window=0)
    pool = torch.randn((4, Hkv, L, d), device=DEV).to(torch.bfloat16)
    for bad in (-1, 4, 2 ** 31 - 1):
        table = torch.tensor([[0, bad, 2, 3]], dtype=torch.int32, device=DEV)
        k, v = pool.clone(), pool.clone()
        kept = torch.tensor([[5, 70, 130, 131]], dtype=torch.int32, device=DEV)
        w = torch.rand((1, 1, cap), device=DEV)
        w0 = w.clone()
        cache.cobs_compact_cache(cfg, k, v, kept, torch.tensor([256], dtype=torch.int32, device=DEV),
                                 first=torch.tensor([2], dtype=torch.int32, device=DEV), weights=w, block_table=table,
                                 num_pages=4)
        want = pool.clone()
        want[0, 0, 2], want[0, 0, 4], want[0, 0, 5] = pool[0, 0, 5], pool[2, 0, 2], pool[2, 0, 3]
        assert torch.equal(k, want) and torch.equal(v, want)
        assert torch.equal(w[0, 0, :6], torch.stack([w0[0, 0, 0], w0[0, 0, 1], w0[0, 0, 5], 0 * w0[0, 0, 0], w0[0, 0, 130], w0[0, 0, 131]]))
        assert bool((w[0, 0, 6:] == 0).all())


def test_compaction_to_other_pages_of_the_same_pool():
    B, Hkv, L, d, T, keep = 2, 2, 32, 128, (200, 150), 70
    cfg = cobs.Config(batch=B, num_q_heads=Hkv, num_kv_heads=Hkv, head_dim=d, max_seq_len=224, rank=0, budget=0, window=0,
                      block_size=L)
    g = torch.Generator().manual_seed(4)
    perm = torch.randperm(24, generator=g).to(torch.int32)
    table, new = perm[:14].view(2, 7).to(DEV), perm[14:20].view(2, 3).to(DEV)
    k, v = (torch.randn((24, Hkv, L, d), generator=g).to(torch.bfloat16).to(DEV) for _ in range(2))
    k0, v0 = k.cpu().clone(), v.cpu().clone()
    kept = torch.stack([torch.stack([torch.randperm(T[b], generator=g)[:keep].sort()[0] for _ in range(Hkv)]) for b in range(B)])
    cache.cobs_compact_cache(cfg, k, v, kept.to(torch.int32).to(DEV), torch.tensor(T, dtype=torch.int32, device=DEV), k_out=k,
                             v_out=v, block_table=table, num_pages=24, out_block_table=new, out_num_pages=24)
    t, n = table.cpu(), new.cpu()
    for b in range(B):
        for h in range(Hkv):
            for j in range(keep):
                s = int(kept[b, h, j])
                for x in (k0, v0):
                    x[n[b, j // L], h, j % L] = x[t[b, s // L], h, s % L]
    assert torch.equal(k.cpu(), k0) and torch.equal(v.cpu(), v0)


def test_offsets_past_32_bits():
    """A cache whose last tokens lie 2^32 elements behind its first: rows 2^22 elements apart."""
    T, N, d, st = 1024, 3, 64, 1 << 22
    p = Problem(DEV, B=1, Hkv=1, G=4, d=d, T=T - N, N=N).upload()
    big = torch.empty((T - 1) * st + 2 * d, dtype=torch.bfloat16, device=DEV)
    k, v = (torch.as_strided(big, (1, 1, T, d), (0, 0, st, 1), o) for o in (0, d))
    k.copy_(p.kd), v.copy_(p.vd)
    out, lse = run_tree(p)
    w = run_weights(p, lse, torch.zeros((1, 1, T), device=DEV))
    p.kd, p.vd = k, v
    out2, lse2 = run_tree(p)
    w2 = run_weights(p, lse, torch.zeros((1, 1, T), device=DEV))
    assert torch.equal(out, out2) and torch.equal(lse, lse2) and torch.equal(w, w2)
    kept = torch.arange(1, T, 2, dtype=torch.int32, device=DEV).view(1, 1, -1)
    want = k[:, :, 1::2].clone()
    cache.cobs_compact_cache(p.cfg, k, v, kept, torch.tensor([T], dtype=torch.int32, device=DEV))
    assert torch.equal(k[:, :, :T // 2], want)


@pytest.mark.parametrize("kv,io,N,G", [("bf16", "bf16", 1, 1), ("bf16", "f32", 9, 4), ("bf16", "bf16", 33, 4), ("f32", "f32", 2, 1)])
def test_long_parts_of_many_rows(kv, io, N, G):
    """256 rows that are one row 256 times over (a batch stride of 0): few parts a row, each longer than the table of
    frames.  Every row has the same bits, the first row is checked."""
    say(f"long parts {kv} {io} {N} {G}")
    p = Problem(DEV, B=1, Hkv=1, G=G, d=64, L=32, T=17000, N=N, kv=kv, io=io).upload()
    q = Problem(DEV, B=1, Hkv=1, G=G, d=64, L=32, T=17000, N=N, kv=kv, io=io).upload()
    B = 256
    q.cfg.batch = q.B = B
    q.qd, q.seq, q.drafts, q.mask = (x.repeat(B, *[1] * (x.dim() - 1)) for x in (p.qd, p.seq, p.drafts, p.mask))
    q.kd, q.vd = (x.expand(B, -1, -1, -1) for x in (p.kd, p.vd))
    out, lse = run_tree(q)
    weights = run_weights(q, lse, torch.zeros((B, 1, q.cap), device=DEV))
    sync()
    assert torch.equal(out, out[:1].expand_as(out)) and torch.equal(lse, lse[:1].expand_as(lse))
    assert torch.equal(weights, weights[:1].expand_as(weights))
    p.check_tree(out[:1], lse[:1])
    p.check_weights(weights[:1], lse[:1], None, np.zeros((1, 1, p.cap)))


@pytest.mark.parametrize("seed", range(40))
def test_random_problems(seed):
    """Tree attention and weights over random shapes, types, layouts, selections, windows and drafts."""
    r = np.random.default_rng(1000 + seed)
    G = int(r.choice([1, 2, 4, 8, 16]))
    N = int(r.integers(1, 65)) if r.random() < 0.5 else int(r.integers(1, 6))
    B = int(r.integers(1, 4))
    T = [int(x) for x in np.exp(r.uniform(0, np.log(2500 if N * G < 300 else 700), B))]
    draft = bool(r.random() < 0.8)
    sparse = bool(r.random() < 0.5)
    a = dict(B=B, Hkv=int(r.integers(1, 4)), G=G, d=int(r.choice([64, 128])), L=int(r.choice([32, 64, 128])), T=T, N=N,
             drafts=[int(r.integers(0, N + 1)) for _ in range(B)], draft=draft, s=int(r.integers(0, 20)) if sparse else -1,
             w=int(r.integers(0, 300)) if sparse else 0, kv=str(r.choice(["bf16", "bf16", "f32"])),
             io=str(r.choice(["bf16", "f32"])), layout=str(r.choice(["contiguous", "pages", "strided"])), seed=seed,
             extra=int(r.integers(0, 200)))
    say(f"random {a}")
    if draft and r.random() < 0.4:      # any bits, past the draft too
        a["bits"] = [[int(x) for x in r.integers(0, 2 ** 64, N, dtype=np.uint64)] for _ in range(B)]
    p = Problem(DEV, **a).upload()
    out, lse = run_tree(p)
    sync()
    p.check_tree(out, lse)
    before = torch.full((p.B, p.Hkv, p.cap), 7.0, device=DEV)
    w = run_weights(p, lse, before.clone())
    sync()
    p.check_weights(w, lse, None, f64(before))
    no_lse = torch.full_like(out, float("nan"))
    cache.cobs_tree_decode(p.cfg, p.qd, p.kd, p.vd, p.seq, p.drafts, p.mask, no_lse, cache.new_tree_workspace(p.cfg, N, DEV),
                           sel=p.sel_d, **p.pages)
    assert torch.equal(out, no_lse)


def test_a_serving_loop_runs_them_in_turn():
    """Prompt statistics, a selection, a draft attended to over it, its weights, the accepted path moved up, eviction,
    compaction, the records rebuilt, and a decode step on the shorter cache, each against fp64."""
    B, Hkv, G, d, L, N = 2, 2, 4, 128, 64, 8
    p = Problem(DEV, B=B, Hkv=Hkv, G=G, d=d, L=L, T=(1000, 611), N=N, drafts=(8, 5), s=4, w=100).upload()
    cfg = p.cfg
    cfg.rank = 2
    rec = cobs.new_summaries(cfg, DEV)
    cobs.cobs_build_block_stats(cfg, p.kd, p.vd, p.seq, rec)
    sel_ws = cobs.new_workspace(cfg, cobs.OP_SELECT, DEV)
    sel = torch.empty((B, Hkv, 4), dtype=torch.int32, device=DEV)
    cobs.cobs_select(cfg, p.qd[:, 0].contiguous(), rec, p.seq, sel, sel_ws)
    p.sel_d = sel
    p.sel = sel.cpu().numpy()
    out, lse = run_tree(p)
    p.check_tree(out, lse)
    # the path to the last live node of each row is accepted; the other queries add no weight
    paths = [[j for j in range(p.n[b]) if (p.bits[b][p.n[b] - 1] >> j) & 1] for b in range(B)]
    for b in range(B):
        for i in range(N):
            if i not in paths[b]:
                lse[b, i] = float("inf")
    weights = torch.zeros((B, Hkv, p.cap), device=DEV)
    run_weights(p, lse, weights, weights)
    p.check_weights(weights, lse, np.zeros((B, Hkv, p.cap)), np.zeros((B, Hkv, p.cap)))
    accepted = torch.full((B, N), -1, dtype=torch.int32)
    for b in range(B):
        accepted[b, :len(paths[b])] = torch.tensor([p.T[b] + j for j in paths[b]])
    k0, v0, w0 = p.kd.clone(), p.vd.clone(), weights.clone()
    cache.cobs_compact_cache(cfg, p.kd, p.vd, accepted.to(DEV), p.seq + p.drafts, first=p.seq, weights=weights)
    lens = p.seq + torch.tensor([len(x) for x in paths], dtype=torch.int32, device=DEV)
    for b in range(B):
        rows = list(range(p.T[b])) + [p.T[b] + j for j in paths[b]]
        assert torch.equal(p.kd[b, :, :len(rows)], k0[b][:, rows]) and torch.equal(p.vd[b, :, :len(rows)], v0[b][:, rows])
        assert torch.equal(weights[b, :, :len(rows)], w0[b][:, rows])
        assert bool((weights[b, :, len(rows):p.T[b] + p.n[b]] == 0).all())
    # eviction to 512 tokens, in place
    keep = 512
    kept = torch.empty((B, Hkv, keep), dtype=torch.int32, device=DEV)
    short = torch.empty(B, dtype=torch.int32, device=DEV)
    cache.cobs_evict(cfg, weights, lens, kept, cache.new_evict_workspace(cfg, DEV), sinks=4, recent=100, new_lens=short)
    k1, v1 = p.kd.clone(), p.vd.clone()
    cache.cobs_compact_cache(cfg, p.kd, p.vd, kept, lens, weights=weights)
    for b in range(B):
        for h in range(Hkv):
            want = O.evict(f64(w0)[b, h][list(range(p.T[b])) + [p.T[b] + j for j in paths[b]]], int(lens[b]), keep, 4, 100)
            assert kept[b, h].tolist() == want
            assert torch.equal(p.kd[b, h, :keep], k1[b, h, want]) and torch.equal(p.vd[b, h, :keep], v1[b, h, want])
    assert short.tolist() == [keep, keep]
    # the next token, and a decode step over the shorter cache: attention of its union, like the tree's
    for b in range(B):
        p.kd[b, :, keep], p.vd[b, :, keep] = 0.5, 1.5
    short += 1
    cobs.cobs_build_block_stats(cfg, p.kd, p.vd, short, rec)
    o2, l2 = torch.empty((B, Hkv * G, d), device=DEV), torch.empty((B, Hkv * G), device=DEV)
    q = p.qd[:, 0].contiguous()
    cobs.cobs_decode_step(cfg, q, p.kd, p.vd, short, rec, o2, cobs.new_workspace(cfg, cobs.OP_STEP, DEV), sel=sel, lse=l2)
    p.T, p.n, p.N, p.draft, p.bits = [keep + 1] * B, [0] * B, 1, False, None
    p.q, p.k, p.v, p.qd = q.cpu()[:, None], p.kd.cpu(), p.vd.cpu(), q[:, None].contiguous()
    p.seq, p.drafts, p.mask, p.sel = short, None, None, sel.cpu().numpy()
    out, lse = run_tree(p)
    p.check_tree(out, lse)
    assert float((out[:, 0] - o2).norm() / o2.norm()) < 2e-3 and float((lse[:, 0] - l2).abs().max()) < 1e-4


def test_streams_and_graphs():
    """Two problems of different sizes interleaved on two streams, and a graph of every operator captured on a side
    stream and replayed three times with eager work between, give the bits of the calls one after the other."""
    ps = [Problem(DEV, B=2, T=(700, 200), N=16, G=8, io="bf16", seed=1).upload(),
          Problem(DEV, B=1, T=(4000,), N=5, s=6, w=64, seed=2).upload()]
    want = [run_tree(p) for p in ps]
    ww = [run_weights(p, z, torch.zeros((p.B, p.Hkv, p.cap), device=DEV)) for p, (_, z) in zip(ps, want)]
    sync()
    streams = [torch.cuda.Stream() for _ in ps]
    wss = [cache.new_tree_workspace(p.cfg, p.N, DEV) for p in ps]
    got = []
    for _ in range(4):
        for p, st, ws in zip(ps, streams, wss):
            with torch.cuda.stream(st):
                got.append(run_tree(p, ws=ws))
    sync()
    for i, (o, z) in enumerate(got):
        assert torch.equal(o, want[i % 2][0]) and torch.equal(z, want[i % 2][1])

    p = ps[0]
    keep = 100
    ews = cache.new_evict_workspace(p.cfg, DEV)
    total = p.seq + p.drafts
    out, lse = torch.zeros_like(p.qd), torch.zeros((p.B, p.N, 16), device=DEV)
    weights = torch.zeros((p.B, p.Hkv, p.cap), device=DEV)
    kept = torch.zeros((p.B, p.Hkv, keep), dtype=torch.int32, device=DEV)
    ko, vo = (torch.zeros((p.B, p.Hkv, 128, p.d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    wo = torch.zeros((p.B, p.Hkv, 128), device=DEV)
    outs = (out, lse, weights, kept, ko, vo, wo)

    def calls():
        cache.cobs_tree_decode(p.cfg, p.qd, p.kd, p.vd, p.seq, p.drafts, p.mask, out, wss[0], lse=lse)
        cache.cobs_attention_weights(p.cfg, p.qd, p.kd, p.vd, p.seq, p.drafts, p.mask, lse, weights)
        cache.cobs_evict(p.cfg, weights, total, kept, ews, sinks=2, recent=10)
        cache.cobs_compact_cache(p.cfg, p.kd, p.vd, kept, total, k_out=ko, v_out=vo, weights=weights, weights_out=wo)

    calls()
    sync()
    eager = [x.clone() for x in outs]
    assert torch.equal(out, want[0][0]) and torch.equal(weights, ww[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        calls()
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            calls()
    for _ in range(3):
        for x in outs:
            x.fill_(0)
        run_tree(ps[1])                       # eager work between the replays
        sync()
        graph.replay()
        sync()
        for x, e in zip(outs, eager):
            assert torch.equal(x, e)
