"""The cache operators on values at the edges, against fp64: bf16 outputs as exact results rounded once, keys and
values that are infinite where queries look, rows that add no weight, the smallest scales, short rows in long batches."""

import numpy as np
import pytest
import torch

from oracle import cache as O
from paper_2607_09052_amd import cache, cobs
from tests.cache_util import HALF, U32, Problem, run_tree, run_weights
from tests.gpu_util import DEV, f64, say, sync

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


def _ids(x):
    return "-".join(f"{k}{v}" for k, v in x.items()) if isinstance(x, dict) else str(x)


# Every form of the attention kernels: 32, 64, 128 query rows a workgroup and 256, one part of a context and many, by
# the rows' lengths in the last.
FORMS = [
    dict(T=(150, 40), N=4), dict(T=(3001, 5), N=3, d=64), dict(T=(200, 33), N=8, G=8, d=64), dict(T=(129, 64), N=8, G=8),
    dict(T=(300, 77), N=33, G=8), dict(T=(1500, 700), N=20, G=16, d=64, layout="pages"),
    dict(T=(900, 333), N=16, s=3, w=100), dict(T=(300, 77), N=64, G=16, Hkv=8, extra=8192),
    dict(B=8, Hkv=8, G=4, d=64, T=(8100, 64, 33, 700, 2500, 1, 0, 4000), N=5, extra=700),
]


@pytest.mark.parametrize("shape", FORMS, ids=_ids)
def test_bf16_outputs_are_rounded_once(shape):
    """bf16 queries and keys of small whole numbers at a scale of 2^-4: scores are exact, at most 16 in size, and the
    exponent (24 in log2 units) takes three roundings, so a probability is off by 3 * 24 + 8 (the exponential's) half
    steps of fp32, the normaliser too, and each sum over n tokens by 4 sqrt(n) of them.  As two bf16 parts a
    probability loses 2^-17 of itself (allowed: 2^-16).  The rest is the output's one rounding."""
    say(f"rounded once {shape}")
    p = Problem(DEV, io="bf16", c=2.0 ** -4, **shape)
    g = torch.Generator().manual_seed(11)
    p.q = torch.randint(-2, 3, p.q.shape, generator=g).to(torch.bfloat16)
    p.k = torch.randint(-1, 2, p.k.shape, generator=g).to(torch.bfloat16)
    out, lse = run_tree(p.upload())
    sync()
    worst = 0.0
    for b in range(p.B):
        for h in range(p.Hkv):
            q, K, V, see = p.unit(b, h)
            want, wl = O.tree_attention(q, K, V, see, p.cfg.scale)
            for i in range(p.N):
                t = np.nonzero(see[i])[0]
                if len(t) == 0:
                    continue
                mass = np.exp(p.cfg.scale * (q[i] @ K[t].T) - wl[i][:, None]) @ np.abs(V[t])
                tol = (mass * (2 * (80 + 4 * np.sqrt(len(t))) * U32 + 2.0 ** -16) + HALF["bf16"] * np.abs(want[i]) * 1.01)
                off = np.abs(f64(out)[b, i, h * p.G:(h + 1) * p.G] - want[i])
                worst = max(worst, float((off / tol).max()))
    say(f"worst error / tolerance {worst:.3f}")
    assert worst <= 1.0


def _check_any(p, out, lse):
    """Outputs and normalisers that need not be finite: the same infinities and NaN as the definition, and finite ones
    within check_tree's tolerance (its errors over the finite keys, as an infinite one's score is exact, and bf16 queries'
    probabilities as above)."""
    got, gl = f64(out), f64(lse)
    for b in range(p.B):
        for h in range(p.Hkv):
            q, K, V, see = p.unit(b, h)
            with np.errstate(all="ignore"):
                want, wl = O.tree_attention(q, K, V, see, p.cfg.scale)
            finite = np.isfinite(K).all(1)
            e = p.score_error(q, np.where(finite[:, None], K, 0.0), see & finite)
            for i in range(p.N):
                t = np.nonzero(see[i] & finite)[0]
                g, z = got[b, i, h * p.G:(h + 1) * p.G], gl[b, i, h * p.G:(h + 1) * p.G]
                assert np.array_equal(np.isnan(g), np.isnan(want[i])), (b, h, i)
                assert np.array_equal(np.isnan(z), np.isnan(wl[i])), (b, h, i, z, wl[i])
                big = np.isinf(want[i])
                assert np.array_equal(g[big], want[i][big]), (b, h, i)
                with np.errstate(all="ignore"):
                    prob = np.exp(p.cfg.scale * (q[i] @ K[t].T) - wl[i][:, None])
                    mass = prob @ np.where(np.isfinite(V[t]), np.abs(V[t]), 0.0)
                    sums = (8 + 4 * np.sqrt(len(t))) * U32
                    rnd = 2.0 ** -16 if p.kv == "bf16" and p.io == "bf16" else 0.0
                    tol = mass * (2 * e[i][:, None] + rnd + 2 * sums) + HALF[p.io] * np.abs(want[i]) * 1.01 + 1e-30
                    off, zoff = np.abs(g - want[i]), np.abs(z - wl[i])
                    ok = np.isfinite(want[i])
                    assert np.all(off[ok] <= tol[ok]), (b, h, i, float((off[ok] / tol[ok]).max()))
                    fin = np.isfinite(wl[i])
                    ltol = e[i] + sums + np.abs(wl[i]) * 2 * U32
                    assert np.all(zoff[fin] <= ltol[fin]), (b, h, i, zoff, ltol)


@pytest.mark.parametrize("kv,io", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("shape", FORMS, ids=_ids)
def test_infinite_keys_and_values_where_queries_look(shape, kv, io):
    """Element 0 of every query is positive.  A key with -inf there has score -inf: its token is as if it were not
    attended to.  One with +inf makes every output of its head NaN.  A value reaches the outputs as probability times value."""
    if shape.get("extra") == 8192 and io != "bf16":
        shape = dict(shape, Hkv=1, extra=0)
    say(f"infinities {shape} {kv} {io}")
    p = Problem(DEV, kv=kv, io=io, seed=5, **shape)
    p.q[..., 0] = p.q[..., 0].abs() + 0.25
    last = p.T[0] - 1                                         # (in the window, where there is one)
    p.k[0, :, last - 20, 0] = -INF
    p.v[0, :, last - 33, 3], p.v[0, :, last - 1, 4] = INF, -INF
    p.v[0, :, last - 33, 5], p.v[0, :, last - 1, 5] = INF, -INF
    p.v[0, :, last - 7, 6] = NAN
    p.k[0, :, p.T[0] + 1, 0] = -INF                           # drafted token 1
    p.v[0, :, p.T[0], 7] = INF
    p.k[1, 0, p.T[1] - 2, 0] = INF
    out, lse = run_tree(p.upload())
    sync()
    _check_any(p, out, lse)


def test_a_query_that_is_not_a_number_stays_by_itself():
    """NaN and infinities in one query's elements reach its own outputs alone."""
    for io in ("f32", "bf16"):
        p, clean = (Problem(DEV, T=(300, 90), N=5, io=io).upload() for _ in range(2))
        p.qd[0, 2, 3, 7], p.qd[1, 4, 6, 0] = NAN, INF
        (out, lse), (want, wl) = run_tree(p), run_tree(clean)
        for b, i, head in ((0, 2, 3), (1, 4, 6)):
            assert bool(out[b, i, head].isnan().all()) and bool(lse[b, i, head].isnan())
            out[b, i, head], lse[b, i, head] = want[b, i, head], wl[b, i, head]
        assert torch.equal(out, want) and torch.equal(lse, wl)


WEIGHT_ROWS = [
    dict(T=(300, 77), N=1, G=4), dict(T=(300, 77), N=5, G=4), dict(T=(200, 64), N=16, G=4), dict(T=(200, 90), N=3, G=1, d=64),
    dict(T=(700, 130), N=64, G=4), dict(T=(150, 90), N=9, G=16), dict(T=(150, 90), N=40, G=8), dict(T=(900, 333), N=7, G=2, s=3, w=100),
    dict(T=(300, 77), N=1, G=4, draft=False), dict(T=(500, 250), N=20, G=2, layout="pages", d=64),
    dict(B=8, Hkv=8, G=4, d=64, T=(8100, 77, 33, 700, 2500, 1, 0, 4000), N=5, extra=700),
]


@pytest.mark.parametrize("dead", ["some", "none", "all"])
@pytest.mark.parametrize("kv,io", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("shape", WEIGHT_ROWS, ids=_ids)
def test_weights_of_infinite_keys_and_of_heads_that_add_nothing(shape, kv, io, dead):
    """Keys of score -inf add 0, of +inf infinity, NaN ones NaN; a head with an infinite lse adds nothing to any of
    them, whatever its query holds."""
    say(f"weights, infinities {shape} {kv} {io} {dead}")
    p = Problem(DEV, kv=kv, io=io, seed=6, **shape)
    g = torch.Generator().manual_seed(7)
    p.q[..., 0] = p.q[..., 0].abs() + 0.25
    lse = 5.0 + torch.rand((p.B, p.N, p.Hkv * p.G), generator=g)
    if dead == "some":
        gone = torch.rand(lse.shape, generator=g) < 0.3
        gone[:, 0, 0], gone[:, 0, -1] = True, True
        lse[gone] = torch.where(torch.rand(lse.shape, generator=g) < 0.5, INF, -INF)[gone]
        p.q[0, 0, 0], p.q[1, 0, -1, 3] = NAN, INF                 # queries of heads that add nothing
    elif dead == "all":
        lse[:] = INF
        lse[:, ::2] = -INF
        p.q[1, 0, 0] = NAN
    for b in range(2):
        last = p.T[b] - 1
        p.k[b, :, last - 20, 0], p.k[b, :, last - 30, 0], p.k[b, :, last - 40, 5] = -INF, INF, NAN
        if p.n[b] > 1:
            p.k[b, :, p.T[b] + 1, 0] = -INF
    prev = torch.rand((p.B, p.Hkv, p.cap), generator=g).to(DEV)
    z = lse.to(DEV)
    got = f64(run_weights(p.upload(), z, torch.zeros_like(prev), prev))
    sync()
    lse = f64(lse).reshape(p.B, p.N, p.Hkv, p.G)
    for b in range(p.B):
        E = p.T[b] + p.n[b]
        for h in range(p.Hkv):
            q, K, _, see = p.unit(b, h)
            live = np.isfinite(lse[b, :, h])
            add = np.zeros(E)
            with np.errstate(all="ignore"):
                for i in range(p.N):
                    for j in range(p.G):
                        if live[i, j]:
                            s = p.cfg.scale * (K @ q[i, j])
                            add += np.where(see[i], np.exp(np.where(see[i], s, 0.0) - lse[b, i, h, j]), 0.0)
            finite, sure = np.isfinite(K).all(1), np.where(np.isfinite(q).all(-1, keepdims=True), q, 0.0)
            e = p.score_error(sure, np.where(finite[:, None], K, 0.0), see & finite).max() + 2.0 ** -17
            want = f64(prev)[b, h, :E] + add
            assert np.array_equal(np.isnan(got[b, h, :E]), np.isnan(want)), (b, h, np.nonzero(np.isnan(got[b, h, :E]) != np.isnan(want)))
            big = np.isinf(want)
            assert np.array_equal(got[b, h, :E][big], want[big])
            ok = np.isfinite(want)
            tol = add[ok] * (e + (8 + 4 * np.sqrt(p.N * p.G)) * U32) + np.abs(want[ok]) * 2 * U32 + 1e-37
            assert np.all(np.abs(got[b, h, :E][ok] - want[ok]) <= tol), (b, h)


@pytest.mark.parametrize("c", [1e-30, 1.6e-38, 1e-38, 1e-44])
@pytest.mark.parametrize("shape", [FORMS[i] for i in (0, 1, 3, 4, 7)], ids=_ids)
def test_the_smallest_scales_average(shape, c):
    """Any positive scale is taken: at these every token has the same weight."""
    for io in ("bf16", "f32") if not shape.get("extra") else ("bf16",):
        p = Problem(DEV, io=io, c=c, **shape).upload()
        out, lse = run_tree(p)
        sync()
        p.check_tree(out, lse)


@pytest.mark.parametrize("io,N", [("bf16", 1), ("f32", 3), ("bf16", 64)])
def test_a_short_row_takes_no_more_parts_than_it_has_passes(io, N):
    """One row of 300 tokens among empty ones, in a capacity of 131072: its 10 frames are at most 10 parts, and an empty
    row is one, each of N rows of 64 outputs, a maximum and a sum in the workspace; nothing else is written there."""
    B, d, cap = 64, 64, 131072
    p = Problem(DEV, B=1, Hkv=1, G=1, d=d, T=300, N=N, io=io, draft=False)
    cfg = cobs.Config(batch=B, num_q_heads=1, num_kv_heads=1, head_dim=d, max_seq_len=cap, rank=0, budget=0, window=0)
    k, v = (torch.zeros((1, 1, cap, d), dtype=torch.bfloat16) for _ in range(2))
    k[:, :, :p.cap], v[:, :, :p.cap] = p.k, p.v
    k, v, q = k.to(DEV).expand(B, 1, cap, d), v.to(DEV).expand(B, 1, cap, d), p.q.to(DEV).expand(B, N, 1, d).contiguous()
    for at in (0, 37):
        seq = torch.zeros(B, dtype=torch.int32, device=DEV)
        seq[at] = 300
        ws = torch.full((cache.tree_workspace_bytes(cfg, N),), 0x7b, dtype=torch.uint8, device=DEV)
        out, lse = torch.empty_like(q), torch.empty((B, N, 1), device=DEV)
        cache.cobs_tree_decode(cfg, q, k, v, seq, None, None, out, ws, lse=lse)
        sync()
        p.check_tree(out[at:at + 1], lse[at:at + 1])
        rest = torch.arange(B, device=DEV) != at
        assert bool((out[rest] == 0).all()) and bool((lse[rest] == -INF).all())
        written = int((ws.view(torch.int32) != 0x7b7b7b7b).sum())
        assert written <= (10 + B - 1) * N * (d + 2), written
