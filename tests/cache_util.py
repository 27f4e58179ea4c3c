"""Inputs and comparison rules of the cache operators' tests."""

import numpy as np
import torch

from oracle import cache as O
from paper_2607_09052_amd import cache, cobs
from tests.gpu_util import f64

U32 = 2.0 ** -24          # half a step of fp32
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


def tree_bits(N, rng, chain=False):
    """Ancestor bits, itself included, of a random tree (or a chain)."""
    bits = []
    for i in range(N):
        parent = i - 1 if chain else i - 1 - int(rng.integers(0, 4))
        bits.append((1 << i) | (bits[parent] if parent >= 0 else 0))
    return bits


def to_mask(rows, device):
    """Python words to the signed 64-bit tensor that carries them."""
    return torch.tensor([[x - (1 << 64) if x >> 63 else x for x in r] for r in rows], dtype=torch.int64, device=device)


class Problem:
    """One call's inputs on `device`, and their fp64 forms per (row, KV head)."""

    def __init__(self, device, B=2, Hkv=2, G=4, d=128, L=64, T=(300, 77), N=8, drafts=None, kv="bf16", io="f32",
                 s=-1, w=0, layout="contiguous", seed=0, draft=True, bits=None, extra=0, scale=0.0, c=0.0):
        rng = np.random.default_rng(seed)
        gen = torch.Generator().manual_seed(seed)
        T = [T] * B if isinstance(T, int) else list(T)
        assert len(T) == B
        drafts = ([N] * B if drafts is None else list(drafts)) if draft else [0] * B
        cap = -(-(max(t + n for t, n in zip(T, drafts)) + extra) // L) * L
        cap = max(cap, L)
        self.cfg = cobs.Config(batch=B, num_q_heads=Hkv * G, num_kv_heads=Hkv, head_dim=d, max_seq_len=cap, rank=0,
                               budget=max(s, 0), window=w, kv_dtype=kv, block_size=L, softmax_scale=c)
        self.B, self.Hkv, self.G, self.d, self.L, self.N, self.cap = B, Hkv, G, d, L, N, cap
        self.T, self.n, self.kv, self.io, self.device, self.draft = T, drafts, kv, io, device, draft
        self.k = torch.randn((B, Hkv, cap, d), generator=gen).to(TORCH[kv])
        self.v = torch.randn((B, Hkv, cap, d), generator=gen).to(TORCH[kv])
        self.q = ((1.0 + scale) * torch.randn((B, N, Hkv * G, d), generator=gen)).to(TORCH[io])
        self.bits = None
        if draft:
            self.bits = bits if bits is not None else [tree_bits(N, rng) for _ in range(B)]
        self.sel = None
        if s >= 0:
            self.sel = np.full((B, Hkv, s), -1, dtype=np.int32)
            for b in range(B):
                nc = -(-max(0, T[b] - w) // L)
                for h in range(Hkv):
                    m = min(s, nc)
                    self.sel[b, h, :m] = np.sort(rng.choice(nc, m, replace=False)) if m else []
        self.layout = layout
        self.rng = rng

    def upload(self):
        """The device tensors: self.args (keyword arguments that the attention calls share)."""
        dev = self.device
        k, v, extra = self.k, self.v, {}
        if self.layout == "pages":
            nb = self.cap // self.L
            perm = torch.from_numpy(self.rng.permutation(self.B * nb + 3)[:self.B * nb].astype(np.int32)).view(self.B, nb)
            pool = []
            for x in (k, v):
                p = torch.full((self.B * nb + 3, self.Hkv, self.L, self.d), float("nan"), dtype=x.dtype)
                p[perm.long()] = x.view(self.B, self.Hkv, nb, self.L, self.d).permute(0, 2, 1, 3, 4)
                pool.append(p.to(dev))
            k, v = pool
            extra = dict(block_table=perm.to(dev), num_pages=k.shape[0])
        elif self.layout == "strided":      # [B, T, H, d + 8], heads inside tokens, NaN between the rows
            out = []
            for x in (k, v):
                p = torch.full((self.B, self.cap, self.Hkv, self.d + 8), float("nan"), dtype=x.dtype)
                p[..., :self.d] = x.permute(0, 2, 1, 3)
                out.append(p.to(dev)[..., :self.d].permute(0, 2, 1, 3))
            k, v = out
        else:
            k, v = k.to(dev), v.to(dev)
        self.seq = torch.tensor(self.T, dtype=torch.int32, device=dev)
        self.drafts = torch.tensor(self.n, dtype=torch.int32, device=dev) if self.draft else None
        self.mask = to_mask(self.bits, dev) if self.draft else None
        self.sel_d = None if self.sel is None else torch.from_numpy(self.sel).to(dev)
        self.pages = extra
        self.kd, self.vd, self.qd = k, v, self.q.to(dev)
        return self

    def see(self, b, h):
        sel = None if self.sel is None else [int(x) for x in self.sel[b, h] if x >= 0]
        return O.visible(self.T[b], self.n[b], self.N, self.L, self.cfg.window, sel,
                         self.bits[b] if self.draft else None)

    def unit(self, b, h):
        """fp64 q [N, G, d], K, V [T + n, d] and the flags of one (row, KV head)."""
        E = self.T[b] + self.n[b]
        q = f64(self.q)[b].reshape(self.N, self.Hkv, self.G, self.d)[:, h]
        return q, f64(self.k[b, h, :E]), f64(self.v[b, h, :E]), self.see(b, h)

    def score_error(self, q, K, see):
        """Largest error [N, G] that the score arithmetic allows in a score c q.k of a query: the roundings of the
        fp32 sums (an fp32 query over bf16 keys is three bf16 operands, so 3 d products, each exact) and 4 more."""
        terms = 3 * self.d if (self.kv == "bf16" and self.io == "f32") else self.d
        big = np.zeros(q.shape[:2])
        for i in range(self.N):
            t = np.nonzero(see[i])[0]
            if len(t):
                big[i] = (np.abs(q[i]) @ np.abs(K[t]).T).max(1)
        return self.cfg.scale * big * (terms + 4) * U32

    def check_tree(self, out, lse):
        """Each output within its arithmetic's error: with |score error| <= e, every probability moves by 2 e of itself
        at most (its own score and the normaliser's), by the exponential's (8 steps of fp32) and, with bf16 outputs
        over bf16 caches, by its rounding for the product with the values (2^-8; taken at 2^-7); sums over n tokens add 4 sqrt(n) half steps (independent roundings); the
        output is rounded to its type.  |lse - exact| <= e + the sum's error + half a step of it."""
        cfg = self.cfg
        worst = 0.0
        got, gl = f64(out), f64(lse)
        for b in range(self.B):
            for h in range(self.Hkv):
                q, K, V, see = self.unit(b, h)
                want, wl = O.tree_attention(q, K, V, see, cfg.scale)
                e = self.score_error(q, K, see)
                rnd = 2.0 ** -7 if self.kv == "bf16" and self.io == "bf16" else 0.0
                for i in range(self.N):
                    t = np.nonzero(see[i])[0]
                    g = got[b, i, h * self.G:(h + 1) * self.G]
                    z = gl[b, i, h * self.G:(h + 1) * self.G]
                    if len(t) == 0:
                        assert np.all(g == 0.0) and np.all(z == -np.inf), (b, h, i)
                        continue
                    p = np.exp(cfg.scale * (q[i] @ K[t].T) - wl[i][:, None])
                    mass = p @ np.abs(V[t])
                    sums = (8 + 4 * np.sqrt(len(t))) * U32
                    tol = mass * (2 * e[i][:, None] + rnd + 2 * sums) + HALF[self.io] * np.abs(want[i]) * 1.01 + 1e-30
                    off = np.abs(g - want[i])
                    assert np.all(off <= tol), (b, h, i, float((off / tol).max()))
                    worst = max(worst, float((off / tol).max()))
                    ltol = e[i] + sums + np.abs(wl[i]) * 2 * U32
                    assert np.all(np.abs(z - wl[i]) <= ltol), (b, h, i, np.abs(z - wl[i]), ltol)
        return worst

    def check_weights(self, weights, lse, prev, before):
        """weights against fp64: a term moves by its score's error, the exponential's (8 steps) and the rounding of
        score - lse (half a step of |score| + |lse|, at most 2^7 here: 2^-17); the sum of m terms adds sqrt(m)
        half steps (4 of them), as does the last addition."""
        got, z = f64(weights), f64(lse).reshape(self.B, self.N, self.Hkv, self.G)
        for b in range(self.B):
            E = self.T[b] + self.n[b]
            for h in range(self.Hkv):
                q, K, _, see = self.unit(b, h)
                add = O.attention_weights(q, K, see, z[b, :, h], self.cfg.scale)
                e = self.score_error(q, K, see).max() + 2.0 ** -17 + (8 + 4 * np.sqrt(self.N * self.G)) * U32
                base = prev[b, h, :E] if prev is not None else np.zeros(E)
                tol = add * e + (np.abs(base) + add) * 2 * U32 + 1e-37
                off = np.abs(got[b, h, :E] - (base + add))
                assert np.all(off <= tol), (b, h, float((off / tol).max()), int((off / tol).argmax()))
                assert np.array_equal(got[b, h, E:], before[b, h, E:])


def run_tree(p, stream=None, ws=None):
    ws = cache.new_tree_workspace(p.cfg, p.N, p.device) if ws is None else ws
    out = torch.full_like(p.qd, float("nan"))
    lse = torch.full((p.B, p.N, p.Hkv * p.G), float("nan"), device=p.device)
    cache.cobs_tree_decode(p.cfg, p.qd, p.kd, p.vd, p.seq, p.drafts, p.mask, out, ws, sel=p.sel_d, lse=lse,
                           stream=stream, **p.pages)
    return out, lse


def run_weights(p, lse, weights, prev=None, stream=None):
    cache.cobs_attention_weights(p.cfg, p.qd, p.kd, p.vd, p.seq, p.drafts, p.mask, lse, weights, prev=prev,
                                 sel=p.sel_d, stream=stream, **p.pages)
    return weights
