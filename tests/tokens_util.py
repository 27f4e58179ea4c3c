"""Inputs and comparison rules of the token operators' tests."""

import numpy as np
import torch

from oracle import cache as O
from oracle import tokens as R
from paper_2607_09052_amd import tokens
from tests.cache_util import HALF, TORCH, U32, Problem
from tests.gpu_util import f64

E4M3 = tokens.E4M3
NAN_CODE = 0x7f


def rotation_tolerance(x, want, half, inter, scale, out):
    """|rotated - exact| of x [..., d]: cosine and sine are within 3 half steps of fp32 (the reduced angle's rounding, the
    series' own), times the scale one more, the two products and their sum three: 8 (|lo| + |hi|) scale half steps
    of fp32, and the output's rounding."""
    a = np.abs(x)
    pair = np.zeros_like(a)
    lo = 2 * np.arange(half) if inter else np.arange(half)
    hi = lo + 1 if inter else lo + half
    pair[..., lo] = pair[..., hi] = a[..., lo] + a[..., hi]
    return 8 * U32 * pair * abs(scale) + HALF[out] * np.abs(want) * 1.01 + 1e-37


class Problem8(Problem):
    """A Problem whose cache holds 8-bit floats: codes of normal keys and values at scales that are not powers of two,
    NaN codes and NaN scales wherever no token is."""

    def __init__(self, device, seed=0, **over):
        super().__init__(device, kv="bf16", seed=seed, **over)
        rng = np.random.default_rng(seed + 1000)
        table = R.e4m3_values()
        nb = self.cap // self.L
        self.codes, self.scales = [], []
        for i, x in enumerate((self.k, self.v)):
            scale = (2.0 ** rng.integers(-9, -4, size=(self.B, self.Hkv, nb)) * rng.uniform(1, 2, size=(self.B, self.Hkv, nb))).astype(np.float32)
            codes = R.e4m3_codes(np.clip(f64(x) / np.repeat(scale, self.L, -1)[..., None].astype(np.float64), -448, 448))
            for b in range(self.B):
                codes[b, :, self.T[b] + self.n[b]:] = NAN_CODE
                scale[b, :, -(-(self.T[b] + self.n[b]) // self.L):] = np.nan
            self.codes.append(codes)
            self.scales.append(scale)
        self.refresh(table)

    def refresh(self, table=None):
        """k, v: what the codes and scales stand for, in fp64."""
        table = R.e4m3_values() if table is None else table
        self.k, self.v = (torch.from_numpy(table[c] * np.repeat(s, self.L, -1)[..., None].astype(np.float64))
                          for c, s in zip(self.codes, self.scales))

    def upload(self):
        real = self.k, self.v
        self.k, self.v = (torch.from_numpy(c).float() for c in self.codes)     # as numbers, so that the base lays them out
        super().upload()
        to8 = lambda x: torch.nan_to_num(x, nan=float(NAN_CODE)).to(torch.uint8)  # noqa: E731
        if self.layout == "strided":       # rows of 16-byte multiples, NaN codes between them
            base = [x._base if x._base is not None else x for x in (self.kd, self.vd)]
            wide = [torch.nn.functional.pad(to8(x), (0, 8), value=NAN_CODE) for x in base]
            kd, vd = (x[..., :self.d].permute(0, 2, 1, 3) for x in wide)
        else:
            kd, vd = to8(self.kd), to8(self.vd)
        ks, vs = (torch.from_numpy(s) for s in self.scales)
        if self.layout == "pages":
            table = self.pages["block_table"].cpu().long()
            pools = []
            for s in (ks, vs):
                pool = torch.full((kd.shape[0], self.Hkv), float("nan"))
                pool[table] = s.permute(0, 2, 1)
                pools.append(pool)
            ks, vs = pools
        self.cache8 = tokens.Cache8(kd.view(E4M3), vd.view(E4M3), ks.to(self.device).contiguous(), vs.to(self.device).contiguous())
        self.k, self.v = real
        return self

    def check(self, out, lse):
        """Each output within its arithmetic's error.  A score is a sum of d products (fp32 queries: 3 d, each exact), times
        the scales and less the maximum: (terms + 6) half steps of fp32 of sum |q k| c, e below.  A probability moves by 2 e of
        itself (its own score's, the normaliser's), by the exponential's and the scale's product (8 half steps) and, with
        bf16 queries, by its two bf16 parts (2^-17; taken at 2^-16); sums over n tokens add 4 sqrt(n) half steps
        (independent roundings); the output is rounded to its type.  |lse - exact| <= e + the sum's + half a step of it."""
        worst, got, gl, cfg = 0.0, f64(out), f64(lse), self.cfg
        terms = (3 if self.io == "f32" else 1) * self.d
        for b in range(self.B):
            for h in range(self.Hkv):
                q, K, V, see = self.unit(b, h)
                want, wl = O.tree_attention(q, K, V, see, cfg.scale)
                for i in range(self.N):
                    t = np.nonzero(see[i])[0]
                    g, z = got[b, i, h * self.G:(h + 1) * self.G], gl[b, i, h * self.G:(h + 1) * self.G]
                    if len(t) == 0:
                        assert np.all(g == 0.0) and np.all(z == -np.inf), (b, h, i)
                        continue
                    e = cfg.scale * (np.abs(q[i]) @ np.abs(K[t]).T).max(1) * (terms + 6) * U32
                    p = np.exp(cfg.scale * (q[i] @ K[t].T) - wl[i][:, None])
                    sums = (8 + 4 * np.sqrt(len(t))) * U32
                    rnd = 2.0 ** -16 if self.io == "bf16" else 0.0
                    tol = (p @ np.abs(V[t])) * (2 * e[:, None] + rnd + 2 * sums) + HALF[self.io] * np.abs(want[i]) * 1.01 + 1e-30
                    off = np.abs(g - want[i])
                    assert np.all(off <= tol), (b, h, i, float((off / tol).max()))
                    worst = max(worst, float((off / tol).max()))
                    assert np.all(np.abs(z - wl[i]) <= e + sums + np.abs(wl[i]) * 2 * U32), (b, h, i, z, wl[i])
        return worst


def run_decode8(p, ws=None, stream=None):
    ws = tokens.new_decode8_workspace(p.cfg, p.N, p.device) if ws is None else ws
    out = torch.full_like(p.qd, float("nan"))
    lse = torch.full((p.B, p.N, p.Hkv * p.G), float("nan"), device=p.device)
    tokens.cobs_decode8(p.cfg, p.qd, p.cache8, p.seq, p.drafts, p.mask, out, ws, sel=p.sel_d, lse=lse, stream=stream, **p.pages)
    return out, lse


class Appending:
    """New tokens of a few rows and the cache that they go to, on `device`; `want` in fp64 on the host."""

    def __init__(self, device, B=2, Hkv=2, G=2, d=128, L=64, N=5, T=(70, 3), new=None, cap=None, io="bf16", kv="bf16", out="bf16",
                 r=None, inter=False, scale=1.0, base=10000.0, shift=None, layout="contiguous", fused=True, eight=False, seed=0,
                 spread=True, q=True):
        from paper_2607_09052_amd import cobs
        rng = np.random.default_rng(seed)
        gen = torch.Generator().manual_seed(seed)
        T = [T] * B if isinstance(T, int) else list(T)
        new = [N] * B if new is None else list(new)
        cap = cap or max(-(-max(t + n for t, n in zip(T, new)) // L) * L, L)
        self.cfg = cobs.Config(batch=B, num_q_heads=Hkv * G, num_kv_heads=Hkv, head_dim=d, max_seq_len=cap, rank=0, budget=0, window=0,
                               kv_dtype=kv, block_size=L)
        self.B, self.Hkv, self.G, self.d, self.L, self.N, self.cap, self.T, self.new = B, Hkv, G, d, L, N, cap, T, new
        self.io, self.kv, self.out, self.inter, self.scale, self.eight, self.device = io, kv, out, inter, scale, eight, device
        rows = torch.randn((B, N, Hkv * (G + 2), d), generator=gen)
        if spread:                           # magnitudes over many powers of two, so that scales grow now and then
            rows *= 2.0 ** torch.randint(-12, 13, (B, N, Hkv * (G + 2), 1), generator=gen)
        rows = rows.to(TORCH[io])
        self.rows = rows
        r = d if r is None else r
        self.rope = self.positions = None
        self.half = 0
        if r:
            freq = tokens.rope_frequencies(r, base=base)
            self.half = r // 2
            self.freq = freq.double().numpy()
            self.rope = tokens.Rope(freq.to(device), inter, scale)
            if shift is not None:
                at = torch.tensor(T).view(B, 1) + torch.arange(N) + torch.from_numpy(rng.integers(-shift, shift, size=(B, N)))
                self.positions = at.to(torch.int32)
        cut = [0, Hkv * G, Hkv * (G + 1), Hkv * (G + 2)]
        on = rows.to(device)
        parts = [on[:, :, cut[i]:cut[i + 1]] for i in range(3)]
        if not fused:
            parts = [x.contiguous() for x in parts]
        self.qd, self.kn, self.vn = parts
        self.host = [f64(rows[:, :, cut[i]:cut[i + 1]]) for i in range(3)]
        self.with_q = q
        nb = cap // L
        pages = B * nb + 3
        self.table = rng.permutation(pages)[:B * nb].astype(np.int32).reshape(B, nb) if layout == "pages" else None
        shape = (pages, Hkv, L, d) if self.table is not None else (B, Hkv, cap, d)
        sshape = (pages, Hkv) if self.table is not None else (B, Hkv, nb)
        self.layout = layout
        if eight:
            self.codes = [rng.integers(0, 256, size=shape).astype(np.uint8) for _ in range(2)]
            self.scales = [(2.0 ** rng.integers(-20, 3, size=sshape)).astype(np.float32) for _ in range(2)]
        else:
            self.before = [torch.randn(shape, generator=gen).to(TORCH[kv]) for _ in range(2)]
        self.lens = torch.tensor(T, dtype=torch.int32, device=device)

    def fresh(self):
        """New device copies of the cache and the outputs."""
        dev = self.device

        def laid(x, fill):
            if self.layout != "strided":
                return x.to(dev)
            p = torch.full((self.B, self.cap, self.Hkv, self.d + 16), fill, dtype=x.dtype)
            p[..., :self.d] = x.permute(0, 2, 1, 3)
            return p.to(dev)[..., :self.d].permute(0, 2, 1, 3)
        if self.eight:
            k, v = (laid(torch.from_numpy(c), NAN_CODE) for c in self.codes)
            self.cache8 = tokens.Cache8(k, v, *(torch.from_numpy(s).to(dev) for s in self.scales))
        else:
            self.kd, self.vd = (laid(x, float("nan")) for x in self.before)
        self.q_out = torch.full((self.B, self.N, self.Hkv * self.G, self.d), 7.5, dtype=TORCH[self.out], device=dev) if self.with_q else None
        self.after = torch.full((self.B,), -1, dtype=torch.int32, device=dev)
        return self

    def call(self, new_lens=True, stream=None):
        kw = dict(new_lens=torch.tensor(self.new, dtype=torch.int32, device=self.device) if new_lens else None, rope=self.rope,
                  positions=None if self.positions is None else self.positions.to(self.device).contiguous(), new_seq_lens=self.after, stream=stream)
        if self.with_q:
            kw.update(q=self.qd, q_out=self.q_out)
        if self.table is not None:
            kw.update(block_table=torch.from_numpy(self.table).to(self.device), num_pages=self.pages_in_use())
        if self.eight:
            tokens.cobs_append8(self.cfg, self.kn, self.vn, self.cache8, self.lens, **kw)
        else:
            tokens.cobs_append(self.cfg, self.kn, self.vn, self.kd, self.vd, self.lens, **kw)
        return self

    def pages_in_use(self):
        return self.B * (self.cap // self.L) + 3

    def at(self, b):
        if self.positions is not None:
            return self.positions[b].numpy()
        return self.room(b)[0] + np.arange(self.N)         # (the clamped length)

    def turned(self, which, b):
        x = self.host[which][b]
        return R.rotate(x, self.at(b), self.freq, self.inter, self.scale) if self.half and which < 2 else x

    def check_queries(self):
        if not self.with_q:
            return
        got = f64(self.q_out)
        for b in range(self.B):
            n = min(max(self.new[b], 0), self.N)
            want = self.turned(0, b)
            tol = rotation_tolerance(self.host[0][b], want, self.half, self.inter, self.scale, self.out)
            assert np.all(np.abs(got[b, :n] - want[:n]) <= tol[:n]), float((np.abs(got[b, :n] - want[:n]) / tol[:n]).max())
            assert np.all(got[b, n:] == 7.5)

    def room(self, b):
        T = min(max(self.T[b], 0), self.cap)
        return T, min(min(max(self.new[b], 0), self.N), self.cap - T)

    def place(self, b, t):
        """Index of a token's rows [Hkv, d]; None where its page is out of range."""
        if self.table is None:
            return (b, slice(None), t)
        page = int(self.table[b, t // self.L])
        return (page, slice(None), t % self.L) if 0 <= page < self.pages_in_use() else None

    def check_cache(self):
        """A bf16 or fp32 cache: keys within the rotation's error, values the input rounded, all else as it was."""
        got = [f64(x) for x in (self.kd, self.vd)]
        for which in (0, 1):
            want, tol = f64(self.before[which]), np.zeros(self.before[which].shape)
            for b in range(self.B):
                T, n = self.room(b)
                y = self.turned(1 + which, b)
                if which == 1 or not self.half:
                    y = f64(torch.from_numpy(y).to(TORCH[self.kv]))
                    e = np.zeros_like(y)
                else:
                    e = rotation_tolerance(self.host[1][b], y, self.half, self.inter, self.scale, self.kv)
                for i in range(n):
                    at = self.place(b, T + i)
                    if at is not None:
                        want[at], tol[at] = y[i], e[i]
            off = np.abs(got[which] - want)
            assert np.all(off <= tol), (which, float(off.max()), np.argwhere(off > tol)[:3].tolist())
        self.check_lens()

    def check_lens(self):
        for b in range(self.B):
            T, n = self.room(b)
            assert int(self.after[b]) == T + n, b

    def check_cache8(self):
        """Codes and scales of every block: a rotated key's code is one of those that the definition gives for values within the
        rotation's error, a value's the definition's own; the rest as it was."""
        got = [x.cpu().numpy() for x in self.cache8[:2]]
        gs = [x.cpu().numpy() for x in self.cache8[2:]]
        table = R.e4m3_values()
        for which in (0, 1):
            want, ws = self.codes[which].copy(), self.scales[which].copy()
            seen = np.zeros(want.shape, dtype=bool)            # codes compared below, with a tolerance
            for b in range(self.B):
                T, n = self.room(b)
                x, y = self.host[1 + which][b], self.turned(1 + which, b)
                exact = which == 1 or not self.half
                e = np.zeros_like(y) if exact else rotation_tolerance(x, y, self.half, self.inter, self.scale, "f32")
                i = 0
                while i < n:
                    j, lo = (T + i) // self.L, (T + i) % self.L
                    m = min(self.L - lo, n - i)
                    at = self.place(b, j * self.L)
                    i += m
                    if at is None:
                        continue
                    for h in range(self.Hkv):
                        sl = (b, h, j) if self.table is None else (at[0], h)
                        blk = (b, h, slice(j * self.L, (j + 1) * self.L)) if self.table is None else (at[0], h)
                        new, tol = y[i - m:i, h], e[i - m:i, h]
                        old = float(ws[sl])
                        codes, scale = R.append_block(want[blk], old, lo, new)
                        if not exact and float(gs[which][sl]) != scale:
                            # a largest element within its error of a border between two scales
                            top = np.abs(new)
                            options = {max(R.scale_for((top + s * tol).max()), old if lo else 0.0) for s in (-1, 1)}
                            assert float(gs[which][sl]) in options, (which, b, h, j)
                            scale = float(gs[which][sl])
                            codes, _ = R.append_block(want[blk], max(scale, old), lo, new) if scale >= old else (codes, scale)
                        want[blk], ws[sl] = codes, scale
                        if exact:
                            continue
                        rows = slice(lo, lo + m)
                        value = table[got[which][blk][rows]] * scale
                        step = np.maximum(np.abs(new) * 2.0 ** -4, scale * 2.0 ** -10)
                        assert np.all(np.abs(value - new) <= step * 1.0001 + tol), (which, b, h, j)
                        # and no more than a few codes off the definition's, those of values at a tie
                        ties = np.abs(np.abs(value - new) - np.abs(table[codes[rows]] * scale - new)) <= 2.1 * tol
                        assert np.all((got[which][blk][rows] == codes[rows]) | ties), (which, b, h, j)
                        flags = np.zeros(got[which][blk].shape, dtype=bool)
                        flags[rows] = True
                        seen[blk] = flags
            same = (got[which] == want) | seen | (((got[which] & 127) == 127) & ((want & 127) == 127))
            assert np.all(same), (which, np.argwhere(~same)[:4].tolist(), got[which][~same][:4], want[~same][:4])
            assert np.array_equal(gs[which], ws), which
        self.check_lens()
