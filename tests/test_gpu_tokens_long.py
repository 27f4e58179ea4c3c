"""The token operators' attention over long rows, whose parts go by the rows' lengths or take more frames than one
table describes, and appends whose workgroups take several heads of large blocks in turn."""

import math

import numpy as np
import pytest
import torch

from oracle import cache as O
from oracle import tokens as R
from paper_2607_09052_amd import cobs, tokens
from tests.cache_util import HALF, TORCH, U32, to_mask, tree_bits
from tests.gpu_util import DEV, f64, say, sync
from tests.tokens_util import E4M3, Appending

pytestmark = pytest.mark.gpu


class Long8:
    """A call of cobs_decode8 over long rows, made on the GPU: normal keys and values as codes, scales that are no powers of two,
    NaN codes and scales wherever no token is.  One unit at a time is brought to the host."""

    def __init__(self, B, Hkv, G, d, N, T, L=64, io="bf16", paged=False, draft=False, seed=0):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        rng = np.random.default_rng(seed)
        n = N if draft else 0
        nb = -(-(max(T) + n) // L)
        self.B, self.Hkv, self.G, self.d, self.N, self.T, self.L, self.io, self.n, self.nb = B, Hkv, G, d, N, T, L, io, n, nb
        self.cfg = cobs.Config(batch=B, num_q_heads=Hkv * G, num_kv_heads=Hkv, head_dim=d, max_seq_len=nb * L, rank=0, budget=0, window=0, block_size=L)
        E = torch.tensor(T, device=DEV).view(B, 1, 1) + n
        dead = torch.arange(nb * L, device=DEV).view(1, 1, -1) >= E
        empty = torch.arange(nb, device=DEV).view(1, 1, -1) * L >= E
        self.codes, self.scales = [], []
        for _ in range(2):
            x = torch.randn((B, Hkv, nb * L, d), generator=gen, device=DEV).to(E4M3).view(torch.uint8)
            self.codes.append(x.masked_fill_(dead.unsqueeze(-1), 0x7f))
            s = 0.25 + 0.75 * torch.rand((B, Hkv, nb), generator=gen, device=DEV)
            self.scales.append(s.masked_fill_(empty, math.nan))
        self.q = torch.randn((B, N, Hkv * G, d), generator=gen, device=DEV).to(TORCH[io])
        self.seq = torch.tensor(T, dtype=torch.int32, device=DEV)
        self.bits = [tree_bits(N, rng) for _ in range(B)] if draft else None
        self.pages = {}
        self.table = torch.from_numpy(rng.permutation(B * nb).astype(np.int32)).view(B, nb).to(DEV) if paged else None

    def run(self, ws=None):
        def pool(x, shape):                                # [B, Hkv, nb, ...] to [pages, Hkv, ...]
            y = torch.empty(shape, dtype=x.dtype, device=DEV)
            y[self.table.long()] = x.transpose(1, 2)
            return y
        B, Hkv, nb, L, d = self.B, self.Hkv, self.nb, self.L, self.d
        codes, scales, pages = self.codes, self.scales, {}
        if self.table is not None:
            codes = [pool(x.view(B, Hkv, nb, L, d), (B * nb, Hkv, L, d)) for x in codes]
            scales = [pool(x, (B * nb, Hkv)) for x in scales]
            pages = dict(block_table=self.table, num_pages=B * nb)
        drafts = mask = None
        if self.n:
            drafts, mask = torch.full((B,), self.n, dtype=torch.int32, device=DEV), to_mask(self.bits, DEV)
        ws = tokens.new_decode8_workspace(self.cfg, self.N, DEV) if ws is None else ws
        out, lse = torch.full_like(self.q, math.nan), torch.full((B, self.N, Hkv * self.G), math.nan, device=DEV)
        tokens.cobs_decode8(self.cfg, self.q, tokens.Cache8(*codes, *scales), self.seq, drafts, mask, out, ws, lse=lse, **pages)
        sync()
        return out, lse

    def parts(self):
        """Parts of a context, by the bytes that the workspace has for them."""
        up = lambda x: -(-x // 256) * 256  # noqa: E731
        rows = self.B * self.Hkv * self.N * self.G
        have = tokens.decode8_workspace_bytes(self.cfg, self.N) - 16384
        return next(n for n in range(1, 129) if up(8 * n * rows) + up(4 * n * rows * self.d) == have)

    def check(self, out, lse, units):
        """The units' outputs and log sums, by the bounds of Problem8.check."""
        table, worst = R.e4m3_values(), 0.0
        for b, h in units:
            E = self.T[b] + self.n
            K, V = (table[c[b, h, :E].cpu().numpy()] * np.repeat(f64(s[b, h]), self.L)[:E, None] for c, s in zip(self.codes, self.scales))
            heads = slice(h * self.G, (h + 1) * self.G)
            q = f64(self.q[b, :, heads]).reshape(-1, self.d)
            got, gl = f64(out[b, :, heads]).reshape(-1, self.d), f64(lse[b, :, heads]).reshape(-1)
            if E == 0:
                assert np.all(got == 0.0) and np.all(gl == -np.inf)
                continue
            see = O.visible(self.T[b], self.n, self.N, self.L, 0, None, None if self.bits is None else self.bits[b])
            see = np.repeat(see, self.G, 0)
            c, terms = self.cfg.scale, (3 if self.io == "f32" else 1) * self.d
            s = np.where(see, c * (q @ K.T), -np.inf)
            top = s.max(1)
            wl = top + np.log(np.exp(s - top[:, None]).sum(1))
            p = np.exp(s - wl[:, None])
            want, mass = p @ V, p @ np.abs(V)
            e = c * (np.abs(q) @ np.abs(K).T * see).max(1) * (terms + 6) * U32
            sums = (8 + 4 * np.sqrt(see.sum(1))) * U32
            rnd = 2.0 ** -16 if self.io == "bf16" else 0.0
            tol = mass * (2 * e + rnd + 2 * sums)[:, None] + HALF[self.io] * np.abs(want) * 1.01 + 1e-30
            off = np.abs(got - want)
            assert np.all(off <= tol), (b, h, float((off / tol).max()))
            assert np.all(np.abs(gl - wl) <= e + sums + np.abs(wl) * 2 * U32), (b, h)
            worst = max(worst, float((off / tol).max()))
        say(f"worst error / tolerance {worst:.3f}")


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("shape,parts", [
    # of a batch of 16 rows 4 parts on average, by the rows' lengths, joined by the last workgroup of a (row, KV head)
    (dict(B=16, Hkv=8, G=1, d=128, N=1, T=[4100, 0, 1, 31, 4097] + [4000 - 350 * b for b in range(11)]), 4),
    (dict(B=16, Hkv=8, G=4, d=128, N=4, T=[4100 - 256 * b for b in range(16)], draft=True), 4),
    # one long row among short ones: 55 parts of 16 query rows, and one of each other row
    (dict(B=8, Hkv=8, G=16, d=128, N=1, T=[8190, 5, 0, 33, 64, 1, 70, 96]), 8),
    # 64-element heads, three workgroups a CU
    (dict(B=4, Hkv=16, G=2, d=64, N=2, T=[12280, 9000, 17, 3000]), 12),
], ids=str)
def test_parts_by_the_rows_lengths_joined_by_the_last_workgroup(shape, parts, paged, io):
    """Parts go to rows by their lengths where a batch has 4 to 128 a row, each of 32 frames of 32 tokens and more; the last workgroup
    joins up to 128 part rows a KV head of 16 query rows at most.  Twice on one workspace, whose counters are zero again."""
    say(f"joined parts {shape} {paged} {io}")
    p = Long8(io=io, paged=paged, **shape)
    frames, rows = p.nb * p.L // 32, p.N * p.G
    assert p.parts() == parts and 4 <= parts <= 128 and frames >= 32 * parts and rows <= 16 and parts * rows <= 128
    ws = tokens.new_decode8_workspace(p.cfg, p.N, DEV)
    out, lse = p.run(ws)
    assert not ws[:16384].any()
    again = p.run(ws)
    assert not ws[:16384].any() and torch.equal(out, again[0]) and torch.equal(lse, again[1])
    p.check(out, lse, [(b, h) for b in range(p.B) for h in {0, p.Hkv - 1}])


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("shape,parts", [
    (dict(B=2, Hkv=2, G=16, d=128, N=32, T=[8260, 700], draft=True), 8),            # 16 row tiles
    (dict(B=4, Hkv=8, G=8, d=128, N=5, T=[8300, 17, 8200, 0]), 8),                  # 2 of 32 rows, the second of 8
    (dict(B=3, Hkv=8, G=16, d=128, N=1, T=[22000, 300, 21000]), 21),                # one of 16, with too many parts for a workgroup
    (dict(B=4, Hkv=8, G=8, d=64, N=4, T=[24600, 9000, 0, 3000], draft=True), 24),   # (16 parts for fp32 queries)
], ids=str)
def test_parts_by_the_rows_lengths_joined_by_a_launch(shape, parts, paged, io):
    say(f"parts {shape} {paged} {io}")
    p = Long8(io=io, paged=paged, **shape)
    frames, rows = p.nb * p.L // 32, p.N * p.G
    got = p.parts()
    say(f"{got} parts, {frames} frames")
    assert got == parts and 4 <= parts <= 128 and frames >= 32 * parts and (rows > 16 or parts * rows > 128)
    out, lse = p.run()
    again = p.run()
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    p.check(out, lse, [(b, h) for b in range(p.B) for h in {0, p.Hkv - 1}])


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("shape,parts", [
    (dict(B=1, Hkv=8, G=16, d=128, N=64, T=[20001]), 2),                            # 314 frames a part
    (dict(B=1, Hkv=8, G=16, d=64, N=64, T=[26010], paged=True, draft=True), 3),     # 272, of fp32 queries 407
    (dict(B=16, Hkv=1, G=16, d=128, N=64, T=[18011] + [90 * b for b in range(15)], L=128, draft=True), 1),      # 566 in one part
    (dict(B=96, Hkv=16, G=1, d=64, N=1, T=[9001] + [8 * b for b in range(95)], L=32), 1),                      # rows of 16, 282
], ids=str)
def test_frames_beyond_one_table(shape, parts, io):
    """More than 256 frames in a part: the frames' table filled again with outputs, maximum and sum carried over."""
    say(f"tables {shape} {io}")
    p = Long8(io=io, **shape)
    frames = -(-(p.T[0] + p.n) // 32)
    got = p.parts()
    say(f"{got} parts, {frames} frames")
    assert got == parts and frames > 256 * parts
    out, lse = p.run()
    p.check(out, lse, [(0, 0), (0, p.Hkv - 1), (p.B - 1, 0)])
    if not p.n:
        return
    # a NaN among the drafted values of head 0, in the last table: the queries that see it, in its column
    j, column = 5, 37
    p.codes[1][0, 0, p.T[0] + j, column] = 0x7f
    bad, same = p.run()
    nan = torch.zeros_like(out, dtype=torch.bool)
    for i, bits in enumerate(p.bits[0]):
        nan[0, i, :p.G, column] = bool(bits >> j & 1)
    assert 0 < int(nan.sum()) and torch.equal(torch.isnan(bad), nan) and torch.equal(same, lse)
    assert torch.equal(bad[~nan], out[~nan])


# ---------------------------------------------------------- appends, heads --
@pytest.mark.parametrize("shape,io", [
    (dict(B=32, d=128, N=300), "bf16"),           # four heads in turn, their rows in four passes of a workgroup's lanes
    (dict(B=32, d=128, N=300, inter=True, r=64), "f32"),
    (dict(B=32, d=64, N=300), "bf16"),            # in two
    (dict(B=32, d=64, N=300), "f32"),
    (dict(B=64, d=128, N=270), "bf16"),           # all eight
], ids=str)
def test_append8_of_blocks_of_128_by_workgroups_of_several_heads(shape, io):
    """A workgroup takes as many of the 8 heads' keys or values as leave 512 workgroups of the B * 4 blocks * 16: 4, or all."""
    say(f"append8 {shape} {io}")
    B, N = shape["B"], shape["N"]
    p = Appending(DEV, Hkv=8, G=1, L=128, T=[37 * b % 257 for b in range(B)], new=[N - 53 * b % (N // 2) for b in range(B)], io=io, out="bf16",
                  layout="pages", eight=True, **shape).fresh().call()
    sync()
    p.check_cache8()
    p.check_queries()
