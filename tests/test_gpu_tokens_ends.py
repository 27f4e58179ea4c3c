"""The token operators at the ends of what their header allows, in small problems whose answers are known by arithmetic."""

import math
from decimal import Decimal, localcontext

import numpy as np
import pytest
import torch

from oracle import tokens as R
from paper_2607_09052_amd import cobs, tokens
from tests.cache_util import TORCH, U32
from tests.gpu_util import DEV, f64, say, sync
from tests.tokens_util import E4M3

pytestmark = pytest.mark.gpu


# ----------------------------------------------------------- probabilities --
@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("d,G,N", [(64, 1, 1), (64, 4, 4), (128, 16, 1), (128, 1, 2)])
def test_probabilities_of_up_to_16_rows_enter_with_all_their_bits(d, G, N, io):
    """A token of value 1 and probability p below the largest, and five of the largest score whose values add up to -p but for
    2^-18: what is left of the sum shows how p was rounded for its product.

    The error allowed, in half steps u = 2^-24 of fp32: p's exponent is at most 1 and rounded twice (2 u ln 2), the exponential is
    within one step (2 u), p is at most 0.8: 2.7 u.  Three products of bf16 parts add up values of at most 1, each by
    no more than 8 roundings: 24 u.  Parts of 16 bits would be off by up to 2^-18 = 64 u, and by more than half of that in some row."""
    say(f"probabilities {d} {G} {N} {io}")
    B, Hkv, L, tail = 64, 2, 32, 5
    cfg = cobs.Config(batch=B, num_q_heads=Hkv * G, num_kv_heads=Hkv, head_dim=d, max_seq_len=L, rank=0, budget=0, window=0,
                      block_size=L, softmax_scale=0.125)
    first = torch.linspace(2.0, 5.5, B).bfloat16()
    q = torch.zeros((B, N, Hkv * G, d))
    q[..., 0] = first.float().view(B, 1, 1)
    p = np.exp(-0.125 * f64(first))
    k, v = (np.zeros((B, Hkv, L, d), dtype=np.uint8) for _ in range(2))
    k[:, :, 0, 0] = R.e4m3_codes(-1.0)
    v[:, :, 0] = R.e4m3_codes(256.0)
    rest = -256.0 * p
    for i in range(1, 1 + tail):
        code = R.e4m3_codes(rest)
        v[:, :, i] = code[:, None, None]
        rest = rest - R.e4m3_values()[code]
    assert np.all(np.abs(rest) <= 2.0 ** -10)
    scales = torch.ones((B, Hkv, 1), device=DEV)
    c8 = tokens.Cache8(*(torch.from_numpy(x).to(DEV).view(E4M3) for x in (k, v)), scales, scales / 256)
    qd = q.to(TORCH[io]).to(DEV)
    out = torch.empty_like(qd)
    lens = torch.full((B,), 1 + tail, dtype=torch.int32, device=DEV)
    tokens.cobs_decode8(cfg, qd, c8, lens, None, None, out, tokens.new_decode8_workspace(cfg, N, DEV))
    sync()
    want = (-rest / 256.0 / (p + tail))[:, None, None, None]
    off = np.abs(f64(out) - want) * (p + tail)[:, None, None, None]
    say(f"largest error {off.max() / U32:.1f} half steps")
    assert np.all(off <= 27 * U32 + 2.0 ** -8 * np.abs(want) * (p + tail)[:, None, None, None])


# ------------------------------------------------------------------ angles --
PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803482534211706798")


def exact_turn(t, f):
    """Cosine and sine of t f, whose exact product is reduced with 100 digits."""
    with localcontext() as ctx:
        ctx.prec = 160
        a = float((Decimal(t) * Decimal(f)) % (2 * PI))
    return math.cos(a), math.sin(a)


FAR_FREQUENCIES = [2.0 ** 20, 2.0 ** 20 - 2.0 ** -4, 543210.9375, 12345.678, 1.0, 0.9999999, 1.0 / 3.0, 1e-6]
FAR_POSITIONS = [(1 << 31) - 1, -(1 << 31), (1 << 31) - 12345, -(1 << 30) - 1, 1 << 29, 987654321, 4099, -7, 0]


def _turned(positions, frequencies):
    """Cosines and sines [positions, frequencies] that a rotation of (1, 0) gives, 8 pairs at a time."""
    x = torch.zeros((1, len(positions), 1, 64), device=DEV)
    x[..., :8] = 1.0
    y = torch.empty_like(x)
    at = torch.tensor([positions], dtype=torch.int64).to(torch.int32).to(DEV)
    freq = torch.zeros(8)
    freq[:len(frequencies)] = torch.tensor(frequencies, dtype=torch.float64).float()
    tokens.cobs_rotate(x, tokens.Rope(freq.to(DEV)), at, y)
    sync()
    n = len(frequencies)
    return freq[:n].double().tolist(), f64(y)[0, :, 0, :n], f64(y)[0, :, 0, 8:8 + n]


def test_angles_up_to_2_51():
    """Every position at frequencies of up to 2^20: the product of both has up to 55 bits."""
    freq, cos, sin = _turned(FAR_POSITIONS, FAR_FREQUENCIES)
    for i, t in enumerate(FAR_POSITIONS):
        for j, f in enumerate(freq):
            c, s = exact_turn(t, f)
            # (the tolerance of a rotation of (1, 0) in fp32: rotation_tolerance)
            assert abs(cos[i, j] - c) <= 8 * U32 + U32 * abs(c), (t, f)
            assert abs(sin[i, j] - s) <= 8 * U32 + U32 * abs(s), (t, f)


def test_angles_past_2_51_give_nan():
    far = [2.0 ** 21, 2.0 ** 22, 2.0 ** 31, 1e12, 1e20, 1e30, 3e38, math.inf]
    freq, cos, sin = _turned([(1 << 31) - 1, -(1 << 31), 1 << 30, 1, 0], far)
    for i, t in enumerate(((1 << 31) - 1, -(1 << 31), 1 << 30, 1, 0)):
        for j, f in enumerate(freq):
            if abs(t) * f <= 2.0 ** 51:                    # (0 times infinity is not)
                c, s = exact_turn(t, f)
                assert abs(cos[i, j] - c) <= 9 * U32 and abs(sin[i, j] - s) <= 9 * U32, (t, f)
            else:
                assert np.isnan(cos[i, j]) and np.isnan(sin[i, j]), (t, f)


# --------------------------------------------------------- many workgroups --
def test_unpack8_of_more_blocks_than_a_launch_takes():
    """4096 rows of up to 128k tokens in blocks of 32: 2^24 blocks and rows, of which a few hold tokens."""
    B, T, L, d = 4096, 1 << 17, 32, 64
    cfg = cobs.Config(batch=B, num_q_heads=1, num_kv_heads=1, head_dim=d, max_seq_len=T, rank=0, budget=0, window=0, block_size=L)
    pages = 12
    table = torch.full((B, T // L), -1, dtype=torch.int32)
    lens = torch.zeros(B, dtype=torch.int32)
    held = {}
    for page, (b, j, n) in enumerate(((0, 0, 5), (1, 4095, 32), (2047, 7, 1), (2048, 0, 32), (2049, 4095, 31), (4095, 0, 32), (4095, 4095, 32))):
        table[b, j] = page + 2
        lens[b] = max(int(lens[b]), j * L + n)
        held[page + 2] = n
    c8 = tokens.new_cache8(cfg, DEV, num_pages=pages)
    gen = torch.Generator().manual_seed(1)
    for x in c8[:2]:
        x.copy_(torch.randn(x.shape, generator=gen).to(E4M3))
    for x in c8[2:]:
        x.copy_(2.0 ** torch.randint(-3, 4, x.shape, generator=gen))
    k, v = (torch.full((pages, 1, L, d), 9.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    table = table.to(DEV)
    tokens.cobs_unpack8(cfg, c8, lens.to(DEV), k, v, block_table=table, num_pages=pages, out_block_table=table, out_num_pages=pages)
    sync()
    for got, codes, scale in ((k, c8.k, c8.k_scale), (v, c8.v, c8.v_scale)):
        want = torch.full_like(got, 9.0)
        for page, n in held.items():
            want[page, :, :n] = (codes[page, :, :n].float() * scale[page].view(1, 1, 1)).bfloat16()
        assert torch.equal(got, want)


def test_rotation_of_more_tokens_than_a_launch_takes():
    """2^27 tokens of one head and a few more, 8 to a workgroup, in place."""
    n, d = (1 << 27) + 13, 64
    assert torch.cuda.mem_get_info()[0] > 4 * n * d
    rope = tokens.Rope(tokens.rope_frequencies(d).to(DEV))
    few = torch.ones((1, 5, 1, d), dtype=torch.bfloat16, device=DEV)
    tokens.cobs_rotate(few, rope, torch.arange(5, dtype=torch.int32, device=DEV).view(1, 5), few)
    x = torch.ones((1, n, 1, d), dtype=torch.bfloat16, device=DEV)
    at = (torch.arange(n, dtype=torch.int32, device=DEV) % 5).view(1, n)
    tokens.cobs_rotate(x, rope, at, x)
    sync()
    for i in range(0, n, 1 << 24):
        piece = slice(i, min(n, i + (1 << 24)))
        assert torch.equal(x[0, piece], few[0, at[0, piece].long()]), i
