"""The token operators at the ends of what their header allows, in small problems whose answers are known by arithmetic."""

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
