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


# Every form of the attention kernels: 32, 64, 128 query rows a workgroup and 256, one part of a context and many.
FORMS = [
    dict(T=(150, 40), N=4), dict(T=(3001, 5), N=3, d=64), dict(T=(200, 33), N=8, G=8, d=64), dict(T=(129, 64), N=8, G=8),
    dict(T=(300, 77), N=33, G=8), dict(T=(1500, 700), N=20, G=16, d=64, layout="pages"),
    dict(T=(900, 333), N=16, s=3, w=100), dict(T=(300, 77), N=64, G=16, Hkv=8, extra=8192),
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
