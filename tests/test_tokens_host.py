"""The token operators without a GPU: the oracle's identities, and the refusals of the C entry points and of
the binding, which come before any launch."""

import ctypes
import math
import os
import re

import numpy as np
import pytest
import torch

from oracle import tokens as R
from paper_2607_09052_amd import cobs, tokens

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# ------------------------------------------------------------------ oracle --
def test_a_rotation_keeps_lengths_and_shows_relative_positions():
    r = np.random.default_rng(0)
    q, k = r.normal(size=(1, 1, 64)), r.normal(size=(1, 1, 64))
    f = tokens.rope_frequencies(32).double().numpy()
    for inter in (False, True):
        turn = lambda x, t: R.rotate(x, [t], f, inter)[0, 0]  # noqa: E731
        assert abs(np.linalg.norm(turn(q, 77)) - np.linalg.norm(q)) < 1e-12
        assert abs(turn(q, 1000) @ turn(k, 990) - turn(q, 10) @ turn(k, 0)) < 1e-10
        assert np.array_equal(turn(q, 5)[32:], q[0, 0, 32:])
        assert np.allclose(R.rotate(R.rotate(q, [9], f, inter), [-9], f, inter), q, atol=1e-14)


def test_the_two_layouts_differ_by_the_order_of_elements():
    x = np.random.default_rng(1).normal(size=(3, 2, 16))
    f = tokens.rope_frequencies(16).double().numpy()
    order = np.concatenate([np.arange(0, 16, 2), np.arange(1, 16, 2)])
    assert np.allclose(R.rotate(x, [1, 2, 3], f, True)[..., order], R.rotate(x[..., order], [1, 2, 3], f), atol=1e-15)


def test_frequencies():
    f = tokens.rope_frequencies(64, base=500.0)
    assert f.dtype == torch.float32 and f.numel() == 32 and f[0] == 1.0
    assert np.allclose(f.double().numpy(), 500.0 ** (-np.arange(32) / 32), rtol=2.0 ** -24)
    assert torch.equal(tokens.rope_frequencies(64, base=500.0, factor=4.0), f / 4)
    g = tokens.rope_frequencies(64, base=500.0, factor=4.0, original_len=1024)
    turns = 1024 * f.double() / (2 * math.pi)
    assert torch.equal(g[turns >= 32], f[turns >= 32]) and torch.equal(g[turns <= 1], f[turns <= 1] / 4)
    assert (g <= f).all() and (g >= f / 4).all() and (g[1:] < g[:-1]).all()


def test_codes_are_the_casts():
    x = torch.cat([torch.linspace(-448, 448, 200001), 2.0 ** -10 * torch.arange(-64.0, 64.0), torch.tensor([0.0, -0.0])])
    want = x.to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(R.e4m3_codes(x.double().numpy()), want)
    every = torch.arange(256).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(R.e4m3_values(), every, equal_nan=True)


def test_scales_are_the_smallest_powers_that_fit():
    for top in (1e-300, 2.0 ** -92, 3e-9, 1.0, 447.9, 448.0, 448.1, 449.0, 896.0, 1e30):
        s = R.scale_for(top)
        assert np.log2(s) % 1 == 0 and top / s <= 448.0 and (s == 2.0 ** -100 or top / (s / 2) > 448.0)
    assert R.scale_for(0.0) == 2.0 ** -100 == R.scale_for(1e-40)


def test_a_block_in_pieces():
    r = np.random.default_rng(2)
    x = r.normal(size=(32, 8)) * 2.0 ** np.arange(32)[:, None] / 64
    codes, scale = np.full((32, 8), 0x7f, np.uint8), 0.0
    for i in range(0, 32, 5):
        codes, scale = R.append_block(codes, scale, i, x[i:i + 5])
    assert scale == R.scale_for(np.abs(x).max())
    assert np.all(np.abs(R.e4m3_values()[codes] * scale - x) <= np.abs(x) * 2.0 ** -4 + 7 * scale * 2.0 ** -10)


# ---------------------------------------------------------------- refusals --
def test_library_exports_what_the_header_declares():
    with open(os.path.join(ROOT, "include", "cobs_tokens.h")) as f:
        declared = sorted(set(re.findall(r"^\s*(?:size_t|cobs_status_t)\s+(cobs_\w+)\s*\(", f.read(), re.M)))
    assert declared == sorted(tokens.EXPORTS)
    for name in declared:
        assert hasattr(cobs.lib(), name)


FAKE, OTHER = 1 << 20, 1 << 24


def _cfg(**over):
    base = dict(batch=2, num_q_heads=8, num_kv_heads=2, head_dim=128, max_seq_len=4096, rank=0, budget=8, window=128)
    base.update(over)
    return cobs.Config(**base)


def _heads(**over):
    base = dict(p=FAKE, stride_b=1 << 16, stride_n=1 << 12, stride_h=128)
    base.update(over)
    return tokens._pack_heads(base["p"] or 0, *list(base.values())[1:])


def _rope(**over):
    base = dict(inv_freq=FAKE, rotary_dim=128, interleaved=0, scale=1.0)
    base.update(over)
    return tokens._pack_rope(base["inv_freq"] or 0, *list(base.values())[1:])


def _kv(**over):
    base = dict(k=FAKE, v=FAKE + 4096, stride_b=1 << 20, stride_h=1 << 19, stride_t=128, block_table=None, num_pages=0)
    base.update(over)
    return cobs._KV(*base.values())


def _kv8(**over):
    base = dict(k=FAKE, v=FAKE + 4096, k_scale=FAKE + 8192, v_scale=FAKE + 16384, stride_b=1 << 20, stride_h=1 << 19, stride_t=128,
                block_table=None, num_pages=0)
    base.update(over)
    return tokens._pack_kv8(*(x or 0 for x in base.values()))


def _ref(x):
    return x if x is None or isinstance(x, bytes) else ctypes.byref(x)


def _rotate(**over):
    a = dict(x=_heads(), io=1, B=2, N=8, H=4, d=128, rope=_rope(), at=FAKE, y=_heads(p=OTHER), out=1)
    a.update(over)
    return tokens.lib().cobs_rotate(_ref(a["x"]), a["io"], a["B"], a["N"], a["H"], a["d"], _ref(a["rope"]), a["at"], _ref(a["y"]), a["out"], None)


@pytest.mark.parametrize("edit,code", [
    (dict(x=None), 1), (dict(y=None), 1), (dict(rope=None), 1), (dict(at=None), 1),
    (dict(x=_heads(p=FAKE + 8)), 1), (dict(y=_heads(p=None)), 1),
    (dict(x=_heads(stride_h=132)), 1), (dict(x=_heads(stride_b=-128)), 1),
    (dict(io=2), 1), (dict(out=3), 1), (dict(B=0), 1), (dict(N=0), 1), (dict(H=0), 1), (dict(d=96), 2), (dict(d=0), 1),
    (dict(rope=_rope(inv_freq=None)), 1), (dict(rope=_rope(rotary_dim=0)), 1), (dict(rope=_rope(rotary_dim=24)), 2),
    (dict(rope=_rope(rotary_dim=144)), 1), (dict(rope=_rope(interleaved=2)), 1), (dict(rope=_rope(scale=math.inf)), 1),
    (dict(rope=_rope(scale=math.nan)), 1),
    (dict(y=_heads(p=OTHER, stride_h=64)), 1),                     # heads that share memory
    (dict(y=_heads(p=OTHER, stride_n=256)), 1), (dict(y=_heads(p=OTHER, stride_b=0)), 1),
    (dict(y=_heads(), out=0), 1), (dict(y=_heads(stride_n=1 << 13, stride_b=1 << 17)), 1),      # x itself, as another type or shape
    (dict(B=1 << 16, N=1 << 14, H=4), 2),
])
def test_rotate_refuses(edit, code):
    assert _rotate(**edit) == code


def _append(eight, cfg=None, **over):
    a = dict(k_new=_heads(), v_new=_heads(p=FAKE + 512), io=1, N=8, kv=_kv8() if eight else _kv(), seq=FAKE, new=FAKE, rope=_rope(), at=FAKE,
             q=_heads(p=FAKE + 1024), q_out=_heads(p=OTHER), out=0, after=OTHER)
    a.update(over)
    fn = tokens.lib().cobs_append8 if eight else tokens.lib().cobs_append
    return fn(_ref((cfg or _cfg()).c_struct()), _ref(a["k_new"]), _ref(a["v_new"]), a["io"], a["N"], _ref(a["kv"]), a["seq"], a["new"],
              _ref(a["rope"]), a["at"], _ref(a["q"]), _ref(a["q_out"]), a["out"], a["after"], None)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("edit,code", [
    (dict(k_new=None), 1), (dict(v_new=None), 1), (dict(k_new=_heads(p=FAKE + 2)), 1), (dict(v_new=_heads(stride_n=4)), 1),
    (dict(kv=None), 1), (dict(seq=None), 1), (dict(io=2), 1), (dict(N=0), 1), (dict(N=1 << 24, q=None, q_out=None), 2),
    (dict(q=None), 1), (dict(q_out=None), 1), (dict(out=2), 1), (dict(q_out=_heads(p=OTHER, stride_n=512)), 1),
    (dict(q_out=_heads(p=FAKE)), 1), (dict(q_out=_heads(p=FAKE + 512)), 1),      # over the keys, over the values
    (dict(q_out=_heads(p=FAKE + 1024), out=0), 1),                 # the queries themselves as another type
    (dict(rope=_rope(rotary_dim=8)), 2), (dict(rope=_rope(rotary_dim=256)), 1),
    (dict(after=FAKE), 1),                                         # over the lengths
])
def test_append_refuses(eight, edit, code):
    assert _append(eight, **edit) == code


def test_caches_whose_keys_are_their_values_are_not_written():
    assert _append(False, kv=_kv(v=FAKE)) == 1 and _append(False, kv=_kv(v=FAKE, block_table=FAKE, num_pages=4)) == 1
    assert _append(True, kv=_kv8(v=FAKE)) == 1 and _append(True, kv=_kv8(v_scale=FAKE + 8192)) == 1
    assert _unpack(dst=_kv(k=OTHER, v=OTHER)) == 1


def test_caches_that_share_rows_and_bad_caches_are_refused():
    for over in (dict(stride_b=0), dict(stride_h=0), dict(stride_t=64), dict(stride_t=130), dict(k=None), dict(v=FAKE + 8),
                 dict(block_table=FAKE, num_pages=0)):
        assert _append(False, kv=_kv(**over)) == 1
        assert _append(True, kv=_kv8(**over)) == 1
    assert _append(True, kv=_kv8(stride_t=1 << 23)) == 2 and _append(True, kv=_kv8(stride_h=136)) == 1
    for name in ("k_scale", "v_scale"):
        assert _append(True, kv=_kv8(**{name: None})) == 1 and _append(True, kv=_kv8(**{name: FAKE + 2})) == 1


@pytest.mark.parametrize("over", [
    dict(stride_b=16), dict(stride_b=(1 << 19) + 128), dict(stride_b=(1 << 20) - 16),           # rows: inside heads, over the last tokens
    dict(stride_h=64), dict(stride_h=128), dict(stride_h=(1 << 19) - 128),                     # heads: inside a token, on tokens
    dict(stride_h=128, stride_t=192), dict(stride_h=64, stride_t=128),                         # heads beside each other in too short a token
    dict(stride_b=256, stride_h=128, stride_t=384),                                            # rows beside each other, too
    dict(stride_t=1 << 19, stride_h=1 << 20),                                                  # a head's tokens over the next's
], ids=str)
def test_caches_whose_rows_or_heads_overlap_are_not_written(over):
    assert _append(False, kv=_kv(**over)) == 1 and _append(True, kv=_kv8(**over)) == 1
    assert _unpack(dst=_kv(k=OTHER, v=OTHER + 4096, **over)) == 1


@pytest.mark.parametrize("over", [
    dict(), dict(stride_t=256, stride_h=128), dict(stride_t=512, stride_h=128, stride_b=256), dict(stride_b=128, stride_t=256, stride_h=1 << 20),
    dict(stride_h=(1 << 19) + 16, stride_b=(1 << 20) + 64),
], ids=str)
def test_layouts_without_overlap_are_taken(over):
    """(as far as the next check, which finds too many tokens)"""
    assert _append(False, kv=_kv(**over), N=1 << 24, q=None, q_out=None) == 2 and _append(True, kv=_kv8(**over), N=1 << 24, q=None, q_out=None) == 2
    one = _cfg(batch=1, num_kv_heads=1, num_q_heads=4)               # strides of dimensions of 1 are not used
    assert _append(False, one, kv=_kv(stride_b=0, stride_h=0), N=(1 << 24) + 1, q=None, q_out=None) == 2


@pytest.mark.parametrize("edit,code", [(dict(num_q_heads=6), 2), (dict(head_dim=96), 2), (dict(block_size=48, max_seq_len=4800), 2),
                                       (dict(max_seq_len=100), 1), (dict(batch=0), 1), (dict(num_kv_heads=3), 1)])
def test_configs_are_refused(edit, code):
    cfg = _cfg(**edit)
    assert _append(False, cfg) == code and _append(True, cfg) == code and _decode(cfg) == code and _unpack(cfg) == code
    assert tokens.decode8_workspace_bytes(cfg, 4) == 0


def _decode(cfg=None, **over):
    a = dict(q=FAKE, io=0, N=8, kv=_kv8(), seq=FAKE, drafts=FAKE, mask=FAKE, sparse=1, sel=FAKE, out=OTHER, lse=FAKE, ws=FAKE, nws=1 << 40)
    a.update(over)
    return tokens.lib().cobs_decode8(_ref((cfg or _cfg()).c_struct()), a["q"], a["io"], a["N"], _ref(a["kv"]), a["seq"], a["drafts"], a["mask"],
                                     a["sparse"], a["sel"], a["out"], a["lse"], a["ws"], a["nws"], None)


@pytest.mark.parametrize("edit,code", [
    (dict(q=None), 1), (dict(q=FAKE + 4), 1), (dict(seq=None), 1), (dict(drafts=None), 1), (dict(mask=None), 1), (dict(mask=FAKE + 4), 1),
    (dict(sel=None), 1), (dict(sparse=0), 1), (dict(sparse=2), 1), (dict(io=2), 1), (dict(N=0), 1), (dict(N=65), 2), (dict(kv=None), 1),
    (dict(kv=_kv8(k=FAKE + 8)), 1), (dict(kv=_kv8(stride_t=64)), 1), (dict(kv=_kv8(block_table=FAKE)), 1), (dict(kv=_kv8(k_scale=None)), 1),
    (dict(out=None), 1), (dict(out=FAKE), 1), (dict(out=OTHER + 4), 1), (dict(ws=None), 3), (dict(ws=FAKE + 16), 3), (dict(nws=1), 3),
])
def test_decode8_refuses(edit, code):
    assert _decode(**edit) == code


def _unpack(cfg=None, **over):
    a = dict(kv=_kv8(), seq=FAKE, first=0, num=64, dst=_kv(k=OTHER, v=OTHER + 4096))
    a.update(over)
    return tokens.lib().cobs_unpack8(_ref((cfg or _cfg()).c_struct()), _ref(a["kv"]), a["seq"], a["first"], a["num"], _ref(a["dst"]), None)


@pytest.mark.parametrize("edit,code", [
    (dict(kv=None), 1), (dict(dst=None), 1), (dict(seq=None), 1), (dict(first=-2), 1), (dict(first=65), 1), (dict(num=-1), 1), (dict(num=65), 1),
    (dict(first=1, num=64), 1), (dict(first=-1, num=65), 1), (dict(dst=_kv(k=FAKE, v=OTHER)), 1), (dict(dst=_kv(k=OTHER, v=FAKE + 8192)), 1),
    (dict(dst=_kv(k=OTHER, v=OTHER + 4096, stride_h=0)), 1), (dict(dst=_kv(k=OTHER, v=OTHER + 4096, block_table=FAKE)), 1),
])
def test_unpack8_refuses(edit, code):
    assert _unpack(**edit) == code


# ----------------------------------------------------------------- binding --
def _tensors(B=2, N=3, Hkv=2, G=4, d=128, T=128):
    cfg = cobs.Config(batch=B, num_q_heads=Hkv * G, num_kv_heads=Hkv, head_dim=d, max_seq_len=T, rank=0, budget=2, window=16)
    bf = torch.bfloat16
    rows = torch.zeros((B, N, Hkv * (G + 2), d), dtype=bf)
    c8 = tokens.new_cache8(cfg, "cpu")
    return dict(cfg=cfg, q=rows[:, :, :Hkv * G], k_new=rows[:, :, Hkv * G:Hkv * (G + 1)], v_new=rows[:, :, Hkv * (G + 1):],
                q_out=torch.zeros((B, N, Hkv * G, d)), c8=c8, k=torch.zeros((B, Hkv, T, d), dtype=bf), v=torch.zeros((B, Hkv, T, d), dtype=bf),
                lens=torch.zeros(B, dtype=torch.int32), rope=tokens.Rope(tokens.rope_frequencies(d)),
                at=torch.zeros((B, N), dtype=torch.int32), new=None, after=None)


def _call_append(eight, **over):
    t = _tensors()
    t.update(over)
    kw = dict(new_lens=t["new"], rope=t["rope"], positions=t["at"], q=t["q"], q_out=t["q_out"], new_seq_lens=t["after"],
              block_table=t.get("table"), num_pages=t.get("pages", 0))
    if eight:
        tokens.cobs_append8(t["cfg"], t["k_new"], t["v_new"], t["c8"], t["lens"], **kw)
    else:
        tokens.cobs_append(t["cfg"], t["k_new"], t["v_new"], t["k"], t["v"], t["lens"], **kw)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("edit,text", [
    (dict(k_new=None), "k_new must"), (dict(k_new=torch.zeros((2, 3, 2, 64), dtype=torch.bfloat16)), "k_new must have shape"),
    (dict(v_new=torch.zeros((2, 3, 2, 128))), "v_new must be torch.bfloat16"), (dict(v_new=torch.zeros((2, 4, 2, 128), dtype=torch.bfloat16)), "v_new must have shape"),
    (dict(k_new=torch.zeros((2, 3, 2, 128), dtype=torch.float16)), "k_new must be"),
    (dict(q=None), "go together"), (dict(q_out=None), "go together"), (dict(q_out=torch.zeros((2, 3, 7, 128))), "q_out must have shape"),
    (dict(lens=None), "seq_lens is required"), (dict(lens=torch.zeros(1, dtype=torch.int32)), "seq_lens holds 1"),
    (dict(new=torch.zeros(2)), "new_lens must be"), (dict(after=torch.zeros(2, dtype=torch.int64)), "new_seq_lens must be"),
    (dict(rope=torch.zeros(64)), "tokens.Rope"), (dict(rope=None), "positions needs rope"),
    (dict(rope=tokens.Rope(torch.zeros(64, dtype=torch.float64))), "inv_freq must be"), (dict(at=torch.zeros((2, 3))), "positions must be"),
    (dict(at=torch.zeros((3, 2), dtype=torch.int32)), "positions must have shape"), (dict(), "on a GPU"),
])
def test_binding_names_the_wrong_argument_of_an_append(eight, edit, text):
    with pytest.raises(cobs.CobsError, match=text):
        _call_append(eight, **edit)


def _with(c8, **over):
    return c8._replace(**over)


@pytest.mark.parametrize("edit,text", [
    (lambda c: tuple(c), "tokens.Cache8"), (lambda c: _with(c, k=c.k.float()), "8-bit k must be"), (lambda c: _with(c, v=c.v[..., :64]), "8-bit v must be 4-D"),
    (lambda c: _with(c, k=c.k[:, :, :64], v=c.v[:, :, :64]), "smaller than"), (lambda c: _with(c, v=c.v.transpose(0, 1).contiguous().transpose(0, 1)), "share shape and strides"),
    (lambda c: _with(c, k_scale=c.k_scale.double()), "k_scale must be"), (lambda c: _with(c, v_scale=c.v_scale[..., :1]), "v_scale"),
    (lambda c: _with(c, v_scale=torch.zeros((2, 4, 1))), "v_scale must have shape"),
])
def test_binding_names_the_wrong_part_of_an_8_bit_cache(edit, text):
    t = _tensors()
    bad = edit(t["c8"])
    with pytest.raises(cobs.CobsError, match=text):
        _call_append(True, c8=bad)
    q = torch.zeros((2, 3, 8, 128))
    with pytest.raises(cobs.CobsError, match=text):
        tokens.cobs_decode8(t["cfg"], q, bad, t["lens"], None, None, torch.zeros_like(q), torch.zeros(256, dtype=torch.uint8))
    with pytest.raises(cobs.CobsError, match=text):
        tokens.cobs_unpack8(t["cfg"], bad, t["lens"], t["k"], t["v"])


def test_binding_checks_pages_of_an_8_bit_cache():
    t = _tensors()
    pool = tokens.new_cache8(t["cfg"], "cpu", num_pages=5)
    assert pool.k.shape == (5, 2, 64, 128) and pool.k_scale.shape == (5, 2)
    table = torch.zeros((2, 2), dtype=torch.int32)
    for over, text in ((dict(c8=t["c8"]), "paged 8-bit k"), (dict(pages=6), "num_pages"), (dict(pages=0), "num_pages"), (dict(table=table.long()), "block_table must be"),
                       (dict(c8=pool._replace(k_scale=torch.zeros((4, 2)))), "k_scale holds"), (dict(), "on a GPU")):
        with pytest.raises(cobs.CobsError, match=text):
            _call_append(True, **{**dict(c8=pool, table=table, pages=5), **over})


@pytest.mark.parametrize("edit,text", [
    (dict(q=torch.zeros((2, 65, 8, 128))), "1 to 64"), (dict(out=torch.zeros((2, 3, 8, 128), dtype=torch.bfloat16)), "out must be"), (dict(lse=torch.zeros(3)), "lse holds"),
    (dict(drafts=torch.zeros(2, dtype=torch.int32)), "go together"), (dict(sel=torch.zeros(3, dtype=torch.int32)), "sel holds"), (dict(ws=None), "ws is required"),
    (dict(), "on a GPU"),
])
def test_binding_names_the_wrong_argument_of_an_attention(edit, text):
    t = _tensors()
    a = dict(q=torch.zeros((2, 3, 8, 128)), out=torch.zeros((2, 3, 8, 128)), lse=None, drafts=None, sel=None, ws=torch.zeros(256, dtype=torch.uint8))
    a.update(edit)
    with pytest.raises(cobs.CobsError, match=text):
        tokens.cobs_decode8(t["cfg"], a["q"], t["c8"], t["lens"], a["drafts"], None, a["out"], a["ws"], sel=a["sel"], lse=a["lse"])


def test_binding_names_the_wrong_argument_of_a_rotation_and_of_unpacking():
    t = _tensors()
    for over, text in ((dict(x=None), "x must"), (dict(out=torch.zeros((2, 3, 8, 64))), "out must have shape"), (dict(at=None), "positions is required"),
                       (dict(at=t["at"][:1]), "positions holds"), (dict(rope=None), "tokens.Rope"), (dict(), "on a GPU")):
        a = {**dict(x=t["q"], out=t["q_out"], at=t["at"], rope=t["rope"]), **over}
        with pytest.raises(cobs.CobsError, match=text):
            tokens.cobs_rotate(a["x"], a["rope"], a["at"], a["out"])
    for over, text in ((dict(last=1, first_block=1), "last stands"), (dict(last=-1), "not be negative"), (dict(first_block=-1), "not be negative"), (dict(), "on a GPU")):
        with pytest.raises(cobs.CobsError, match=text):
            tokens.cobs_unpack8(t["cfg"], t["c8"], t["lens"], t["k"], t["v"], **over)
    with pytest.raises(cobs.CobsError, match="k must be"):
        tokens.cobs_unpack8(t["cfg"], t["c8"], t["lens"], t["k"].float(), t["v"].float())
