"""The token operators in plain fp64 NumPy, from their definitions: rotary positions, the nearest 8-bit
float, and the append of tokens to one block of an 8-bit cache."""

import numpy as np

LEAST_SCALE = 2.0 ** -100


def rotate(x, positions, inv_freq, interleaved=False, scale=1.0):
    """x [tokens, heads, d] with the first 2 len(inv_freq) elements of each head turned: pair p of a token at position t
    by the angle t f_p, times `scale`."""
    x = np.asarray(x, dtype=np.float64)
    y, half = x.copy(), len(inv_freq)
    lo = 2 * np.arange(half) if interleaved else np.arange(half)
    hi = lo + 1 if interleaved else lo + half
    a = np.asarray(positions, dtype=np.float64)[:, None] * np.asarray(inv_freq, dtype=np.float64)[None]
    cos, sin = np.cos(a)[:, None], np.sin(a)[:, None]
    y[..., lo] = scale * (x[..., lo] * cos - x[..., hi] * sin)
    y[..., hi] = scale * (x[..., hi] * cos + x[..., lo] * sin)
    return y


def e4m3_values():
    """The numbers that the 256 codes stand for: 4 exponent bits of bias 7, 3 mantissa bits, all ones NaN."""
    code = np.arange(256)
    e, m = (code >> 3) & 15, code & 7
    mag = np.where(e == 0, m / 8.0 * 2.0 ** -6, (1.0 + m / 8.0) * 2.0 ** (e - 7.0))
    mag[(code & 127) == 127] = np.nan
    return np.where(code >= 128, -mag, mag)


def e4m3_codes(x):
    """Codes of the nearest numbers, ties to the even mantissa; NaN for what is not finite; |x| <= 448."""
    x = np.asarray(x, dtype=np.float64)
    mags = e4m3_values()[:127]                           # ascending
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    at = np.clip(np.searchsorted(mags, a), 1, 126)       # mags[at - 1] <= a <= mags[at] (but at the ends)
    low, high = a - mags[at - 1], mags[at] - a
    code = np.where((high < low) | ((high == low) & (at % 2 == 0)), at, at - 1)
    code = np.where(a == 0.0, 0, code)
    code = np.where(np.signbit(x), code + 128, code)
    return np.where(np.isfinite(x), code, 127).astype(np.uint8)


def scale_for(top):
    """The smallest power of two s, 2^-100 at least, with top / s <= 448."""
    if not top > 0.0:
        return LEAST_SCALE
    f, e = np.frexp(top)                                 # top = f 2^e, f in [1/2, 1); 448 = 0.875 * 2^9
    return max(float(np.ldexp(1.0, int(e) - 9 + int(f > 0.875))), LEAST_SCALE)


def append_block(codes, scale, earlier, new):
    """One block of one KV head: codes [L, d], its scale, the tokens that it holds and the new ones [n, d] behind them.
    The codes and the scale after."""
    codes, n = codes.copy(), len(new)
    finite = np.abs(new[np.isfinite(new)])
    need = scale_for(finite.max() if finite.size else 0.0)
    now = scale if earlier > 0 and scale >= need else need
    if earlier > 0 and now != scale:
        codes[:earlier] = e4m3_codes(e4m3_values()[codes[:earlier]] * (scale / now))
    codes[earlier:earlier + n] = e4m3_codes(new / now)
    return codes, now
