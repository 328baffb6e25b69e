"""Plain 64-bit CPU definitions of the operators around a key/value cache: rotary positions, the quantised paged cache,
attention of the newest tokens over it (test infrastructure only)."""
import numpy as np


def rotary(x, positions, freqs, amplitude=1.0, layout="half", backward=False):
    """x [B, H, L, D], positions [B, L] or [L]; pair i turned by positions * freqs[i], stretched by amplitude."""
    x = np.asarray(x, np.float64)
    n = len(freqs)
    # angles in 80-bit numbers: at position 2^31 a double's rounding of 6 radians a position is off by 2^-53 * 1.3e10 = 1.4e-6
    a = np.broadcast_to(np.asarray(positions, np.longdouble), (x.shape[0], x.shape[2]))[:, None, :, None] * np.asarray(freqs, np.longdouble)
    c, s = (amplitude * t(a).astype(np.float64) for t in (np.cos, np.sin))
    s = -s if backward else s
    i1 = np.arange(n) if layout == "half" else 2 * np.arange(n)
    i2 = i1 + (n if layout == "half" else 1)
    y = x.copy()
    y[..., i1] = x[..., i1] * c - x[..., i2] * s
    y[..., i2] = x[..., i2] * c + x[..., i1] * s
    return y


E4M3 = np.array([(-1.0 if i & 128 else 1.0) * (np.ldexp(i & 7, -9) if not i & 120 else np.ldexp(8 + (i & 7), ((i & 120) >> 3) - 10))
                 if i & 127 != 127 else np.nan for i in range(256)])


def quantise(x):
    """Rows [..., D] -> (e4m3 bit patterns, exponent bytes): the smallest k >= -126 with the largest finite magnitude <= 448 * 2^k."""
    x = np.asarray(x, np.float64)
    top = np.where(np.isfinite(x), np.abs(x), 0.0).max(axis=-1)
    k = np.full(top.shape, -126)
    while (top > 448.0 * np.ldexp(1.0, k)).any():
        k = np.where(top > 448.0 * np.ldexp(1.0, k), k + 1, k)
    y = x * np.ldexp(1.0, -k)[..., None]
    pos = E4M3[:127]  # ascending
    mag = np.minimum(np.abs(np.where(np.isfinite(y), y, 0.0)), 448.0)
    hi = np.clip(np.searchsorted(pos, mag), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = pos[hi] - mag, mag - pos[lo]
    q = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    q = np.where(np.isfinite(y), q, 127) | np.where(np.signbit(y), 128, 0)
    return q.astype(np.uint8), (k + 127).astype(np.uint8)


def dequantise(q, e):
    return E4M3[q] * np.ldexp(1.0, e.astype(np.int64) - 127)[..., None]


def attend(q, keys, values, scale):
    """One sequence: q [H_q, n, D], keys and values [H_kv, len, D]; the newest n of the len tokens are q's own, and token t of them
    sees the first len - n + 1 + t keys.  Returns (O, ln sum exp); a token without keys has O = 0 and -inf."""
    q, keys, values = (np.asarray(t, np.float64) for t in (q, keys, values))
    H_q, n, _ = q.shape
    g, length = H_q // keys.shape[0], keys.shape[1]
    O, S = np.zeros((H_q, n, values.shape[2])), np.full((H_q, n), -np.inf)
    for h in range(H_q):
        for t in range(n):
            end = length - n + 1 + t
            if end <= 0:
                continue
            x = scale * keys[h // g, :end] @ q[h, t]
            m = x.max()
            w = np.exp(x - m)
            O[h, t], S[h, t] = w @ values[h // g, :end] / w.sum(), m + np.log(w.sum())
    return O, S
