"""Rotary positions on several axes and the 8-bit cache in float64, from their definitions, and an independent
reader of the cache's byte layout.  Plain numpy; nothing here is shared with the library."""
from __future__ import annotations

import numpy as np

D, G = 128, 32
LEVEL = {0: 127.0, 1: 448.0}
LEAST, MOST = 2.0 ** -40, 2.0 ** 40


def rotary(x, pos, sections, theta=10000.0, rot_dim=None, adjacent=False, inverse=False, freq=None):
    """x [B, H, n, d], pos [axes, B, n] -> y1 = x1 cos a - x2 sin a, y2 = x2 cos a + x1 sin a for every pair.
    Angles in extended precision: a position of 2^31 leaves 33 bits of the turn."""
    rot_dim = x.shape[-1] if rot_dim is None else rot_dim
    pairs = rot_dim // 2
    y = np.array(x, dtype=np.float64)
    axis = np.repeat(np.arange(len(sections)), sections)
    for i in range(pairs):
        f = np.longdouble(theta) ** (-np.longdouble(i) / pairs) if freq is None else np.longdouble(freq[i])
        a = pos[axis[i]].astype(np.longdouble) * f
        c, s = np.cos(a).astype(np.float64)[:, None], np.sin(a).astype(np.float64)[:, None]
        if inverse:
            s = -s
        u, v = (2 * i, 2 * i + 1) if adjacent else (i, i + pairs)
        y[..., u] = x[..., u] * c - x[..., v] * s
        y[..., v] = x[..., v] * c + x[..., u] * s
    return y


def e4m3_values():
    """The 256 bytes' numbers (NaN at 0x7f and 0xff)."""
    b = np.arange(256)
    e, m = (b >> 3) & 15, (b & 7).astype(np.float64)
    v = np.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * 2.0 ** (e - 7.0))
    v = np.where((b & 127) == 127, np.nan, v)
    return np.where(b > 127, -v, v)


def value_of(byte, code):
    return byte.astype(np.int8).astype(np.float64) if code == 0 else e4m3_values()[byte]


def byte_of(r, code):
    """The code nearest to r (in the code's units), ties to the even code.  e4m3 has two zeros: a number below zero that
    rounds to it becomes 0x80, a zero of either sign 0."""
    if code == 0:
        return np.clip(np.rint(r), -127, 127).astype(np.int8).view(np.uint8)
    pos = e4m3_values()[:127]                                  # 0 .. 448, ascending
    a = np.minimum(np.abs(r), 448.0)
    i = np.clip(np.searchsorted(pos, a), 1, 126)
    lo, hi = pos[i - 1], pos[i]
    up = (a - lo > hi - a) | ((a - lo == hi - a) & (i % 2 == 0))
    return (np.where(up, i, i - 1) | np.where(r < 0, 128, 0)).astype(np.uint8)


def write(x, start, count, bytes_, mags, code):
    """Append x [H, n, 128] (float64) as tokens start .. start + count - 1 to one sequence's codes [H, C, 128] and
    magnitudes [H, C/32], in place."""
    cap = bytes_.shape[1]
    end = min(start + count, cap)
    if start < 0:
        return
    for t0 in range(start // G * G, end, G):
        lo, hi = max(start, t0), min(end, t0 + G)
        for h in range(x.shape[0]):
            new = x[h, lo - start:hi - start]
            old = mags[h, t0 // G] if t0 < start else 0.0
            a = min(max(np.abs(new).max(), old, LEAST), MOST)
            if t0 < start and a > old:
                live = bytes_[h, t0:start]
                bytes_[h, t0:start] = byte_of(value_of(live, code) * old / a, code)
            bytes_[h, lo:hi] = byte_of(new * LEVEL[code] / a, code)
            mags[h, t0 // G] = a


def values(bytes_, mags, code):
    """[.., C, 128] values of codes and magnitudes."""
    return value_of(bytes_, code) * (np.repeat(mags.astype(np.float64), G, axis=-1) / LEVEL[code])[..., None]


def attention(q, K, V, scale, limit):
    """One head's queries q [n, 128] over K, V [T, 128]; query i sees the first limit[i] tokens."""
    out = np.zeros(q.shape)
    for i in range(q.shape[0]):
        t = int(limit[i])
        if t > 0:
            x = scale * (K[:t] @ q[i])
            p = np.exp(x - x.max())
            out[i] = (p / p.sum()) @ V[:t]
    return out


def unpack(buf, L, B, H, cap):
    """(K codes, V codes [L, B, H, C, 128] uint8, K, V magnitudes [L, B, H, C/32]) of a cache buffer."""
    up = lambda n: -(-n // 256) * 256  # noqa: E731
    nb = L * B * H * cap // G
    codes, m = up(nb * G * D), up(nb * 4)
    kc = buf[:nb * G * D].reshape(L, B, H, cap, D)
    rec = buf[codes:codes + nb * G * D].reshape(nb, 4, 4, 16, 2, 8)
    vc = np.zeros((nb, G, D), np.uint8)
    for mp in range(4):
        for kb in range(4):
            for mh in range(2):
                for j in range(8):
                    t = 4 * kb + j if j < 4 else 16 + 4 * kb + j - 4
                    vc[:, t, 32 * mp + 16 * mh:32 * mp + 16 * mh + 16] = rec[:, mp, kb, :, mh, j]
    mag = [buf[2 * codes + i * m:2 * codes + i * m + 4 * nb].view(np.float32).reshape(L, B, H, cap // G) for i in (0, 1)]
    return kc, vc.reshape(L, B, H, cap, D), mag[0], mag[1]
