"""Plain numpy models of 4-bit rows (include/lg_fp4.h), written from their definition and sharing no code with the
kernels: groups of 32 values with a unit 2^(x - 127), codes of a sign and 0, 0.5, 1, 1.5, 2, 3, 4, 6 units."""
from __future__ import annotations

import numpy as np

GROUP = 32
STEPS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def exponent(m):
    """The exponent bytes of groups whose largest magnitudes are m (float64 array): smallest unit with m <= 6 units."""
    e = np.full(m.shape, -125)
    for k in range(-124, 126):
        e = np.where(m > 6 * 2.0 ** (k - 1), k, e)
    return np.where(np.isfinite(m), e + 127, 255)


def nearest(y):
    """Codes of the magnitudes y, in units: the nearest step, ties to the even code."""
    y = np.where(np.isfinite(y), y, 0)
    low = np.clip(np.searchsorted(STEPS, y, side="right") - 1, 0, 7)
    high = np.minimum(low + 1, 7)
    up, down = STEPS[high] - y, y - STEPS[low]
    take = (up < down) | ((up == down) & (high % 2 == 0))
    return np.where(take, high, low)


def encode(x):
    """x [..., D] -> codes uint8 [..., D] and exponents uint8 [..., D / 32]."""
    g = np.asarray(x, np.float64).reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    with np.errstate(invalid="ignore"):
        odd = ~np.isfinite(g).all(-1)
        exps = np.where(odd, 255, exponent(np.abs(np.where(odd[..., None], 0, g)).max(-1)))
        codes = nearest(np.abs(g) / 2.0 ** (exps[..., None] - 127.0)) + 8 * np.signbit(g)
    codes = np.where(odd[..., None], 0, codes)
    return codes.reshape(x.shape).astype(np.uint8), exps.astype(np.uint8)


def values(codes, exps):
    """float64 values of codes [..., D] with exponents [..., D / 32]."""
    unit = np.where(exps > 252, np.nan, 2.0 ** (exps.astype(np.float64) - 127))
    v = np.where(codes >= 8, -1.0, 1.0) * STEPS[codes & 7]
    return (v.reshape(*exps.shape, GROUP) * unit[..., None]).reshape(codes.shape)


def pack(codes, exps):
    """codes, exps [..., page_size, D or D / 32] as blocks of bytes [..., page_size (D / 2 + D / 32)]."""
    rows = codes[..., 0::2] | codes[..., 1::2] << 4
    return np.concatenate([x.reshape(*x.shape[:-2], -1) for x in (rows, exps)], -1)


def unpack(blocks, page_size, D):
    """The codes and exponents of blocks of bytes."""
    rows = blocks[..., :page_size * D // 2].reshape(*blocks.shape[:-1], page_size, D // 2)
    exps = blocks[..., page_size * D // 2:].reshape(*blocks.shape[:-1], page_size, D // GROUP)
    codes = np.empty(rows.shape[:-1] + (D,), np.uint8)
    codes[..., 0::2], codes[..., 1::2] = rows & 15, rows >> 4
    return codes, exps


def pages(x):
    """Pages of values x [n][heads][page_size][D] as bytes."""
    return pack(*encode(x))


def rope_axes(x, coord, axis, inv_freq, rot, interleaved, scale):
    """x [T][H][D] rotated with pair j at coord[axis[j]], in float64, and the sums |x| + |y| of its pairs."""
    y = x.astype(np.float64).copy()
    size = np.abs(y)
    for j in range(rot // 2):
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)
        ang = coord[axis[j]].astype(np.longdouble) * np.longdouble(np.float32(inv_freq[j]))
        c, s = np.cos(ang).astype(np.float64)[:, None], np.sin(ang).astype(np.float64)[:, None]
        u, w = x[..., a].astype(np.float64), x[..., b].astype(np.float64)
        y[..., a], y[..., b] = scale * (u * c - w * s), scale * (w * c + u * s)
        size[..., a] = size[..., b] = scale * (np.abs(u) + np.abs(w))
    return y, size
