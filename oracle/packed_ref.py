"""Plain statements, in 64 bits, of head rotation and of the 4-bit form of cached rows (test infrastructure).

Written from the definitions in include/stand.h; numpy only.
"""
import numpy as np

SCALES = np.array([f / 8 * 2.0**-14 for f in range(8)] + [(1 + f / 8) * 2.0 ** (e - 15) for e in range(1, 31) for f in range(8)])


def pack(x):
    """Rows [.., D] -> codes [.., D / 2] and scales [.., D / 16], uint8."""
    g = x.astype(np.float64).reshape(x.shape[:-1] + (x.shape[-1] // 16, 16))
    top = np.abs(g).max(-1)
    fine = np.isfinite(top)
    byte = np.minimum(np.searchsorted(7 * SCALES, np.where(fine, top, 0.0)), len(SCALES) - 1)
    s = SCALES[byte][..., None]
    with np.errstate(all="ignore"):
        quotient = (g.astype(np.float32) / s.astype(np.float32)).astype(np.float64)
    k = np.where((s > 0) & fine[..., None], np.clip(np.rint(np.where(np.isfinite(quotient), quotient, 0.0)), -7, 7), 0).astype(np.int64) + 8
    k = k.reshape(x.shape)
    out = np.zeros(x.shape[:-1] + (x.shape[-1] // 2,), np.uint8)
    for d in range(x.shape[-1]):
        e = d % 8  # of a word of four bytes: bits 4 (e / 2) of its low or high half
        bit = 4 * (e // 2) + 16 * (e % 2)
        out[..., d // 8 * 4 + bit // 8] |= (k[..., d] << (bit % 8)).astype(np.uint8)
    return out, np.where(fine, byte, 0xFF).astype(np.uint8)


def values(codes, scales):
    """What codes [.., D / 2] and scales [.., D / 16] stand for, [.., D]."""
    D = codes.shape[-1] * 2
    out = np.zeros(codes.shape[:-1] + (D,))
    for d in range(D):
        e = d % 8
        bit = 4 * (e // 2) + 16 * (e % 2)
        k = (codes[..., d // 8 * 4 + bit // 8] >> (bit % 8) & 15).astype(np.float64) - 8
        byte = scales[..., d // 16]
        out[..., d] = np.where(byte >= 0xF8, np.nan, k * SCALES[np.minimum(byte, 0xF7)])
    return out


def blocks(rows):
    """Rows [.., page, D] -> blocks [.., page * D * 9 / 16]: all codes, then all scales."""
    codes, scales = pack(rows)
    flat = lambda a: a.reshape(a.shape[:-2] + (a.shape[-2] * a.shape[-1],))  # noqa: E731
    return np.concatenate([flat(codes), flat(scales)], -1)


def block_values(block, page, D):
    cut = page * D // 2
    return values(block[..., :cut].reshape(block.shape[:-1] + (page, D // 2)), block[..., cut:].reshape(block.shape[:-1] + (page, D // 16)))


def rotate(x, pos, freq, interleaved=False, weight=None, eps=None):
    """Rows x [.., D] at positions pos [..] -> (result, size): size is the sum of the magnitudes that an element is made of.
    weight: None with eps None: no norm."""
    y = x.astype(np.float64)
    if eps is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps)
        if weight is not None:
            y = y * weight.astype(np.float64)
    out, size = y.copy(), np.abs(y)
    for i in range(0 if freq is None else len(freq)):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + len(freq))
        t = np.asarray(pos, np.longdouble) * np.longdouble(freq[i])  # 31 and 24 bits: exact in 64
        c, s = np.cos(t).astype(np.float64), np.sin(t).astype(np.float64)
        out[..., a] = y[..., a] * c - y[..., b] * s
        out[..., b] = y[..., a] * s + y[..., b] * c
        size[..., a] = size[..., b] = np.abs(y[..., a]) + np.abs(y[..., b])
    return out, size
