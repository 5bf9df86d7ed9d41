"""Microscaled 4-bit floating point in float64 NumPy, from the format's
definition: blocks of 32 along a row, E2M1 elements, an E8M0 scale."""
from __future__ import annotations

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def scale_bytes(v):
    """The scale byte of every block of v [rows, cols]."""
    b = np.abs(np.asarray(v, np.float64)).reshape(v.shape[0], -1, 32)
    bad = ~np.isfinite(b).all(-1)
    m = np.where(bad, 0.0, np.where(np.isfinite(b), b, 0.0).max(-1))
    _, e = np.frexp(m)                       # m = f 2^e, f in [0.5, 1)
    s = np.where(m > 0, np.maximum(e.astype(np.int64) - 3 + 127, 0), 0)
    return np.where(bad, 255, s).astype(np.uint8)


def quantize(v):
    """(codes [rows, cols / 2], scales [rows, cols / 32])."""
    v = np.asarray(v, np.float64)
    s = scale_bytes(v)
    b = v.reshape(v.shape[0], -1, 32)
    with np.errstate(invalid="ignore"):
        t = np.ldexp(np.abs(b), (127 - s.astype(np.int64))[..., None])
    mid = (E2M1[1:] + E2M1[:-1]) / 2
    t = np.where(np.isfinite(t), t, 0.0)
    below = np.searchsorted(mid, t, side="left")      # borders below t
    upto = np.searchsorted(mid, t, side="right")      # ... or at it
    c = np.where(below % 2 == 0, below, upto)         # on a border: the even code
    c = c | (np.signbit(b).astype(np.int64) << 3)
    c = np.where((s == 255)[..., None], 0, c).reshape(v.shape).astype(np.uint8)
    return c[:, 0::2] | (c[:, 1::2] << 4), s


def dequantize(codes, scales):
    """The values [rows, cols] in float64."""
    c = np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[0], -1)
    v = E2M1[c & 7] * np.where(c >= 8, -1.0, 1.0)
    v = np.ldexp(v.reshape(codes.shape[0], -1, 32), (scales.astype(np.int64) - 127)[..., None])
    return np.where((scales == 255)[..., None], np.nan, v).reshape(codes.shape[0], -1)


def pack(codes, scales, row_tiles):
    """The BASE_W_MXFP4 bytes of one expert's matrix: codes [rows, K / 2], scales
    [rows, K / 32], row_tiles: the first row of every 16-row tile, in order."""
    K = 2 * codes.shape[1]
    steps = -(-K // 128)
    out = []
    for r0 in row_tiles:
        for c in range(0, steps, 4):
            here = range(c, min(c + 4, steps))
            sc = np.zeros((64, 4), np.uint8)
            st = np.zeros((len(here), 64, 16), np.uint8)
            for j, s in enumerate(here):
                for lane in range(64):
                    row, k = r0 + lane % 16, 128 * s + 32 * (lane // 16)
                    if k < K:
                        sc[lane, j] = scales[row, k // 32]
                        st[j, lane] = codes[row, k // 2:k // 2 + 16]
            out += [sc.ravel(), st.ravel()]
    return np.concatenate(out)


def w13_tiles(I):
    return [r + h * I for r in range(0, I, 16) for h in (0, 1)]


def w2_tiles(d):
    return list(range(0, d, 16))
