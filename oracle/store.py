"""The two block formats of the 4-bit weights and the 8-bit activation checkpoints, in plain numpy.

TEST INFRASTRUCTURE ONLY.  Written from the formats' definition: 32 neighbouring values of a row share a scale 2^e; the codes
are the numbers of a small floating-point format (4 bits: 1 sign, 2 exponent, 1 mantissa; 8 bits: 1, 4, 3).  The nearest code
is found by comparing with every code's value, the scale by trying every exponent upwards.
"""
from __future__ import annotations

import numpy as np

BLOCK = 32
VALUES4 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=np.float64)
# exponent field 0: multiples of 2^-9; otherwise (1 + mantissa / 8) 2^(field - 7); the last code is NaN
VALUES8 = np.array([(c & 7) * 2.0 ** -9 if c < 8 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) for c in range(127)])
BOUNDS4 = {"f16": (-23, 13), "bf16": (-125, 125), "f32": (-125, 125)}
BOUNDS8 = {"f16": (-15, 8), "bf16": (-117, 120), "f32": (-117, 120)}
MOST8 = {"f16": 61440.0, "bf16": 1.875 * 2.0 ** 127, "f32": 1.875 * 2.0 ** 127}


def nearest(v, values):
    """Index of the value nearest to |v|, ties to the even index; `values` with the number that would follow its last one
    behind it, so that what rounds past the last code shows."""
    nxt = 2 * values[-1] - values[-2] if values[-1] != 6 else 8.0
    wide = np.append(values, nxt)
    mid = (wide[:-1] + wide[1:]) / 2
    a = np.abs(np.asarray(v, dtype=np.float64))
    k = np.searchsorted(mid, a, side="left")  # the first midpoint not below a
    tie = (k < len(mid)) & (a == mid[np.minimum(k, len(mid) - 1)])
    return np.where(tie & (k % 2 == 1), k + 1, k)


def scale_exponent(most, values, bounds):
    lo, hi = bounds
    for e in range(lo, hi + 1):
        if most <= 2.0 ** (e + 20) and nearest(most / 2.0 ** e, values) < len(values):
            return e
    return hi


def _blocks(x):
    rows, cols = x.shape
    wide = np.zeros((rows, -(-cols // BLOCK) * BLOCK), dtype=np.float64)
    wide[:, :cols] = x
    return wide.reshape(rows, -1, BLOCK)


def _pack(x, values, bounds, sign_bit):
    b = _blocks(np.asarray(x, dtype=np.float64))
    finite = np.isfinite(b)
    codes = np.zeros(b.shape, dtype=np.uint8)
    exps = np.zeros(b.shape[:2], dtype=np.int64)
    for i in range(b.shape[0]):
        for j in range(b.shape[1]):
            v = np.where(finite[i, j], b[i, j], 0.0)
            e = exps[i, j] = scale_exponent(np.abs(v).max(), values, bounds)
            k = np.minimum(nearest(v / 2.0 ** e, values), len(values) - 1)
            codes[i, j] = k + sign_bit * np.signbit(v)
    return codes, exps, finite


def pack4(W, M, dtype):
    """W float64 [m, n], mask M (or None) -> codes uint8 [m, blocks * 32] (one a byte), scale bytes uint8 [m, blocks]."""
    W = np.asarray(W, dtype=np.float64)
    codes, exps, finite = _pack(W if M is None else np.where(M != 0, W, 0.0), VALUES4, BOUNDS4[dtype], 8)
    bad = ~finite.all(axis=2)
    codes[bad] = 0
    return codes.reshape(W.shape[0], -1), np.where(bad, 255, exps + 127).astype(np.uint8)


def unpack4(codes, scales, n):
    with np.errstate(invalid="ignore"):
        scale = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
        v = np.where(codes & 8, -1.0, 1.0) * VALUES4[codes & 7]
        return (v.reshape(codes.shape[0], -1, BLOCK) * scale[:, :, None]).reshape(codes.shape[0], -1)[:, :n]


def pack8(X, dtype):
    """X float64 [n, N] -> codes uint8 [n, blocks * 32], scale bytes uint8 [n, blocks]."""
    X = np.asarray(X, dtype=np.float64)
    cut = np.where(np.isfinite(X), np.clip(X, -MOST8[dtype], MOST8[dtype]), X)
    codes, exps, finite = _pack(cut, VALUES8, BOUNDS8[dtype], 128)
    codes = np.where(finite, codes, 0x7F).astype(np.uint8)
    return codes.reshape(X.shape[0], -1), (exps + 127).astype(np.uint8)


def unpack8(codes, scales, N):
    table = np.append(VALUES8, np.nan)
    v = np.where(codes & 128, -1.0, 1.0) * table[codes & 127]
    scale = 2.0 ** (scales.astype(np.float64) - 127)
    return (v.reshape(codes.shape[0], -1, BLOCK) * scale[:, :, None]).reshape(codes.shape[0], -1)[:, :N]


def nibbles(packed):
    """Bytes of two codes -> one code a byte."""
    return np.stack((packed & 15, packed >> 4), axis=2).reshape(packed.shape[0], -1)


def packed_nibbles(codes):
    return (codes[:, ::2] | (codes[:, 1::2] << 4)).astype(np.uint8)
