"""Oracle of the 8-bit block format and the layer that uses it -- TEST INFRASTRUCTURE ONLY.

A block's scale is 2^e with e the least integer >= -126 for which every finite |x| of the block is <= 448 * 2^e; its
codes are e4m3(x / 2^e), to nearest even, with infinities and NaN as the NaN code.  Rounding works on a table of the
256 codes' values, not on bit patterns.
"""
from __future__ import annotations

import numpy as np

from .layer import backward, swiglu

BLOCK = 128


def _code_values():
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
        v[c] = -x if c & 128 else x
    v[0x7F] = v[0xFF] = np.nan
    return v


VALUES = _code_values()
_POS = VALUES[:0x7F]  # 0 .. 448, ascending


def encode(x):
    """Codes of x / 2^e (|x| <= 448 where finite), nearest, ties to the even code."""
    a = np.abs(np.nan_to_num(x, nan=0.0, posinf=0.0, neginf=0.0))
    hi = np.clip(np.searchsorted(_POS, a), 0, 0x7E)
    lo = np.clip(hi - 1, 0, 0x7E)
    up, down = _POS[hi] - a, a - _POS[lo]
    c = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    c = np.where(np.isfinite(x), c, 0x7F)
    return (c | (np.signbit(x) << 7)).astype(np.uint8)


def exponents(x, block):
    """e of every block[0] x block[1] block of x [rows, cols]."""
    r, c = x.shape
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    out = np.empty((-(-r // block[0]), -(-c // block[1])), np.int64)
    for i in range(out.shape[0]):
        rows = a[i * block[0]:(i + 1) * block[0]]
        for j in range(out.shape[1]):
            m = rows[:, j * block[1]:(j + 1) * block[1]].max()
            e = -126 if m == 0 else max(-126, int(np.floor(np.log2(m))) - 10)
            while m > 448 * 2.0 ** e:
                e += 1
            out[i, j] = e
    return out


def quantize(x, block=(1, BLOCK)):
    """(codes, e per block, values) of x [rows, cols] in fp64."""
    x = np.asarray(x, np.float64)
    e = exponents(x, block)
    s = np.ldexp(1.0, np.repeat(np.repeat(e, block[0], 0)[:x.shape[0]], block[1], 1)[:, :x.shape[1]])
    q = encode(x / s)
    return q, e, VALUES[q] * s


def through(x, block=(1, BLOCK)):
    return quantize(x, block)[2]


def through_halves(x, block=(1, BLOCK)):
    n = x.shape[1] // 2
    return np.concatenate([through(x[:, :n], block), through(x[:, n:], block)], 1)


def through_experts(W1, W2):
    sq = (BLOCK, BLOCK)
    return np.stack([through_halves(w, sq) for w in W1]), np.stack([through(w, sq) for w in W2])


def forward_quant(X, W1, W2, R, b1=None, b2=None):
    """The forward with 8-bit expert products, in fp64: O, H, A (both before their rounding), its values A8, and Y.
    W1, W2: the 16-bit weights."""
    X8 = through(X)
    W1q, W2q = through_experts(np.asarray(W1, np.float64), np.asarray(W2, np.float64))
    T, d = X8.shape
    n = W2q.shape[1]
    H, A = np.zeros((R.P, 2 * n)), np.zeros((R.P, n))
    A8, Y, O = np.zeros((R.P, n)), np.zeros((R.P, d)), np.zeros((T, d))
    for e in range(W1q.shape[0]):
        a, b = int(R.offsets[e]), int(R.offsets[e + 1])
        if a == b:
            continue
        H[a:b] = X8[R.row_token[a:b]] @ W1q[e] + (0 if b1 is None else np.asarray(b1[e], np.float64))
        A[a:b] = swiglu(H[a:b])
        A8[a:b] = through(A[a:b])
        Y[a:b] = A8[a:b] @ W2q[e] + (0 if b2 is None else np.asarray(b2[e], np.float64))
    np.add.at(O, R.row_token, R.row_w.astype(np.float64)[:, None] * Y)
    return {"O": O, "H": H, "A": A, "A8": A8, "Y": Y, "W2q": W2q, "X8": X8}


def backward_ckpt(dO, X, H, W1, W2, Wr, R, b2=None):
    """The backward from kept values X and H, in fp64."""
    return backward(dO, X, H, W1, W2, Wr, R, dtype=np.float64, b2=b2)
