"""The 8-bit paged cache's operators in float64 NumPy, one sequence, block and
head at a time, from their definitions (include/m2r2_kv8.h).  Shares nothing
with the HIP path."""
from __future__ import annotations

import math

import numpy as np

# the 256 e4m3 codes' values: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7f and 0xff are NaN
CODE = np.array([(-1.0 if c & 0x80 else 1.0) *
                 (math.nan if c & 0x7f == 0x7f else
                  (c & 7) * 2.0 ** -9 if not c & 0x78 else (8 + (c & 7)) * 2.0 ** ((c >> 3 & 15) - 10))
                 for c in range(256)])
_POS = CODE[:0x7f]
_BETWEEN = (_POS[1:] + _POS[:-1]) / 2


def encode(x: np.ndarray) -> np.ndarray:
    """Codes nearest to finite |x| <= 448, ties to the even code; NaN and infinities: NaN."""
    mag = np.abs(np.where(np.isfinite(x), x, 0.0))
    lo = np.searchsorted(_BETWEEN, mag, side="left")     # a tie goes to the lower code ...
    tie = (lo < len(_BETWEEN)) & (mag == _BETWEEN[np.minimum(lo, len(_BETWEEN) - 1)])
    code = np.where(tie & (lo % 2 == 1), lo + 1, lo)     # ... unless that is odd
    code = np.where(np.signbit(x), code | 0x80, code)
    return np.where(np.isfinite(x), code, 0x7f).astype(np.uint8)


def exponent(amax: float) -> int:
    """The least e in [-120, 112] with 448 * 2^e >= amax."""
    e = -120
    while e < 112 and 448.0 * 2.0 ** e < amax:
        e += 1
    return e


class Cache:
    """One layer: codes [block][head][slot][dim] and exponents [block][head], keys (0) and values (1)."""

    def __init__(self, codes, scales):
        self.codes = [np.array(c, dtype=np.uint8) for c in codes]
        self.exps = [np.rint(np.log2(np.asarray(s, np.float64))).astype(int) for s in scales]

    def append(self, which: int, blocks, p0: int, y: np.ndarray) -> None:
        """Rows y [n][head][dim] at positions p0.. of the sequence with that block list."""
        codes, exps = self.codes[which], self.exps[which]
        bs = codes.shape[2]
        top = 448.0 * 2.0 ** 112
        for lb in range(p0 // bs, (p0 + len(y) - 1) // bs + 1):
            b0, b1 = max(p0, lb * bs), min(p0 + len(y), (lb + 1) * bs)
            blk, first = blocks[lb], b0 - lb * bs
            for h in range(codes.shape[1]):
                new = y[b0 - p0:b1 - p0, h].astype(np.float64)
                fin = new[np.isfinite(new)]
                e = exponent(float(np.max(np.abs(fin))) if fin.size else 0.0)
                if first:
                    old = int(exps[blk, h])
                    e = max(e, old)
                    if e > old:
                        codes[blk, h, :first] = encode(CODE[codes[blk, h, :first]] * 2.0 ** (old - e))
                sat = np.where(np.isfinite(new), np.clip(new, -top, top), new)
                codes[blk, h, first:first + b1 - b0] = encode(sat * 2.0 ** -e)
                exps[blk, h] = e

    def values(self, which: int, blocks, n: int) -> np.ndarray:
        """[n][head][dim] of a sequence's first n positions."""
        bs = self.codes[which].shape[2]
        nb = -(-n // bs)
        v = CODE[self.codes[which][blocks[:nb]]] * 2.0 ** self.exps[which][blocks[:nb]][..., None, None]
        return v.transpose(0, 2, 1, 3).reshape(-1, v.shape[1], v.shape[3])[:n]


def rotate(x: np.ndarray, cs: np.ndarray) -> np.ndarray:
    """x [rows][heads][dim] turned by cs [rows][dim/2][2]; float32, rounded once."""
    x = x.astype(np.float64)
    half = x.shape[-1] // 2
    a, b = x[..., :half], x[..., half:]
    c, s = cs[:, None, :, 0].astype(np.float64), cs[:, None, :, 1].astype(np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        return np.concatenate([a * c - b * s, b * c + a * s], -1).astype(np.float32)


def attend(q, K, V, see: int, scale: float, own=None) -> np.ndarray:
    """One row and head: q [dim] over the first `see` keys (and the own one)."""
    K, V = K[:see], V[:see]
    if own is not None:
        K, V = np.concatenate([K, own[0][None]]), np.concatenate([V, own[1][None]])
    if not len(K):
        return np.zeros(V.shape[-1])
    with np.errstate(invalid="ignore"):
        z = K @ q * scale
        p = np.exp(z - np.max(z))
        return (p[:, None] * V).sum(0) / p.sum()
