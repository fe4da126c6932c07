"""The expanded cache in E4M3 codes with a power of two per block of 32 tokens and group, written out independently of the library.
TEST INFRASTRUCTURE ONLY (same rule as gqla_oracle.py).  The format of the codes is the one of fp8_cache.py.

A block is the tokens 32 i .. 32 i + 31 of one group, K or V apart.  Its scale is 2^e, e the smallest integer with
amax <= 448 * 2^e (amax: the largest finite magnitude), kept in [-100, 118];  code = E4M3(x * 2^-e), infinities and magnitudes
beyond 448 * 2^e become +-448 * 2^e, NaN stays NaN.  Rows appended to a block with older tokens: the larger of its exponent and
the one the new rows need; the older codes are rounded to it.

Page (bytes; P tokens, g groups):  K8 [g][d_h/16][P][16] | V8 [g][P/32][d_v][2][16] | k_R [d_r/8][P][8] 16-bit | scales [g][P/32][2] fp32
"""
from __future__ import annotations

import math

import numpy as np

from .fp8_cache import E4M3_MAX, dequantize_e4m3, quantize_e4m3

BLOCK, E_MIN, E_MAX = 32, -100, 118


def block_exponent(values):
    """By search over the definition; exact in double."""
    v = np.abs(np.asarray(values, np.float64))
    v = v[np.isfinite(v)]
    amax = float(v.max()) if v.size else 0.0
    for e in range(E_MIN, E_MAX):
        if amax <= E4M3_MAX * 2.0 ** e:
            return e
    return E_MAX


def codes_of(x, e):
    q = np.asarray(x, np.float64) * 2.0 ** -e
    nan = np.isnan(q)
    code = quantize_e4m3(np.clip(np.where(nan, 0.0, q), -E4M3_MAX, E4M3_MAX).astype(np.float32))
    return np.where(nan, np.uint8(0x7F), code)


def same_codes(a, b):
    """Equal, either code of NaN being as good as the other."""
    a, b = np.asarray(a), np.asarray(b)
    return (a == b) | (((a & 0x7F) == 0x7F) & ((b & 0x7F) == 0x7F))


class Plane:
    """One sequence's K or V: codes [tokens][g][d] and exponents [blocks][g]."""

    def __init__(self, g, d):
        self.codes, self.e = np.zeros((0, g, d), np.uint8), np.zeros((0, g), np.int64)

    def append(self, x):
        """x [n][g][d], storage-rounded values."""
        x = np.asarray(x, np.float64)
        start, (n, g, d) = len(self.codes), x.shape
        self.codes = np.concatenate([self.codes, np.zeros((n, g, d), np.uint8)])
        blocks = -(-(start + n) // BLOCK)
        self.e = np.concatenate([self.e, np.full((blocks - len(self.e), g), E_MIN - 1, np.int64)])
        for i in range(start // BLOCK, blocks):
            lo, hi = max(start, BLOCK * i), min(start + n, BLOCK * (i + 1))
            if lo >= hi:
                continue
            for j in range(g):
                e = block_exponent(x[lo - start: hi - start, j])
                if lo > BLOCK * i:                                   # older tokens
                    was = int(self.e[i, j])
                    e = max(e, was)
                    if e > was:
                        old = dequantize_e4m3(self.codes[BLOCK * i: lo, j])
                        self.codes[BLOCK * i: lo, j] = codes_of(old, e - was)
                self.e[i, j] = e
                self.codes[lo:hi, j] = codes_of(x[lo - start: hi - start, j], e)
        return self

    def values(self):
        return dequantize_e4m3(self.codes) * 2.0 ** np.repeat(self.e, BLOCK, 0)[: len(self.codes), :, None]


def page_bytes(P, g, d_h, d_v, d_r):
    return P * (g * (d_h + d_v) + 2 * d_r) + g * (P // BLOCK) * 8


def k_offset(j, slot, d, P, g, d_h, d_v, d_r):
    kp, u, h, i = d // 32, d // 16 % 2, d // 8 % 2, d % 8
    return ((j * (d_h // 16) + 2 * kp + h) * P + slot) * 16 + 8 * u + i


def v_offset(j, slot, d, P, g, d_h, d_v, d_r):
    T, u, h, i = slot // 32, slot // 16 % 2, slot // 8 % 2, slot % 8
    return g * P * d_h + (((j * (P // 32) + T) * d_v + d) * 2 + h) * 16 + 8 * u + i


def kr_offset(slot, d, P, g, d_h, d_v, d_r):
    return g * P * (d_h + d_v) + ((d // 8 * P + slot) * 8 + d % 8) * 2


def scale_offset(j, T, kind, P, g, d_h, d_v, d_r):
    return P * (g * (d_h + d_v) + 2 * d_r) + ((j * (P // BLOCK) + T) * 2 + kind) * 4


def store(pool, pages, P, K, V, kR_bits, first_token=0):
    """Tokens first_token .. of one sequence (Plane K and V, k_R as uint16 bit patterns [tokens][d_r]) into pool
    (uint8 [num_pages][page bytes]) at the pages of its table row.  A page id outside the pool: its tokens go nowhere."""
    g, d_h, d_v, d_r = K.codes.shape[1], K.codes.shape[2], V.codes.shape[2], kR_bits.shape[1]
    dims = (P, g, d_h, d_v, d_r)
    j, dk, dv, dr = np.arange(g)[:, None], np.arange(d_h), np.arange(d_v), np.arange(d_r)
    for t in range(first_token, len(K.codes)):
        if t // P >= len(pages) or not 0 <= pages[t // P] < len(pool):
            continue
        page, slot = pool[pages[t // P]], t % P
        page[k_offset(j, slot, dk, *dims)] = K.codes[t]
        page[v_offset(j, slot, dv, *dims)] = V.codes[t]
        o = kr_offset(slot, dr, *dims)
        page[o], page[o + 1] = kR_bits[t] & 0xFF, kR_bits[t] >> 8
    for i in range(first_token // BLOCK, len(K.e)):
        t = BLOCK * i
        if t // P >= len(pages) or not 0 <= pages[t // P] < len(pool):
            continue
        page, T = pool[pages[t // P]], t % P // BLOCK
        for jj in range(g):
            for kind, plane in enumerate((K, V)):
                o = scale_offset(jj, T, kind, *dims)
                page[o: o + 4] = np.frombuffer(np.float32(2.0 ** plane.e[i, jj]).tobytes(), np.uint8)


def attend(qC, qR, K, V, kR, L, hidden=None, scale=None):
    """The GQA-path equation for n query rows at positions L - n .. L - 1:  qC [n][h_q][d_h], qR [n][h_q][d_r]; K [L][g][d_h],
    V [L][g][d_v], kR [L][d_r]; hidden: tokens that no row sees.  -> (o, lse, weight) with weight = softmax |V|, what rounding
    errors of the probabilities are relative to; a row that sees nothing: 0, -inf, 0."""
    qC, qR, K, V, kR = (np.asarray(a, np.float64) for a in (qC, qR, K, V, kR))
    n, h_q, d_h = qC.shape
    G = h_q // K.shape[1]
    sigma = 1.0 / math.sqrt(d_h + qR.shape[2]) if scale is None else scale
    pos = L - n + np.arange(n)
    see = np.arange(L)[None, :] <= pos[:, None]
    if hidden is not None:
        see &= ~np.asarray(hidden)[None, :]
    o, w, lse = np.zeros((n, h_q, V.shape[2])), np.zeros((n, h_q, V.shape[2])), np.full((n, h_q), -np.inf)
    for i in range(h_q):
        z = np.where(see, (qC[:, i] @ K[:, i // G].T + qR[:, i] @ kR.T) * sigma, -np.inf)
        some = see.any(1)
        if not some.any():
            continue
        top = z[some].max(1, keepdims=True)
        p = np.exp(z[some] - top)
        den = p.sum(1, keepdims=True)
        o[some, i], w[some, i] = p / den @ V[:, i // G], p / den @ np.abs(V[:, i // G])
        lse[some, i] = (top + np.log(den))[:, 0]
    return o, lse, w


def logit_error(qC, qR, K, kR, scale):
    """How far an fp32 logit can be off: each of its products and sums rounds by at most 2^-24 of a partial sum."""
    size = np.abs(qC).max(0).max(0) @ np.abs(K).max(0).max(0) + np.abs(qR).max(0).max(0) @ np.abs(kR).max(0)
    return (qC.shape[2] + qR.shape[2] + 2) * 2.0 ** -24 * float(size) * scale
