"""Plain CPU oracle of the MXFP4 format, its product, and an expert layer's rows taken into expert order and back.

Test infrastructure, as ds3_oracle.py; it shares no code with the kernels.  MXFP4 follows the OCP Microscaling
specification's element and scale types (E2M1, E8M0, groups of 32); the scale of a group is this library's choice: the
smallest power of two with which no element exceeds 6, at least 2^-127, 1 for a group of zeros.
"""
from __future__ import annotations

import math

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
GROUP = 32


def e2m1_nearest(y) -> np.ndarray:
    """Codes 0 .. 15 of the nearest value, by search; ties to the even code (the even mantissa), the sign copied."""
    y = np.asarray(y, dtype=np.float64)
    d = np.abs(np.abs(y)[..., None] - E2M1)
    best = d.min(-1, keepdims=True)
    hit = d == best                                      # one, or two neighbours
    code = np.where(hit.sum(-1) == 1, hit.argmax(-1), np.where(hit.argmax(-1) % 2 == 0, hit.argmax(-1), hit.argmax(-1) + 1))
    return (code + 8 * np.signbit(y)).astype(np.uint8)


def e2m1_decode(code) -> np.ndarray:
    c = np.asarray(code).astype(np.int64)
    return np.where(c & 8, -1.0, 1.0) * E2M1[c & 7]


def scale_exponent(amax: float) -> int:
    """Exponent of the group's scale, by trial."""
    if amax == 0:
        return 0
    e = max(-127, math.frexp(amax)[1] - 5)
    while 6.0 * 2.0 ** e < amax:
        e += 1
    return e


def quant_mxfp4(x):
    """x float32 [M][K] -> (packed codes uint8 [M][ceil(K/2)], scale bytes uint8 [M][4 * ceil(K/128)])."""
    x = np.asarray(x, dtype=np.float32)
    m, k = x.shape
    kw = -(-k // 128)
    g = np.zeros((m, kw * 4, GROUP))
    g.reshape(m, -1)[:, :k] = x
    bad = ~np.isfinite(g).all(2)
    amax = np.where(np.isfinite(g), np.abs(g), 0).max(2)
    e = np.vectorize(scale_exponent, otypes=[np.int64])(amax)
    y = np.where(bad[..., None], 0.0, np.ldexp(np.where(np.isfinite(g), g, 0.0), -e[..., None]))
    codes = e2m1_nearest(y).reshape(m, -1)[:, : k + k % 2]
    return codes[:, 0::2] | (codes[:, 1::2] << 4), np.where(bad, 255, e + 127).astype(np.uint8)


def dequant_mxfp4(q, s, cols=None) -> np.ndarray:
    """float64 [M][cols] from packed codes and scale bytes."""
    q = np.asarray(q)
    v = np.stack([e2m1_decode(q & 15), e2m1_decode(q >> 4)], -1).reshape(q.shape[0], -1)
    v = v[:, : v.shape[1] if cols is None else cols]
    sc = np.where(s == 255, np.nan, np.ldexp(1.0, np.asarray(s).astype(np.int64) - 127))
    return v * np.repeat(sc, GROUP, axis=1)[:, : v.shape[1]]


def words(s) -> np.ndarray:
    """Scale bytes [M][4 * KB] as int32 words [M][KB], the first byte lowest."""
    return np.ascontiguousarray(s).view("<i4")


def moe_sort(ids, groups: int, first: int):
    """(offsets [groups + 1], row of every choice or -1), one choice after the other."""
    ids = np.asarray(ids)
    of = [[] for _ in range(groups)]
    for t in range(ids.shape[0]):
        for j in range(ids.shape[1]):
            if first <= int(ids[t, j]) < first + groups:
                of[int(ids[t, j]) - first].append((t, j))
    rows = np.full(ids.shape, -1, np.int32)
    off = [0]
    for group in of:
        for i, (t, j) in enumerate(group):
            rows[t, j] = off[-1] + i
        off.append(off[-1] + len(group))
    return np.array(off, np.int32), rows


def combine(y, rows, w=None):
    """float64 sums of each token's rows."""
    y = np.asarray(y, dtype=np.float64)
    out = np.zeros((rows.shape[0], y.shape[1]))
    for t, j in zip(*np.nonzero((rows >= 0) & (rows < y.shape[0]))):
        out[t] += (1.0 if w is None else float(w[t, j])) * y[rows[t, j]]
    return out


def combine_bwd(dout, y, rows, w=None):
    """(dy float64, NaN in rows that no choice names; dw float64)."""
    y, dout = np.asarray(y, dtype=np.float64), np.asarray(dout, dtype=np.float64)
    dy, dw = np.full(y.shape, np.nan), np.zeros(rows.shape)
    for t, j in zip(*np.nonzero((rows >= 0) & (rows < y.shape[0]))):
        dy[rows[t, j]] = (1.0 if w is None else float(w[t, j])) * dout[t]
        dw[t, j] = dout[t] @ y[rows[t, j]]
    return dy, dw
