"""fp64 CPU oracle of the rotary tables, the rotation and the paged cache of 8-bit codes.

TEST INFRASTRUCTURE ONLY, like the rest of this package.  Plain numpy loops over sequences, pages and heads:
the definitions of include/rvq.h, written without the library and without its layout tricks.  The cache's arrays are
those of the header: codes uint8 [n_pages][n_kv_heads][2][64 * head_dim], scales [n_pages][n_kv_heads][2].
"""
from __future__ import annotations

import math

import numpy as np

PAGE = 64
ADJACENT, HALVES = 0, 1


def tables(positions, rot, base=10000.0, factor=1.0, orig_len=0.0, alpha=1.0, beta=32.0, amplitude=1.0):
    half = rot // 2
    theta = np.empty(half)
    for i in range(half):
        f = base ** (-2.0 * i / rot)
        g = 0.0
        if orig_len > 0.0:
            g = min(1.0, max(0.0, (orig_len * f / (2.0 * math.pi) - alpha) / (beta - alpha)))
        theta[i] = f if factor == 1.0 else g * f + (1.0 - g) * f / factor
    ang = np.asarray(positions, dtype=np.float64)[:, None] * theta
    return amplitude * np.cos(ang), amplitude * np.sin(ang)


def rotate(x, cos, sin, layout):
    """x [N][heads][hd]; cos, sin [N][rot / 2]."""
    y = np.array(x, dtype=np.float64)
    half = cos.shape[1]
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if layout == ADJACENT else (i, i + half)
        c, s = cos[:, i, None], sin[:, i, None]
        p, q = np.array(x[..., a], dtype=np.float64), np.array(x[..., b], dtype=np.float64)
        y[..., a] = p * c - q * s
        y[..., b] = p * s + q * c
    return y


def _values():
    v = np.empty(256)
    for code in range(256):
        e, m = (code >> 3) & 15, code & 7
        x = (8 + m) * 2.0 ** (e - 10) if e else m * 2.0**-9
        v[code] = math.nan if (code & 127) == 127 else (-x if code & 128 else x)
    return v


VALUES = _values()  # of the 256 codes
_POS = VALUES[:127]


def encode(x):
    """Nearest code of every number, |x| <= 448, ties to even codes; not finite becomes NaN."""
    x = np.asarray(x, dtype=np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    assert a.size == 0 or a.max() <= 448.0
    hi = np.clip(np.searchsorted(_POS, a), 1, 126)
    lo = hi - 1
    dl, dh = a - _POS[lo], _POS[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    code = code | np.where(np.signbit(x), 128, 0)
    return np.where(np.isfinite(x), code, 127).astype(np.uint8)


def scale_of(amax):
    e = -100
    while amax > 448.0 * 2.0**e:
        e += 1
    return 2.0**e


def steps(cu, rows):
    """(first row, rows) of every sequence, inside [0, rows)."""
    out = []
    for lo, hi in zip(cu[:-1], cu[1:]):
        lo = min(max(int(lo), 0), rows)
        hi = min(max(int(hi), lo), rows)
        out.append((lo, hi - lo))
    return out


def page_of(table, b, entry, n_pages):
    if entry < 0 or entry >= table.shape[1]:
        return -1
    p = int(table[b, entry])
    return p if 0 <= p < n_pages else -1


def append(codes, scales, k, v, cu, table, lengths, cos=None, sin=None, layout=ADJACENT):
    """New codes and scales, and the exact (rotated) numbers behind the new tokens' codes: {(page, head, 0|1, slot): vector}."""
    n_pages, heads, _, size = codes.shape
    hd = size // PAGE
    codes, scales = codes.copy(), np.array(scales, dtype=np.float64)
    kk = rotate(k, cos, sin, layout) if cos is not None else np.array(k, dtype=np.float64)
    vv = np.array(v, dtype=np.float64)
    exact = {}
    for b, (row, n) in enumerate(steps(cu, len(kk))):
        p0 = int(lengths[b]) - n
        for entry in sorted({(p0 + i) // PAGE for i in range(n)}):
            page = page_of(table, b, entry, n_pages)
            if page < 0:
                continue
            lo, hi = max(p0, entry * PAGE), min(p0 + n, (entry + 1) * PAGE)
            s0 = lo - entry * PAGE
            for h in range(heads):
                for kind, x in ((0, kk), (1, vv)):
                    part = x[row + lo - p0 : row + hi - p0, h]  # [tokens][hd]
                    fin = np.abs(part[np.isfinite(part)])
                    s = scale_of(fin.max() if fin.size else 0.0)
                    tile = codes[page, h, kind].reshape((PAGE, hd) if kind == 0 else (hd, PAGE))
                    tile = tile if kind == 0 else tile.T  # [slot][channel], a view
                    if s0:
                        old = scales[page, h, kind]
                        if s > old:
                            was = tile[:s0]
                            again = encode(np.where(np.isnan(VALUES[was]), 0.0, VALUES[was]) * (old / s))
                            tile[:s0] = np.where(np.isnan(VALUES[was]), 127, again)
                        s = max(s, old)
                    scales[page, h, kind] = s
                    tile[s0 : s0 + hi - lo] = encode(part / s)
                    for i in range(hi - lo):
                        exact[page, h, kind, s0 + i] = part[i]
    return codes, scales, exact


def token(codes, scales, table, lengths, b, pos):
    """(k, v) [heads][hd] of a token, or None: it is not in the cache."""
    n_pages, heads, _, size = codes.shape
    page = page_of(table, b, pos // PAGE, n_pages) if 0 <= pos < int(lengths[b]) else -1
    if page < 0:
        return None
    hd, slot = size // PAGE, pos % PAGE
    k = VALUES[codes[page, :, 0].reshape(heads, PAGE, hd)[:, slot]] * scales[page, :, 0, None]
    v = VALUES[codes[page, :, 1].reshape(heads, hd, PAGE)[:, :, slot]] * scales[page, :, 1, None]
    return k, v


def read(codes, scales, rows, cu, first, table, lengths, cos=None, sin=None, layout=ADJACENT):
    heads, hd = codes.shape[1], codes.shape[3] // PAGE
    k, v = np.zeros((rows, heads, hd)), np.zeros((rows, heads, hd))
    for b, (row, n) in enumerate(steps(cu, rows)):
        for i in range(n):
            t = token(codes, scales, table, lengths, b, int(first[b]) + i)
            if t is not None:
                k[row + i], v[row + i] = t
    if cos is not None:
        cos, sin = np.asarray(cos, dtype=np.float64), np.asarray(sin, dtype=np.float64)
        square = cos * cos + sin * sin  # of the tables' amplitude
        k = rotate(k, cos / square, -sin / square, layout)
    return k, v


def attend(codes, scales, q, cu, table, lengths, scale, window=0, sinks=0):
    """out, and for every row and head the largest |k| |q| and |v| sums a tolerance is made of: (out, score size, value size)."""
    n_pages, heads, _, size = codes.shape
    hd = size // PAGE
    q = np.asarray(q, dtype=np.float64)
    rows, hq, _ = q.shape
    rep = hq // heads
    out, score_size, value_size = np.zeros(q.shape), np.zeros((rows, hq)), np.zeros((rows, hq, hd))
    for b, (row, n) in enumerate(steps(cu, rows)):
        if n == 0:
            continue
        held = [t for t in range(max(0, int(lengths[b]))) if page_of(table, b, t // PAGE, n_pages) >= 0]
        pairs = [token(codes, scales, table, lengths, b, t) for t in held]
        held = np.array(held, dtype=np.int64)
        kk = np.array([x[0] for x in pairs]).reshape(-1, heads, hd)
        vv = np.array([x[1] for x in pairs]).reshape(-1, heads, hd)
        for i in range(n):
            p = int(lengths[b]) - n + i
            sees = (held <= p) & ((window == 0) | (held > p - window) | (held < sinks))
            if not sees.any():
                continue
            for a in range(hq):
                ks, vs, x = kk[sees, a // rep], vv[sees, a // rep], q[row + i, a]
                s = ks @ x * scale
                w = np.exp(s - s.max())
                w /= w.sum()
                out[row + i, a] = w @ vs
                score_size[row + i, a] = (np.abs(ks) @ np.abs(x)).max() * abs(scale)
                value_size[row + i, a] = w @ np.abs(vs)
    return out, score_size, value_size
