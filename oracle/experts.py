"""FP64 reference of what stands around the grouped (mixture-of-experts) layer -- the router's
choice and weights, the sort of token slots by expert, the weighted sum back, and their gradients
(QATFactory Sec. 3.3 "Mixture-of-experts adaptation") -- and of products with packed weights taken
exactly as their codes decode (Eqs. nvfp4-dequant, mxfp4-dequant, q4k-dequant).

Plain numpy loops over tokens and slots; shares no code with the GPU library.
"""
from __future__ import annotations

import math

import numpy as np

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _sigmoid(v):
    return 1.0 / (1.0 + math.exp(-v)) if v >= 0 else math.exp(v) / (1.0 + math.exp(v))


def _log_sigmoid(v):
    return min(v, 0.0) - math.log1p(math.exp(-abs(v)))


def choose(row, k):
    """Experts of the k largest logits, largest first, equal ones by rising expert; NaN above all,
    -inf never."""
    order = sorted(range(len(row)), key=lambda e: (not math.isnan(row[e]), -row[e] if row[e] == row[e] else 0.0, e))
    return [e for e in order if not row[e] == -math.inf][:k]


def scores(row, ids, score, norm):
    """The weights (before the scale) of the chosen experts of one row."""
    if not ids:
        return []
    if norm:
        a = [row[e] if score == "softmax" else _log_sigmoid(row[e]) for e in ids]
        m = max(a)
        x = [math.exp(v - m) for v in a]
        return [v / math.fsum(x) for v in x]
    if score == "sigmoid":
        return [_sigmoid(row[e]) for e in ids]
    m = max(row)
    s = math.fsum(math.exp(v - m) for v in row)
    return [math.exp(row[e] - m) / s for e in ids]


def route(z, k, score="softmax", norm=True, scale=1.0, mask=None):
    T = z.shape[0]
    ids, w = np.full((T, k), -1, np.int32), np.zeros((T, k))
    for t in range(T):
        if mask is not None and not mask[t]:
            continue
        row = [float(v) for v in z[t]]
        c = choose(row, k)
        ids[t, :len(c)] = c
        w[t, :len(c)] = [scale * v for v in scores(row, c, score, norm)]
    return ids, w


def route_bwd(z, ids, dw, score="softmax", norm=True, scale=1.0):
    T, E = z.shape
    dz = np.zeros((T, E))
    for t in range(T):
        slots = [j for j in range(ids.shape[1]) if 0 <= ids[t, j] < E]
        c = [int(ids[t, j]) for j in slots]
        if not c:
            continue
        row = [float(v) for v in z[t]]
        g = [scale * float(dw[t, j]) for j in slots]
        q = scores(row, c, score, norm)
        dot = math.fsum(a * b for a, b in zip(q, g))
        if norm:
            for e, qe, ge in zip(c, q, g):
                dz[t, e] = qe * (ge - dot) * (_sigmoid(-row[e]) if score == "sigmoid" else 1.0)
        elif score == "sigmoid":
            for e, qe, ge in zip(c, q, g):
                dz[t, e] = ge * qe * _sigmoid(-row[e])
        else:
            m = max(row)
            p = [math.exp(v - m) for v in row]
            s = math.fsum(p)
            for e in range(E):
                dz[t, e] = p[e] / s * ((g[c.index(e)] if e in c else 0.0) - dot)
    return dz


def dispatch(ids, E):
    """offsets [E+1], row_of [T, k], slot_of [T k]."""
    flat = ids.reshape(-1)
    n = flat.size
    groups = [[] for _ in range(E + 1)]
    for slot in range(n):
        e = int(flat[slot])
        groups[e if 0 <= e < E else E].append(slot)
    offsets = np.zeros(E + 1, np.int64)
    row_of, slot_of = np.zeros(n, np.int32), np.full(n, -1, np.int32)
    row = 0
    for e, slots in enumerate(groups):
        for slot in slots:
            row_of[slot] = row if e < E else ~row
            if e < E:
                slot_of[row] = slot
            row += 1
        if e < E:
            offsets[e + 1] = row
    return offsets, row_of.reshape(ids.shape), slot_of


def gather(slot_of, X, k):
    out = np.zeros((slot_of.size, X.shape[1]), X.dtype)
    live = slot_of >= 0
    out[live] = X[slot_of[live] // k]
    return out


def combine(row_of, Yg, w=None):
    T, k = row_of.shape
    Y = np.zeros((T, Yg.shape[1]))
    for j in range(k):
        for t in np.nonzero(row_of[:, j] >= 0)[0]:
            Y[t] += (1.0 if w is None else float(w[t, j])) * Yg[row_of[t, j]]
    return Y


def combine_bwd(row_of, dY, Yg, w=None):
    T, k = row_of.shape
    dYg, dw = np.zeros(Yg.shape), np.zeros((T, k))
    for t in range(T):
        for j in range(k):
            r = int(row_of[t, j])
            if r >= 0:
                dYg[r] = (1.0 if w is None else float(w[t, j])) * dY[t]
                dw[t, j] = float(np.dot(dY[t], Yg[r]))
    return dYg, dw


def e4m3(c):
    c = int(c)
    sign, e, m = (-1.0 if c & 128 else 1.0), (c >> 3) & 15, c & 7
    if e == 15 and m == 7:
        return math.nan
    return sign * (m / 512.0 if e == 0 else 2.0 ** (e - 7) * (1 + m / 8))


def decode(fmt, codes, scales=None, S=None):
    """The packed weight [R, K] in 64 bits; codes [R, K/2] (Q4_K: [R, K/256, 144]) bytes."""
    R = codes.shape[0]
    if fmt == "q4k":
        blocks = codes.reshape(R, -1, 144)
        out = np.zeros((R, blocks.shape[1], 8, 32))
        d = np.ascontiguousarray(blocks[..., 0:2]).view(np.float16)[..., 0].astype(np.float64)
        dm = np.ascontiguousarray(blocks[..., 2:4]).view(np.float16)[..., 0].astype(np.float64)
        b = blocks.astype(np.int64)
        for j in range(8):
            if j < 4:
                s6, m6 = b[..., 4 + j] & 63, b[..., 8 + j] & 63
            else:
                s6 = (b[..., 8 + j] & 15) | ((b[..., j] >> 6) << 4)
                m6 = (b[..., 8 + j] >> 4) | ((b[..., 4 + j] >> 6) << 4)
            q = b[..., 16 + 32 * (j // 2):48 + 32 * (j // 2)]
            q = (q & 15) if j % 2 == 0 else (q >> 4)
            out[:, :, j] = (d * s6)[..., None] * q - (dm * m6)[..., None]
        return out.reshape(R, -1)
    K = codes.shape[1] * 2
    nib = np.empty((R, K), np.int64)
    nib[:, 0::2], nib[:, 1::2] = codes & 15, codes >> 4
    lut = np.array(E2M1 + tuple(-v for v in E2M1))
    if fmt == "nvfp4":
        d = np.array([e4m3(c) for c in range(256)])[scales] * np.float64(S)
    else:
        d = np.array([2.0 ** (c - 127) for c in range(255)] + [math.nan])[scales]
    return lut[nib] * np.repeat(d, K // d.shape[1], axis=1)
