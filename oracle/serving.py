"""FP64 reference of the decode step's operators around the packed products: the 4-bit cache of keys and
values in pages, the attention that reads it (QATFactory Sec. 3.2.3's formats) and the low-rank adapters of
many requests (Eq. qad-lora's factors beside a shared projection).

Plain numpy over tokens and heads; shares no code with the GPU library.
"""
from __future__ import annotations

import math

import numpy as np

import oracle
from oracle import experts as ox

BLOCK = {"nvfp4": 16, "mxfp4": 32}


def places(offsets, lens, table, page, pages, T):
    """(page, offset) of each of T rows, None for one without a place; "nobody" for one of no sequence."""
    B = len(lens)
    out = ["nobody"] * T
    for b in range(B):
        lo, hi = (b, b + 1) if offsets is None else (int(offsets[b]), int(offsets[b + 1]))
        for t in range(lo, min(hi, T)):
            pos = int(lens[b]) - (hi - t)
            out[t] = None
            if 0 <= pos < table.shape[1] * page:
                p = int(table[b, pos // page])
                if 0 <= p < pages:
                    out[t] = (p, pos % page)
    return out


def quantize_heads(x, H, fmt, amax=None):
    """codes [T, H, D/2], scales [T, H, D/B], S [H] and x_hat bits [T, H, D] of bf16 bits x [T, H D], head h
    under the tensor amax amax[h] (nvfp4)."""
    T, D = x.shape[0], x.shape[1] // H
    x = x.reshape(T, H, D)
    parts = [oracle.nvfp4(x[:, h], float(amax[h])) if fmt == "nvfp4" else oracle.mxfp4(x[:, h]) for h in range(H)]
    S = np.array([p["S"] for p in parts], np.float32) if fmt == "nvfp4" else None
    return [np.stack([p[n] for p in parts], 1) for n in ("codes", "scales")] + [S, np.stack([p["xhat"] for p in parts], 1)]


def write(codes, scales, where, new_codes, new_scales):
    """Puts the rows' codes and scales [T, H, ..] into copies of the pages [pages, H, page, ..]."""
    codes, scales = codes.copy(), scales.copy()
    for t, w in enumerate(where):
        if w not in (None, "nobody"):
            codes[w[0], :, w[1]], scales[w[0], :, w[1]] = new_codes[t], new_scales[t]
    return codes, scales


def values(codes, scales, S, fmt):
    """FP64 values [pages, H, page, D] of a whole pool."""
    P, H, page, half = codes.shape
    out = np.empty((P, H, page, 2 * half))
    for h in range(H):
        s = scales[:, h].reshape(P * page, -1)
        s = s if s.shape[1] else s
        out[:, h] = ox.decode(fmt, codes[:, h].reshape(P * page, half), s, None if S is None else float(S[h])).reshape(P, page, -1)
    return out


def attention(q, K, V, offsets, lens, table, scale, window=0, max_len=None):
    """O [T, Hq, D], lse [T, Hq] and, for bounds, the largest |scale| sum |q||k| of each row, the weighted
    sums of |v| and the plain sums of |v|.  q FP64 [T, Hq, D]; K, V FP64 [pages, H, page, D].  Rows of no
    sequence are NaN throughout."""
    T, Hq, D = q.shape
    pages, H, page, _ = K.shape
    G = Hq // H
    O, lse = np.full((T, Hq, D), np.nan), np.full((T, Hq), np.nan)
    big, wv, sv = np.zeros((T, Hq)), np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    cap = table.shape[1] * page if max_len is None else min(max_len, table.shape[1] * page)
    for b in range(len(lens)):
        lo, hi = (b, b + 1) if offsets is None else (int(offsets[b]), int(offsets[b + 1]))
        n = max(0, min(int(lens[b]), cap))
        pos = np.arange(n)
        pg = table[b, pos // page] if n else np.zeros(0, np.int64)
        good = (pg >= 0) & (pg < pages)
        pos, pg = pos[good], pg[good]
        k, v = K[pg, :, pos % page], V[pg, :, pos % page]          # [n, H, D]
        for t in range(lo, min(hi, T)):
            own = int(lens[b]) - (hi - t)
            see = pos <= own
            if window:
                see &= pos > own - window
            O[t], lse[t] = 0.0, -math.inf
            if not see.any():
                continue
            for h in range(H):
                kk, vv = k[see, h], v[see, h]
                qq = q[t, h * G:(h + 1) * G]
                with np.errstate(all="ignore"):
                    z = scale * (qq @ kk.T)
                    m = z.max(1, keepdims=True)
                    p = np.exp(z - m)
                    s = p.sum(1, keepdims=True)
                    O[t, h * G:(h + 1) * G] = (p / s) @ vv
                    lse[t, h * G:(h + 1) * G] = (m + np.log(s))[:, 0]
                    big[t, h * G:(h + 1) * G] = (abs(scale) * np.abs(qq) @ np.abs(kk).T).max(1)
                    wv[t, h * G:(h + 1) * G] = (p / s) @ np.abs(vv)
                    sv[t, h * G:(h + 1) * G] = np.abs(vv).sum(0)
    return O, lse, big, wv, sv


def lora_rows(ids, x, A, B, scale, base=None, ranks=None):
    """Y [M, N] of FP64 x [M, K], A [n, r, K], B [n, N, r]; and sum |z||b| |scale| and the largest sum |x||a|
    of a row, for bounds."""
    M, N = x.shape[0], B.shape[1]
    Y = np.zeros((M, N)) if base is None else base.copy()
    mag = np.zeros((M, N))
    for m in range(M):
        a = int(ids[m])
        if not 0 <= a < A.shape[0]:
            continue
        r = A.shape[1] if ranks is None else min(max(int(ranks[a]), 0), A.shape[1])
        z = A[a, :r] @ x[m]
        Y[m] += scale[a] * (B[a, :, :r] @ z)
        mag[m] = abs(scale[a]) * (np.abs(B[a, :, :r]) @ (np.abs(A[a, :r]) @ np.abs(x[m])))
    return Y, mag
