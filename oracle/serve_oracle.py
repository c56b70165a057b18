"""Plain float64 definitions of the microscaled four-bit quantizer, of the
adjustment of logits, and of the gradients' norm and its clipping.

Written from the formulas in the headers (quantize.h, head_logits.h,
spike_clip.h), one step at a time; used by the tests only.
"""
from __future__ import annotations

import math

import numpy as np

F64 = np.float64
LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], F64)


# --- four bits -------------------------------------------------------------

def mx4_level(size):
    """Code of the level nearest to a size >= 0: ties to the even code, above 6 to 6."""
    off = np.abs(LEVELS - min(size, 6.0))
    near = np.flatnonzero(off == off.min())
    return int(near[0]) if len(near) == 1 else int(near[near % 2 == 0][0])


def mx4_quantize(x):
    """(codes [M][K] of 4 bits, scales [M][blocks], values float64 [M][K]) of a float array."""
    M, K = x.shape
    blocks = (K + 31) // 32
    codes, scales = np.zeros((M, K), np.uint8), np.zeros((M, blocks), np.uint8)
    values = np.zeros((M, K), F64)
    x = x.astype(F64)
    for m in range(M):
        for b in range(blocks):
            part = x[m, 32 * b:32 * b + 32]
            if not np.isfinite(part).all():
                scales[m, b] = 255
                values[m, 32 * b:32 * b + 32] = np.nan
                continue
            top = np.abs(part).max()
            p = math.frexp(top)[1] - 1 if top > 0 else -1000
            e = max(p + 125, 0)
            scales[m, b] = e
            for i, v in enumerate(part):
                c = mx4_level(abs(v) / 2.0 ** (e - 127))
                negative = bool(np.signbit(v))
                codes[m, 32 * b + i] = c + 8 * negative
                values[m, 32 * b + i] = (-1.0 if negative else 1.0) * LEVELS[c] * 2.0 ** (e - 127)
    return codes, scales, values


def mx4_pack(codes):
    """Two codes to a byte, the even one low."""
    M, K = codes.shape
    full = np.zeros((M, (K + 1) // 2 * 2), np.uint8)
    full[:, :K] = codes
    return full[:, 0::2] | full[:, 1::2] << 4


def mx4_values(codes, scales):
    """float64 values of codes [M][K] (not packed) and scales [M][blocks]."""
    K = codes.shape[1]
    v = LEVELS[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    power = np.ldexp(1.0, scales.astype(np.int64) - 127)
    power = np.where(scales == 255, np.nan, power)
    return v * np.repeat(power, 32, axis=1)[:, :K]


# --- logits ----------------------------------------------------------------

def logits_adjust(logits, ids=None, n_ids=None, n_prompt=None, drafts=None, repetition=None, presence=None, frequency=None,
                  bias_ids=None, bias=None, mask=None):
    """logits [S][n][V] float64 after penalties, biases and the mask (bool [S][n][V])."""
    S, n, V = logits.shape
    out = logits.astype(F64).copy()
    for s in range(S):
        L = 0 if ids is None else ids.shape[1]
        end = L if n_ids is None else min(max(int(n_ids[s]), 0), L)
        start = 0 if n_prompt is None else min(max(int(n_prompt[s]), 0), end)
        count, seen = np.zeros(V, F64), np.zeros(V, bool)
        for i in range(end):
            t = int(ids[s, i])
            if 0 <= t < V:
                seen[t] = True
                count[t] += i >= start
        r = 1.0 if repetition is None else F64(repetition[s])
        f = 0.0 if frequency is None else F64(frequency[s])
        p = 0.0 if presence is None else F64(presence[s])
        for j in range(n):
            if j > 0 and drafts is not None:
                t = int(drafts[s, j - 1])
                if 0 <= t < V:
                    seen[t] = True
                    count[t] += 1
            for v in np.flatnonzero(seen):
                x = out[s, j, v]
                x = x / r if x > 0 else x * r
                if count[v] > 0:
                    x = x - f * count[v]
                    x = x - p
                out[s, j, v] = x
            if bias_ids is not None:
                last = {}
                for t, b in zip(bias_ids[s], bias[s]):
                    last[int(t)] = F64(b)
                for t, b in last.items():
                    if 0 <= t < V:
                        out[s, j, t] += b
            if mask is not None:
                out[s, j][~mask[s, j]] = -np.inf
    return out


def pack_mask(mask):
    """bool [S][n][V] -> uint32 [S][n][ceil(V / 32)], bit v % 32 of word v / 32."""
    S, n, V = mask.shape
    full = np.zeros((S, n, (V + 31) // 32 * 32), bool)
    full[:, :, :V] = mask
    return np.packbits(full, axis=2, bitorder="little").view("<u4").reshape(S, n, -1)


# --- gradients -------------------------------------------------------------

def clip(grads, max_norm):
    """(norm, factor, outputs) of a list of float64 arrays."""
    norm = math.sqrt(sum(float((g.astype(F64) ** 2).sum()) for g in grads))
    factor = max_norm / norm if math.isfinite(norm) and norm > max_norm else 1.0
    return norm, factor, [g.astype(F64) * factor for g in grads]
