"""Plain float64 definitions of the operators around the projections: the
fused INT8 projection and its gradient, the embedding lookup and its table's
gradient, and the verification of drafted tokens.

Written from the formulas in the headers (dense_fused.h, spike_embed.h,
head_draft.h), one step at a time; used by the tests only.
"""
from __future__ import annotations

import math

import numpy as np

F64 = np.float64
_erf = np.vectorize(math.erf, otypes=[F64])
_erfc = np.vectorize(math.erfc, otypes=[F64])


# --- fused projection ------------------------------------------------------

def act(z, kind):
    if kind == "none":
        return z
    if kind == "relu":
        return np.where(z > 0, z, 0.0)
    if kind == "gelu":
        return z * 0.5 * _erfc(-z / math.sqrt(2.0))
    if kind == "silu":
        return z / (1.0 + np.exp(-z))
    raise ValueError(kind)


def act_slope(z, kind):
    if kind == "none":
        return np.ones_like(z)
    if kind == "relu":
        return (z > 0).astype(F64)
    if kind == "gelu":
        return 0.5 * _erfc(-z / math.sqrt(2.0)) + z * np.exp(-z * z / 2.0) / math.sqrt(2.0 * math.pi)
    if kind == "silu":
        s = 1.0 / (1.0 + np.exp(-z))
        return s + z * s * (1.0 - s)
    raise ValueError(kind)


def fused_pre(Q, scale, x, bias=None):
    """z [B][M]: one scale per output after the exact sum, then the bias."""
    z = (x.astype(F64) @ Q.astype(F64).T) * scale.astype(F64)
    return z if bias is None else z + bias.astype(F64)


def fused_forward(Q, scale, x, bias=None, kind="none", residual=None):
    y = act(fused_pre(Q, scale, x, bias), kind)
    return y if residual is None else y + residual.astype(F64)


def fused_backward(Q, scale, dy, pre=None, kind="none"):
    """(dx, dbias, g) with g = dy * act'(pre)."""
    g = dy.astype(F64)
    if kind != "none":
        g = g * act_slope(pre.astype(F64), kind)
    return (g * scale.astype(F64)) @ Q.astype(F64), g.sum(axis=0), g


# --- embedding -------------------------------------------------------------

def embed_forward(table, ids, scale, row_scale=None):
    out = np.zeros((len(ids), table.shape[1]), F64)
    for t, v in enumerate(ids):
        if 0 <= v < table.shape[0]:
            out[t] = table[v].astype(F64) * (1.0 if row_scale is None else F64(row_scale[v])) * scale
    return out


def embed_backward(grad, ids, V, scale, start=None):
    out = np.zeros((V, grad.shape[1]), F64) if start is None else start.astype(F64).copy()
    for t, v in enumerate(ids):
        if 0 <= v < V:
            out[v] += grad[t].astype(F64) * scale
    return out


# --- drafted tokens --------------------------------------------------------

def probabilities(logits, T):
    """softmax(logits / T) of one row; see head_draft.h for the special cases."""
    x = np.where(np.isnan(logits), -np.inf, logits.astype(F64))
    top = x.max()
    p = np.zeros(len(x), F64)
    if top == -np.inf:
        return p
    if not T > 0:
        p[int(np.argmax(x))] = 1.0
        return p
    if top == np.inf:
        p[x == np.inf] = 1.0
    else:
        p = np.where(x == -np.inf, 0.0, np.exp(np.where(x == -np.inf, 0.0, x - top) / T))
    return p / p.sum()


def draft_verify(target, draft, drafts, uniform, noise, n_draft=None, temperature=None):
    """tokens, n_accepted, accept, prob, and `margin`: how far (relative) the
    nearest decision of each sequence was from falling the other way."""
    S, G1, V = target.shape
    G = G1 - 1
    tokens = np.full((S, G1), -1, np.int32)
    taken = np.zeros(S, np.int32)
    accept, prob, margin = np.zeros((S, G), F64), np.zeros((S, G1), F64), np.full(S, np.inf)
    for s in range(S):
        T = 1.0 if temperature is None else float(temperature[s])
        n = G if n_draft is None else min(max(int(n_draft[s]), 0), G)
        p = [probabilities(target[s, i], T) for i in range(n + 1)]
        q = []
        for i in range(n):
            if draft is not None:
                q.append(probabilities(draft[s, i], T))
            else:
                q.append((np.arange(V) == drafts[s, i]).astype(F64))
        going = True
        for i in range(n):
            d = int(drafts[s, i])
            inside = 0 <= d < V
            pd = p[i][d] if inside else 0.0
            qd = q[i][d] if inside else 0.0
            accept[s, i] = min(1.0, pd / qd) if qd > 0 else float(pd > 0)
            if going:
                lhs = float(uniform[s, i]) * qd
                if max(lhs, pd) > 0:
                    margin[s] = min(margin[s], abs(lhs - pd) / max(lhs, pd))
                if lhs < pd:
                    tokens[s, i], prob[s, i] = d, pd
                    taken[s] += 1
                else:
                    going = False
        j = int(taken[s])
        r = p[j]
        if j < n and (p[j] - q[j] > 0).any():
            r = np.maximum(p[j] - q[j], 0.0)
        e = noise[s].astype(F64)
        ok = e > 0
        score = np.where(ok, r / np.where(ok, e, 1.0), 0.0)
        v = int(np.argmax(score))
        if score[v] > 0:
            tokens[s, j], prob[s, j] = v, p[j][v]
            rest = np.delete(score, v)
            if len(rest) and rest.max() > 0:
                second = rest.max()
                # how sure the two values are: p - q loses digits where they are close
                sure = r[v] / max(p[j][v], 1e-300)
                margin[s] = min(margin[s], (score[v] - second) / score[v] * min(1.0, sure))
    return tokens, taken, accept, prob, margin
