"""CPU oracle of the rotation table, the norm and rotation of queries and keys, and masked attention.  TEST INFRASTRUCTURE ONLY.

Only tests may import this file; the product path never does, and it shares no code with the HIP path.  Everything is plain
numpy in fp64, from the definitions in include/dit_attn.h.
"""
from __future__ import annotations

import math

import numpy as np

__all__ = ["frequencies", "rope_table", "norm_rope", "masked_attention", "visible"]


def frequencies(axis_dim, theta, scaling, factor, original_length=None, low=1.0, high=32.0):
    """(radians per position of every pair, its axis); theta, factor, original_length: one value an axis."""
    freq, axis = [], []
    for a, d in enumerate(axis_dim):
        for j in range(d // 2):
            f = theta[a] ** (-2.0 * j / d)
            if scaling == "linear":
                f = f / factor[a]
            elif scaling == "base":
                f = (theta[a] * factor[a] ** (d / (d - 2.0))) ** (-2.0 * j / d) if d > 2 else f
            elif scaling == "bands":
                turns = original_length[a] * f / (2.0 * math.pi)
                g = min(1.0, max(0.0, (turns - low) / (high - low)))
                f = f * (g + (1.0 - g) / factor[a])
            else:
                assert scaling == "plain"
            freq.append(f)
            axis.append(a)
    return np.array(freq), np.array(axis)


def rope_table(positions, freq, axis, magnitude=1.0):
    """positions [n, axes] -> [n, pairs, 2].  Angles in extended precision: a double's product loses 1e-7 at 2^31."""
    angle = positions[:, axis].astype(np.longdouble) * freq.astype(np.longdouble)[None, :]
    return (np.stack([np.cos(angle), np.sin(angle)], 2) * magnitude).astype(np.float64)


def norm_rope(x, norm, eps, weight, bias, table, rot_dim, half):
    """x [n, H, D] fp64 -> (normed and rotated fp64, the normed values before the rotation)."""
    D = x.shape[2]
    if norm == "layer":
        x = x - x.mean(2, keepdims=True)
    if norm != "none":
        x = x / np.sqrt((x * x).sum(2, keepdims=True) / D + eps)
        x = x * (1.0 if weight is None else weight) + (0.0 if bias is None else bias)
    y = x.copy()
    for j in range(rot_dim // 2):
        a, b = (j, j + rot_dim // 2) if half else (2 * j, 2 * j + 1)
        c, s = table[:, j, 0][:, None], table[:, j, 1][:, None]
        y[:, :, a] = x[:, :, a] * c - x[:, :, b] * s
        y[:, :, b] = x[:, :, b] * c + x[:, :, a] * s
    return y, x


def visible(lq, lk, causal, prefix, q_doc, k_doc):
    """[lq, lk] truth values of one sequence."""
    pos = np.arange(lq)[:, None] + (lk - lq)
    j = np.arange(lk)[None, :]
    seen = (j <= pos) | (j < prefix) if causal else np.ones((lq, lk), bool)
    if q_doc is not None:
        seen = seen & (q_doc[:, None] == k_doc[None, :]) & (k_doc[None, :] >= 0)
    return seen


def masked_attention(q, k, v, cu_q, cu_k, scale, *, causal=False, prefix=None, cap=0.0, slopes=None, q_doc=None, k_doc=None):
    """q [Tq, H, D], k, v [Tk, G, D] fp64 -> (out, lse, mean of |v| under the probabilities, largest |score| that a row sees)."""
    Tq, H, D = q.shape
    G = k.shape[1]
    out, spread = np.zeros((Tq, H, D)), np.zeros((Tq, H, D))
    lse, top = np.full((Tq, H), -np.inf), np.zeros((Tq, H))
    for i in range(len(cu_q) - 1):
        q0, q1, k0, k1 = int(cu_q[i]), int(cu_q[i + 1]), int(cu_k[i]), int(cu_k[i + 1])
        lq, lk = q1 - q0, k1 - k0
        if lq == 0 or lk == 0:
            continue
        seen = visible(lq, lk, causal, 0 if prefix is None else int(prefix[i]), None if q_doc is None else q_doc[q0:q1],
                       None if k_doc is None else k_doc[k0:k1])
        dist = np.abs(np.arange(lq)[:, None] + (lk - lq) - np.arange(lk)[None, :])
        for h in range(H):
            g = h // (H // G)
            kk, vv = k[k0:k1, g], v[k0:k1, g]
            # what no row sees may be anything; what one row sees and another does not must be finite here
            dead = ~seen.any(0)
            kk, vv = np.where(dead[:, None], 0.0, kk), np.where(dead[:, None], 0.0, vv)
            s = q[q0:q1, h] @ kk.T * scale
            if cap:
                s = cap * np.tanh(s / cap)
            if slopes is not None:
                s = s - slopes[h] * dist
            s = np.where(seen, s, -np.inf)
            m = s.max(1, keepdims=True)
            live = m[:, 0] > -np.inf
            p = np.exp(s - np.where(np.isfinite(m), m, 0.0))
            l = p.sum(1)
            w = p / np.where(live, l, 1.0)[:, None]
            out[q0:q1, h] = w @ vv
            spread[q0:q1, h] = w @ np.abs(vv)
            lse[q0:q1, h][live] = m[live, 0] + np.log(l[live])
            top[q0:q1, h] = np.where(seen, np.abs(np.where(seen, s, 0.0)), 0.0).max(1)
    return out, lse, spread, top
