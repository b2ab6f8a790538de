"""CPU oracle for the operators around the attention calls: norms with rotation, their gradients, paged append and attention of a
batch that shares prefixes.

TEST INFRASTRUCTURE ONLY: plain fp64 numpy, written from the definitions, sharing nothing with the CUDA path.

* norm for each head   -- root mean square over the head's values, times a weight: x / sqrt(mean(x^2) + eps) * w.
* position rotation    -- Section 2.3, Eq. 1 (rope_rotate of the block-attention oracle).
* shared prefixes      -- Section 2.1 / 2.5: a token after the prompt sees every earlier token of its sequence; sequences of one group
                          have the same first tokens.
"""
from __future__ import annotations

import numpy as np

from .block_attention import ROPE_ADJACENT, ROPE_HALF


def _pairs(x, layout):
    d = x.shape[-1]
    return (x[..., 0::2], x[..., 1::2]) if layout == ROPE_ADJACENT else (x[..., :d // 2], x[..., d // 2:])


def _unpair(a, b, layout):
    out = np.empty(a.shape[:-1] + (2 * a.shape[-1],))
    if layout == ROPE_ADJACENT:
        out[..., 0::2], out[..., 1::2] = a, b
    else:
        assert layout == ROPE_HALF
        out[..., :a.shape[-1]], out[..., a.shape[-1]:] = a, b
    return out


def rotate(x, pos, theta, layout=ROPE_ADJACENT):
    """x [rows, heads, d], pos [rows]: every pair turned by pos * theta^(-2 m / d)."""
    d = x.shape[-1]
    ang = np.asarray(pos, dtype=np.float64)[:, None, None] * np.array([theta ** (-2.0 * m / d) for m in range(d // 2)])
    a, b = _pairs(x, layout)
    c, s = np.cos(ang), np.sin(ang)
    return _unpair(a * c - b * s, a * s + b * c, layout)


def head_norm(x, w, eps):
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w


def norm_rope(x, pos, w, eps, theta, layout=ROPE_ADJACENT):
    return rotate(x if w is None else head_norm(x, w, eps), pos, theta, layout)


def norm_rope_backward(x, pos, w, eps, theta, dy, layout=ROPE_ADJACENT):
    """(dx, dw): transposed rotation, then the Jacobian of x / n * w with n = sqrt(mean(x^2) + eps)."""
    g = rotate(dy, -np.asarray(pos, dtype=np.float64), theta, layout)
    if w is None:
        return g, None
    n = np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    h = g * w
    dx = h / n - x * (h * x).mean(-1, keepdims=True) / n ** 3
    return dx, (g * x / n).sum((0, 1))


def page_rows_of(page_cu, page_idx, page_rows, lst, n):
    """Pool rows of the first n rows of a list of pages."""
    return [int(page_idx[page_cu[lst] + t // page_rows]) * page_rows + t % page_rows for t in range(n)]


def shared_attend(q, keys_of, values_of, q_cu, own_len, prefix_len_of, scale):
    """q [rows, Hq, d]; keys_of(s), values_of(s): [prefix + own, Hkv, d] of sequence s; prefix_len_of(s).  Row i of the n rows of a
    sequence sees the prefix and own_len - (n - 1 - i) own rows.  Returns o, lse and sum_j p_j |v_j| (what rounding of P is bounded by);
    rows outside all sequences are NaN."""
    rows, hq, d = q.shape
    o, lse, size = np.full((rows, hq, d), np.nan), np.full((rows, hq), np.nan), np.full((rows, hq, d), np.nan)
    for s in range(len(own_len)):
        a, b = int(q_cu[s]), int(q_cu[s + 1])
        k, v = keys_of(s), values_of(s)
        G = hq // k.shape[1]
        for i in range(a, b):
            n = prefix_len_of(s) + max(0, int(own_len[s]) - (b - 1 - i))
            if n == 0:
                o[i], lse[i], size[i] = 0.0, -np.inf, 0.0
                continue
            for h in range(k.shape[1]):                       # the query heads of a KV head together
                heads = slice(h * G, (h + 1) * G)
                z = scale * (q[i, heads] @ k[:n, h].T)
                top = z.max(1, keepdims=True)
                p = np.exp(z - top)
                den = p.sum(1, keepdims=True)
                lse[i, heads] = (top + np.log(den))[:, 0]
                o[i, heads], size[i, heads] = p / den @ v[:n, h], p / den @ np.abs(v[:n, h])
    return o, lse, size
