"""Plain 64-bit references of the chunk calls and of the sampler, on numpy
arrays: the 8-bit cache format, the chunk's rotation and placement, attention
over the gathered rows, and sampling by sorting.  Test infrastructure only."""
import math

import numpy as np

GRID = np.array([(c & 7) / 8 * 2.0 ** -6 if c < 8 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) for c in range(127)])


def decode(codes, scale):
    """e4m3 codes [..., D] with scale bytes [...]."""
    c = codes.astype(np.int64)
    v = np.where((c & 127) == 127, np.nan, GRID[np.minimum(c & 127, 126)]) * np.where(c >= 128, -1.0, 1.0)
    return v * 2.0 ** (scale.astype(np.float64) - 127)[..., None]


def scale_exp(x):
    """Per head row of x [..., D]: the power of two of its scale."""
    a = np.where(np.isfinite(x), np.abs(x), 0.0).max(-1)
    e = np.full(a.shape, -112)
    for i in np.ndindex(a.shape):
        while e[i] < 119 and a[i] > 448 * 2.0 ** e[i]:
            e[i] += 1
    return e


def encode(x):
    """Values of fp32 head rows after 8-bit storage, their scale bytes, and how near each is to a border between two
    codes (relative to the value)."""
    x = x.astype(np.float64)
    e = scale_exp(x)
    y = np.where(np.isfinite(x), x, 0.0) / 2.0 ** e[..., None]
    m = np.minimum(np.abs(y), 448.0)
    hi = np.minimum(np.searchsorted(GRID, m), 126)
    lo = np.maximum(hi - 1, 0)
    mid = (GRID[lo] + GRID[hi]) / 2
    up = (m > mid) | ((m == mid) & (hi % 2 == 0))
    v = np.sign(y) * GRID[np.where(up, hi, lo)] * 2.0 ** e[..., None]
    return np.where(np.isfinite(x), v, np.nan), (e + 127).astype(np.uint8), np.abs(m - mid) / np.maximum(m, 2.0 ** -9)


def rotate(x, pos, theta):
    """Rotate-half RoPE of x [rows, heads, D] at positions pos [rows], float64."""
    D = x.shape[-1]
    ang = pos[:, None] * theta ** (-2.0 * np.arange(D // 2) / D)
    c, s = np.cos(ang)[:, None], np.sin(ang)[:, None]
    a, b = x[..., : D // 2].astype(np.float64), x[..., D // 2:].astype(np.float64)
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


def places(starts, ctx):
    """(sequence, position) of every row of the chunks."""
    seq = np.concatenate([np.full(starts[b + 1] - starts[b], b) for b in range(len(ctx))]).astype(int)
    pos = np.concatenate([ctx[b] + np.arange(starts[b + 1] - starts[b]) for b in range(len(ctx))]).astype(int)
    return seq, pos


def attention(q, k, v, ctx):
    """q [n, H, D], k and v [ctx + n, Hkv, D] float64: row i sees keys 0 .. ctx + i.  Returns the output and, for
    tolerances, sum_t p_t |v_t| and the largest sum_d |q_d k_d| / sqrt(D) of a row."""
    n, H, D = q.shape
    G = H // k.shape[1]
    o, a, b = np.empty((n, H, D)), np.empty((n, H, D)), np.empty((n, H, 1))
    hidden = np.arange(k.shape[0])[None] > ctx + np.arange(n)[:, None]
    for h in range(H):
        kk, vv = k[:, h // G], v[:, h // G]
        s = np.where(hidden, -np.inf, q[:, h] @ kk.T / math.sqrt(D))
        p = np.exp(s - s.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        o[:, h], a[:, h] = p @ vv, p @ np.abs(vv)
        b[:, h] = np.where(hidden, 0, np.abs(q[:, h]) @ np.abs(kk).T / math.sqrt(D)).max(-1, keepdims=True)
    return o, a, b


def sample(l, u, T=1.0, k=0, p=1.0, m=0.0):
    """(token, probabilities) of one row; (-1, zeros) where it cannot be sampled."""
    l = l.astype(np.float64)
    ok = (math.isfinite(T) and T >= 0 and p >= 0 and 0 <= m <= 1 and 0 <= u < 1 and not np.isnan(l).any()
          and np.isfinite(l.max()))
    probs = np.zeros(len(l))
    if not ok:
        return -1, probs
    order = np.argsort(-l, kind="stable")
    order = order[: np.isfinite(l).sum()]
    if T == 0:
        order = order[:1]
    elif k > 0:
        order = order[:k]
    w = np.exp((l[order] - l[order[0]]) / (T or 1.0))
    if p < 1:
        many = max(1, 1 + int(np.searchsorted(np.cumsum(w), np.float64(p) * w.sum())))
        order, w = order[:many], w[:many]
    order, w = order[w >= m], w[w >= m]
    by = np.argsort(order)
    order, w = order[by], w[by]
    c = np.cumsum(w)
    probs[order] = w / c[-1]
    return int(order[min(int(np.searchsorted(c, np.float64(u) * c[-1], side="right")), len(order) - 1)]), probs
