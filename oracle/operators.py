"""Stand-alone operators in float64 (oracle): rotary positions, attention of
documents, sampling, low-rank adapters.  Written from their definitions in include/dllm.h.

Test infrastructure only; see the package docstring.
"""
import math

import numpy as np


def rotary_rates(rot_dim, base=10000.0, scaling="none", factor=1.0, orig_len=0.0, low=1.0, high=32.0):
    """Angle per position of each pair j < rot_dim / 2."""
    f = np.array([base ** (-2.0 * j / rot_dim) for j in range(rot_dim // 2)])
    if scaling == "linear":
        return f / factor
    if scaling == "parts":
        g = np.clip((orig_len * f / (2 * math.pi) - low) / (high - low), 0.0, 1.0)
        return (1 - g) * f / factor + g * f
    return f


def rotary(x, pos, rates, interleaved=False, gain=1.0, inverse=False):
    """x [B, L, H, hd], pos [B, L] -> the same shape, the first 2 len(rates) elements turned."""
    rot = 2 * len(rates)
    ang = np.asarray(pos, dtype=np.float64)[:, :, None, None] * rates
    c, s = gain * np.cos(ang), gain * np.sin(ang) * (-1.0 if inverse else 1.0)
    y = np.array(x, dtype=np.float64, copy=True)
    ia = np.arange(0, rot, 2) if interleaved else np.arange(rot // 2)
    ib = ia + 1 if interleaved else ia + rot // 2
    a, b = y[..., ia].copy(), y[..., ib].copy()
    y[..., ia] = a * c - b * s
    y[..., ib] = b * c + a * s
    return y


def visible(pos, kv, block, prefix):
    """Keys 0 .. n-1 of kv that a query at position pos sees."""
    if block == 0:
        return kv
    return int(min(kv, max((pos // block + 1) * block, prefix, 0)))


def attention(q, k, v, pos, block=0, prefix=0, scale=None, cap=0.0, slopes=None):
    """One document: q [T, Hq, hd], k and v [S, Hkv, hd], the first query at position pos.
    Returns out [T, Hq, hd], mass [T, Hq, hd] = softmax-weighted |v|, and over the keys with a probability above
    zero the largest |score| and the largest sum |q_e k_e| [T, Hq]."""
    T, Hq, hd = q.shape
    S, Hkv, _ = k.shape
    scale = 1.0 / math.sqrt(hd) if scale is None else scale
    out, mass, top, dot = np.zeros((T, Hq, hd)), np.zeros((T, Hq, hd)), np.zeros((T, Hq)), np.zeros((T, Hq))
    for t in range(T):
        n = visible(pos + t, S, block, prefix)
        for h in range(Hq):
            g = h // (Hq // Hkv)
            s = scale * (k[:n, g] @ q[t, h])
            if cap > 0:
                s = cap * np.tanh(s / cap)
            if slopes is not None:
                s = s - slopes[h] * np.abs(pos + t - np.arange(n))
            if n == 0 or s.max() == -np.inf:
                continue
            p = np.exp(s - s.max())
            p /= p.sum()
            out[t, h], mass[t, h] = p @ v[:n, g], p @ np.abs(v[:n, g])
            some = p > 0
            if some.any():
                top[t, h], dot[t, h] = np.abs(s[some]).max(), (np.abs(k[:n, g][some]) @ np.abs(q[t, h])).max()
    return out, mass, top, dot


def shared_attention(q, k, v, pk, pv, pos, block=0, prefix=0, scale=None, cap=0.0, slopes=None):
    """One document behind a prompt: as attention, with the prompt's keys pk and values pv [P, Hkv, hd] at positions -P .. -1,
    visible to every query."""
    T, Hq, hd = q.shape
    P, G = len(pk), Hq // k.shape[1]
    scale = 1.0 / math.sqrt(hd) if scale is None else scale
    out, mass, top, dot = np.zeros((T, Hq, hd)), np.zeros((T, Hq, hd)), np.zeros((T, Hq)), np.zeros((T, Hq))
    for t in range(T):
        n = visible(pos + t, len(k), block, prefix)
        at = np.concatenate([np.arange(-P, 0), np.arange(n)])
        for h in range(Hq):
            kk, vv = np.concatenate([pk[:, h // G], k[:n, h // G]]), np.concatenate([pv[:, h // G], v[:n, h // G]])
            s = scale * (kk @ q[t, h])
            if cap > 0:
                s = cap * np.tanh(s / cap)
            if slopes is not None:
                s = s - slopes[h] * np.abs(pos + t - at)
            if len(at) == 0 or s.max() == -np.inf:
                continue
            p = np.exp(s - s.max())
            p /= p.sum()
            some = p > 0
            out[t, h], mass[t, h] = p @ vv, p @ np.abs(vv)
            if some.any():
                top[t, h], dot[t, h] = np.abs(s[some]).max(), (np.abs(kk[some]) @ np.abs(q[t, h])).max()
    return out, mass, top, dot


def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, mask_id=-1):
    """One row: (token, conf, prob)."""
    x = np.array(logits, dtype=np.float64, copy=True)
    if 0 <= mask_id < len(x):
        x[mask_id] = -np.inf
    bad = np.isnan(x) | (x == np.inf)
    if bad.any():
        return int(np.argmax(bad)), math.nan, math.nan
    if not (x > -np.inf).any():
        return -1, 0.0, 0.0
    top = x.max()
    e = np.exp(x - top)
    order = np.argsort(-x, kind="stable")
    order = order[x[order] > -np.inf]
    if not temperature > 0:
        return int(order[0]), float(1.0 / e.sum()), 1.0
    with np.errstate(over="ignore", invalid="ignore"):
        w = np.exp((x - top) / temperature)
    w[w < 2.0 ** -63] = 0.0
    if top_k >= 1:
        order = order[:top_k]
    if top_p < 1:
        before = np.concatenate([[0.0], np.cumsum(w[order])[:-1]])
        stay = before < top_p * w[order].sum()
        stay[0] = True
        order = order[stay]
    if min_p > 0:
        order = order[(top - x[order]) / temperature <= -math.log(min(min_p, 1.0))]    # w >= min_p
    kept = np.zeros(len(x), dtype=bool)
    kept[order] = True
    c = np.cumsum(np.where(kept, w, 0.0))
    u = min(max(u, 0.0), 1 - 2.0 ** -24) if u == u else 0.0
    token = min(int((c <= u * c[-1]).sum()), int(np.nonzero(kept)[0].max()))
    return token, float(e[token] / e.sum()), float(w[token] / c[-1])


def adapters(x, base, A, B, which, ranks, scales, ends):
    """x [M, K], base [M, N], A [n, S, R, K], B [n, N, R]; ends: each slice's last column + 1.  Returns out [M, N] and
    mass [M, N] = |scale| sum_j |B_j| sum_k |A_jk x_k|, what the two products' errors are relative to."""
    out, mass = np.array(base, dtype=np.float64, copy=True), np.zeros(base.shape)
    for m, a in enumerate(which):
        if not 0 <= a < len(A):
            continue
        r, first = int(min(max(ranks[a], 0), A.shape[2])), 0
        for s, end in enumerate(ends):
            b = B[a, first:end, :r]
            out[m, first:end] += scales[a] * (b @ (A[a, s, :r] @ x[m]))
            mass[m, first:end] = abs(scales[a]) * (np.abs(b) @ (np.abs(A[a, s, :r]) @ np.abs(x[m])))
            first = end
    return out, mass
