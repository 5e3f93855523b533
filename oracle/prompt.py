"""Plain fp64 definitions of what brings prompts into the paged cache and reads shared prefixes.

Written from the formulas of ``include/qfattn.h``: one request, token and head at a time, with no
structure in common with the kernels (test infrastructure only).  Arrays are numpy float64.
"""

from __future__ import annotations

import numpy as np

PAGE = 16


def rotate(x, pos, freqs, layout, amplitude):
    """One head x [D] at position ``pos``: pair i turned by pos * freqs[i], scaled by ``amplitude``."""
    y = np.array(x, dtype=np.float64)
    r = len(freqs)
    for i, f in enumerate(freqs):
        a, b = (i, i + r) if layout == "half" else (2 * i, 2 * i + 1)
        c, s = np.cos(pos * f) * amplitude, np.sin(pos * f) * amplitude
        y[a], y[b] = x[a] * c - x[b] * s, x[b] * c + x[a] * s
    return y


def norm_rotate(x, pos, gain, eps, freqs, layout, amplitude):
    """One head normalised (with a gain), then rotated (with frequencies)."""
    x = np.asarray(x, dtype=np.float64)
    if gain is not None:
        x = x / np.sqrt(np.mean(x * x) + eps) * gain
    return x if freqs is None else rotate(x, pos, freqs, layout, amplitude)


def rope_append(q, k, v, k_cache, v_cache, table, ctx, cu, *, gains=(None, None), eps=1e-6, freqs=None,
                layout="half", amplitude=1.0):
    """(q_out, k_cache, v_cache) after the call; rows of no request of q_out are NaN."""
    q_out = np.full(q.shape, np.nan)
    kc, vc = k_cache.copy(), v_cache.copy()
    for b in range(len(ctx)):
        for t in range(cu[b], cu[b + 1]):
            pos = int(ctx[b]) + t - int(cu[b])
            for h in range(q.shape[1]):
                q_out[t, h] = norm_rotate(q[t, h], pos, gains[0], eps, freqs, layout, amplitude)
            if pos >= table.shape[1] * PAGE or not 0 <= table[b, pos // PAGE] < kc.shape[0]:
                continue
            page = table[b, pos // PAGE]
            for g in range(k.shape[1]):
                kc[page, g, pos % PAGE] = norm_rotate(k[t, g], pos, gains[1], eps, freqs, layout,
                                                      amplitude)
                vc[page, g, pos % PAGE] = v[t, g]
    return q_out, kc, vc


def positions(cache, pages, n, g):
    """The first n positions of KV head g on the given pages, [n, D]."""
    if n == 0:
        return np.zeros((0, cache.shape[-1]))
    return np.concatenate([cache[p, g] for p in pages[: -(-n // PAGE)]])[:n]


def attend(q, k, v, scale):
    """q [D] over k, v [n, D]: (out, lse, the same weighted mean of |v|)."""
    if len(k) == 0:
        return np.zeros(len(q)), -np.inf, np.zeros(len(q))
    s = scale * (k @ q)
    m = np.max(s)
    if m == -np.inf:
        return np.zeros(len(q)), -np.inf, np.zeros(len(q))
    w = np.exp(s - m)
    z = np.sum(w)
    return w @ v / z, m + np.log(z), w @ np.abs(v) / z


def prefill(q, k_cache, v_cache, table, ctx, cu, scale):
    """(out [T, Hq, D], lse [T, Hq], spread [T, Hq, D]); spread is the weighted mean of |v|, which a
    rounding of the weights is measured by.  Rows of no request are NaN."""
    T, Hq, D = q.shape
    G = Hq // k_cache.shape[1]
    out, lse, spread = np.full((T, Hq, D), np.nan), np.full((T, Hq), np.nan), np.full((T, Hq, D), np.nan)
    for b in range(len(ctx)):
        for g in range(k_cache.shape[1]):
            n = int(ctx[b]) + int(cu[b + 1] - cu[b])
            k, v = positions(k_cache, table[b], n, g), positions(v_cache, table[b], n, g)
            for t in range(cu[b], cu[b + 1]):
                seen = int(ctx[b]) + t - int(cu[b]) + 1
                for h in range(g * G, (g + 1) * G):
                    out[t, h], lse[t, h], spread[t, h] = attend(q[t, h], k[:seen], v[:seen], scale)
    return out, lse, spread


def decode_shared(q, k_cache, v_cache, prefix_table, prefix_lens, group_rows, table, ctx, scale):
    """(out [B, Hq, D], lse [B, Hq], spread [B, Hq, D])."""
    B, Hq, D = q.shape
    G = Hq // k_cache.shape[1]
    out, lse, spread = np.zeros((B, Hq, D)), np.zeros((B, Hq)), np.zeros((B, Hq, D))
    for b in range(B):
        of = [i for i in range(len(prefix_lens)) if group_rows[i] <= b < group_rows[i + 1]]
        for g in range(k_cache.shape[1]):
            k, v = (np.concatenate(
                [positions(c, prefix_table[i], int(prefix_lens[i]), g) for i in of]
                + [positions(c, table[b], int(ctx[b]), g)]) for c in (k_cache, v_cache))
            for h in range(g * G, (g + 1) * G):
                out[b, h], lse[b, h], spread[b, h] = attend(q[b, h], k, v, scale)
    return out, lse, spread
