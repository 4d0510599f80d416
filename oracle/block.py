"""Plain CPU implementation, in 64 bits, of the operators of an attention block over voxels: layer norm, rotary
positions with three axes, attention inside the shapes of a ragged batch, with their gradients.  Written from
the formulas; shares no code with the library.  Test infrastructure only."""
from __future__ import annotations

import numpy as np


def layernorm_fwd(x, r, gamma, beta, eps):
    s = np.asarray(x, np.float64) + (0.0 if r is None else np.asarray(r, np.float64))
    mean = s.mean(1)
    rs = 1.0 / np.sqrt(((s - mean[:, None]) ** 2).mean(1) + eps)
    y = (s - mean[:, None]) * rs[:, None]
    if gamma is not None:
        y = y * np.asarray(gamma, np.float64)
    if beta is not None:
        y = y + np.asarray(beta, np.float64)
    return s, y, np.stack([mean, rs], 1)


def layernorm_bwd(x, stats, gamma, dy, ds):
    x, dy, stats = (np.asarray(a, np.float64) for a in (x, dy, stats))
    rs = stats[:, 1:]
    h = (x - stats[:, :1]) * rs
    w = dy if gamma is None else dy * np.asarray(gamma, np.float64)
    dx = rs * (w - w.mean(1, keepdims=True) - h * (w * h).mean(1, keepdims=True))
    if ds is not None:
        dx = dx + np.asarray(ds, np.float64)
    return dx, (dy * h).sum(0), dy.sum(0)


def rope(x, coords, heads, rot_heads, head_dim, sections, base, scale, inverse=False):
    """x [n][heads * head_dim]"""
    n = x.shape[0]
    z = np.array(x, np.float64).reshape(n, heads, head_dim)
    p = 0
    for axis, count in enumerate(sections):
        for j in range(count):
            t = scale * np.asarray(coords, np.float64)[:, axis] * float(base) ** (-j / count)
            t = -t if inverse else t
            co, si = np.cos(t)[:, None], np.sin(t)[:, None]
            a, b = z[:, :rot_heads, 2 * p].copy(), z[:, :rot_heads, 2 * p + 1].copy()
            z[:, :rot_heads, 2 * p] = a * co - b * si
            z[:, :rot_heads, 2 * p + 1] = a * si + b * co
            p += 1
    return z.reshape(n, heads * head_dim)


def _each(q_offsets, k_offsets, mask, heads_q, heads_kv, head_dim):
    """(rows of queries, seen keys, columns of the query head, columns of the key head) of every shape and head"""
    for b in range(len(q_offsets) - 1):
        rows = np.arange(q_offsets[b], q_offsets[b + 1])
        keys = np.arange(k_offsets[b], k_offsets[b + 1])
        if mask is not None:
            keys = keys[np.asarray(mask)[keys] != 0]
        if rows.size == 0 or keys.size == 0:
            continue
        for h in range(heads_q):
            g = h // (heads_q // heads_kv)
            yield rows, keys, h, slice(h * head_dim, (h + 1) * head_dim), slice(g * head_dim, (g + 1) * head_dim)


def _weights(q, k, scale):
    s = scale * (q @ k.T)
    m = s.max(1, keepdims=True)
    z = np.exp(s - m).sum(1, keepdims=True)
    return np.exp(s - m) / z, (m + np.log(z))[:, 0], s


def attention(q, k, v, q_offsets, k_offsets, mask, heads_q, heads_kv, head_dim, scale, do=None):
    """Results, and for each the sums of absolute values that its rounding errors are proportional to:
    o, lse and, with do, dq, dk, dv; o_abs = sum p |v|, dq_abs = scale sum |dS| |k| etc., and d_abs = |dO| . |o|,
    pk_abs = scale sum p |k|, dk_d = scale sum_i d_abs_i p_ij |q_i| (what an error of D costs); top: the largest
    scale sum |q| |k|."""
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    r = dict(o=np.zeros_like(q), o_abs=np.zeros_like(q), lse=np.full((q.shape[0], heads_q), -np.inf), top=0.0)
    if do is not None:
        do = np.asarray(do, np.float64)
        r.update({n: np.zeros_like(q) for n in ("dq", "dq_abs", "pk_abs", "d_abs")})
        r.update({n: np.zeros_like(k) for n in ("dk", "dk_abs", "dk_d", "dv", "dv_abs")})
    for rows, keys, h, cq, ck in _each(q_offsets, k_offsets, mask, heads_q, heads_kv, head_dim):
        i, j = np.ix_(rows, np.arange(cq.start, cq.stop)), np.ix_(keys, np.arange(ck.start, ck.stop))
        p, lse, s = _weights(q[i], k[j], scale)
        r["top"] = max(r["top"], scale * float((np.abs(q[i]) @ np.abs(k[j]).T).max()))
        o = p @ v[j]
        r["o"][i], r["o_abs"][i], r["lse"][rows, h] = o, p @ np.abs(v[j]), lse
        if do is None:
            continue
        g = do[i]
        dp = g @ v[j].T
        ds = p * (dp - (g * o).sum(1, keepdims=True))
        d_abs = (np.abs(g) * np.abs(o)).sum(1, keepdims=True)
        e_abs = p * (np.abs(g) @ np.abs(v[j]).T + d_abs)
        r["dq"][i], r["dq_abs"][i] = scale * ds @ k[j], scale * e_abs @ np.abs(k[j])
        r["pk_abs"][i], r["d_abs"][i] = scale * p @ np.abs(k[j]), d_abs
        r["dk"][j] += scale * ds.T @ q[i]
        r["dk_abs"][j] += scale * e_abs.T @ np.abs(q[i])
        r["dk_d"][j] += scale * (d_abs * p).T @ np.abs(q[i])
        r["dv"][j] += p.T @ g
        r["dv_abs"][j] += p.T @ np.abs(g)
    return r
