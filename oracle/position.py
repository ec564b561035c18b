"""Oracle for the position operators of attention (test infrastructure only): the
norm of queries and keys for each head with the position rotation, attention with a
learned relative position bias by buckets, and their gradients.

All arithmetic is float64, written from the formulas below.

Norm and rotation, u one head of one token, width d:
    n = g * u / sqrt(mean(u^2) + eps),
    pairs (a, b) of the first rot elements:  y_a = n_a c - n_b s, y_b = n_b c + n_a s.
Attention, query i at position i + q_pos, key j:
    z_ij = scale q_i.k_j + bias[bucket[clamp(j - i - q_pos, -M, M) + M]][h],
    over keys j < kv_len, with `causal` also j <= i + q_pos; a bias of -1e30 or less
    takes its keys out; a bucket outside the table adds 0.  Rows without keys give
    o = 0 and lse = -inf.

Pinned by: the norm's unit mean square and its invariance to scale, the rotation's
preserved pair lengths and its dependence on position differences only, position 0
as the identity; zero bias as plain attention, a bias that selects one distance, a
shift of the whole table, explicit loops; every gradient against central finite
differences.
"""
from __future__ import annotations

import math

import numpy as np

MASKED = -1e30


def pairs(rot: int, interleaved: bool):
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def _table(cos, sin, pos, B, L):
    rows = np.broadcast_to(np.arange(L), (B, L)) if pos is None else np.asarray(pos)
    out = []
    for t in (cos, sin):
        t = np.asarray(t, np.float64)
        got = np.full((B, L, t.shape[1]), np.nan)
        ok = (rows >= 0) & (rows < t.shape[0])
        got[ok] = t[rows[ok]]
        out.append(got[:, None, :, None, :])
    return out


def _heads(x, heads):
    x = np.asarray(x, np.float64)
    B, X, L, C = x.shape
    return x.reshape(B, X, L, heads, C // heads)


def rotate(n, cos, sin, pos, interleaved):
    """n [B, X, L, heads, d] turned by the angles of its positions."""
    if cos is None:
        return n
    c, s = _table(cos, sin, pos, n.shape[0], n.shape[2])
    ia, ib = pairs(2 * np.asarray(cos).shape[1], interleaved)
    y = n.copy()
    y[..., ia] = n[..., ia] * c - n[..., ib] * s
    y[..., ib] = n[..., ib] * c + n[..., ia] * s
    return y


def qk_norm_rope(x, heads, g=None, cos=None, sin=None, pos=None, interleaved=False, eps=1e-6):
    u = _heads(x, heads)
    n = u / np.sqrt((u ** 2).mean(-1, keepdims=True) + eps)
    if g is not None:
        n = n * np.asarray(g, np.float64)
    return rotate(n, cos, sin, pos, interleaved).reshape(np.shape(x))


def qk_norm_rope_bwd(x, dy, heads, g=None, cos=None, sin=None, pos=None, interleaved=False, eps=1e-6):
    """(dx, dg)."""
    u, d = _heads(x, heads), _heads(dy, heads)
    dn = rotate(d, cos, None if sin is None else -np.asarray(sin, np.float64), pos, interleaved)
    r = 1.0 / np.sqrt((u ** 2).mean(-1, keepdims=True) + eps)
    dg = (dn * u * r).sum((0, 1, 2, 3))
    w = dn if g is None else dn * np.asarray(g, np.float64)
    dx = r * w - u * r ** 3 * (w * u).mean(-1, keepdims=True)
    return dx.reshape(np.shape(x)), dg


def relpos_buckets(max_dist: int, n_buckets: int, bidirectional: bool) -> np.ndarray:
    """The bucket of each distance key - query in -max_dist .. max_dist: half of the
    buckets of a direction one per distance, the others evenly in its logarithm up
    to max_dist.  Forward distances take the second half of the table when
    bidirectional, and otherwise the bucket of distance 0."""
    out = []
    half = n_buckets // 2 if bidirectional else n_buckets
    near = half // 2
    for d in range(-max_dist, max_dist + 1):
        base = half if bidirectional and d > 0 else 0
        n = abs(d) if bidirectional else max(-d, 0)
        if n >= near:
            # the largest step t with near * (max_dist / near)^(t / (half - near)) <= n
            t = 0
            while t + 1 < half - near and (n / near) ** (half - near) >= (max_dist / near) ** (t + 1) * (1 - 1e-12):
                t += 1
            n = near + t
        out.append(base + n)
    return np.asarray(out, np.int32)


def _scores(q, k, bias, buckets, b, h, grp, causal, q_pos, kv_len, scale):
    """z of (b, all x, h) [X, Lq, n] over the n keys inside the length, -inf where masked."""
    Lq, Lk = q.shape[2], k.shape[2]
    n = Lk if kv_len is None else int(min(max(kv_len[b], 0), Lk))
    first = 0 if q_pos is None else int(q_pos[b])
    M = (len(buckets) - 1) // 2
    dist = np.arange(n)[None, :] - np.arange(Lq)[:, None] - first
    which = np.asarray(buckets)[np.clip(dist, -M, M) + M]
    known = (which >= 0) & (which < len(bias))
    add = np.where(known, np.asarray(bias, np.float64)[np.where(known, which, 0), h], 0.0)
    hide = add <= MASKED
    if causal:
        hide = hide | (dist > 0)
    z = np.matmul(q[b, :, :, h], np.swapaxes(k[b, :, :n, h // grp], -1, -2)) * scale + np.where(hide, 0.0, add)
    return np.where(hide, -np.inf, z), n, np.where(known, which, -1)


def attention_relpos(q, k, v, H, Hkv, bias, buckets, causal=False, q_pos=None, kv_len=None, scale=None, dout=None):
    """(o, lse [B, X, H, Lq]), and with dout also (dq, dk, dv, dbias)."""
    q, k, v = _heads(q, H), _heads(k, Hkv), _heads(v, Hkv)
    B, X, Lq, _, d = q.shape
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    grp = H // Hkv
    o, lse = np.zeros_like(q), np.full((B, X, H, Lq), -np.inf)
    do = None if dout is None else _heads(dout, H)
    dq, dk, dv, db = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v), np.zeros(np.shape(bias))
    for b in range(B):
        for h in range(H):
            z, n, which = _scores(q, k, bias, buckets, b, h, grp, causal, q_pos, kv_len, scale)
            if n == 0 or Lq == 0:
                continue
            top = z.max(-1, keepdims=True)
            top = np.where(np.isneginf(top), 0.0, top)
            p = np.exp(z - top)
            tot = p.sum(-1, keepdims=True)
            with np.errstate(divide="ignore"):
                lse[b, :, h] = (top + np.log(tot))[..., 0]
            p = p / np.where(tot > 0, tot, 1.0)
            vv = v[b, :, :n, h // grp]
            o[b, :, :, h] = np.matmul(p, vv)
            if do is None:
                continue
            g = do[b, :, :, h]
            dv[b, :, :n, h // grp] += np.matmul(np.swapaxes(p, -1, -2), g)
            dp = np.matmul(g, np.swapaxes(vv, -1, -2))
            dz = p * (dp - (p * dp).sum(-1, keepdims=True))
            dq[b, :, :, h] = scale * np.matmul(dz, k[b, :, :n, h // grp])
            dk[b, :, :n, h // grp] += scale * np.matmul(np.swapaxes(dz, -1, -2), q[b, :, :, h])
            per = dz.sum(0)
            for t in range(len(db)):
                db[t, h] += per[which == t].sum()
    flat = lambda t: t.reshape(*t.shape[:3], -1)  # noqa: E731
    if do is None:
        return flat(o), lse
    return flat(o), lse, flat(dq), flat(dk), flat(dv), db
