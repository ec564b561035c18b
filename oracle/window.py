"""Windowed attention and the paged cache in float64, from their definitions.

A query at position p = i + q_pos[b] sees the keys j < kv_len[b] with j <= p + right
(right < 0: no bound) and with j >= p - left (left < 0: no bound) or j < sinks; o is the
softmax of scale q.k over them times v, 0 with a log-sum-exp of -inf where there are none.

Pages: position j of sequence n is slot j % page of page table[n][j // page]; an entry
outside the cache is no page.  In 8 bits a page holds e4m3 values times a power of two
for each head.  Pins: ``tests/test_window_oracle.py``.
"""
from __future__ import annotations

import math

import numpy as np

from .position import _heads, rotate

LEAST_EXP = -64
E4M3_MAX = 448.0


def visible(Lq, Lk, first, n, left, right, sinks):
    """[Lq, Lk] truth values: first is query 0's position, n the sequence's keys."""
    p = np.arange(Lq)[:, None] + int(first)
    j = np.arange(Lk)[None, :]
    ok = np.broadcast_to(j < n, (Lq, Lk)).copy()
    if right >= 0:
        ok &= j <= p + right
    if left >= 0:
        ok &= (j >= p - left) | (j < sinks)
    return ok


def _softmax(z):
    """(probabilities, log-sum-exp) over the last axis; rows of -inf: 0 and -inf."""
    top = z.max(-1, keepdims=True, initial=-np.inf)
    top = np.where(np.isneginf(top), 0.0, top)
    p = np.exp(z - top)
    tot = p.sum(-1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = (top + np.log(tot))[..., 0]
    return p / np.where(tot > 0, tot, 1.0), lse


def attention_window(q, k, v, H, Hkv, left=-1, right=-1, sinks=0, q_pos=None, kv_len=None, scale=None, dout=None):
    """(o, lse [B, X, H, Lq]), and with dout also (dq, dk, dv)."""
    q, k, v = _heads(q, H), _heads(k, Hkv), _heads(v, Hkv)
    B, X, Lq, _, d = q.shape
    Lk, grp = k.shape[2], H // Hkv
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    o, lse = np.zeros_like(q), np.full((B, X, H, Lq), -np.inf)
    do = None if dout is None else _heads(dout, H)
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for b in range(B):
        n = Lk if kv_len is None else int(min(max(kv_len[b], 0), Lk))
        ok = visible(Lq, Lk, 0 if q_pos is None else q_pos[b], n, left, right, sinks)
        used = ok.any(0)              # what no query sees is not looked at
        for h in range(H):
            kk, vv = (np.where(used[:, None], t[b, :, :, h // grp], 0.0) for t in (k, v))
            z = np.matmul(q[b, :, :, h], np.swapaxes(kk, -1, -2)) * scale
            p, lse[b, :, h] = _softmax(np.where(ok, z, -np.inf))
            o[b, :, :, h] = np.matmul(p, vv)
            if do is None:
                continue
            g = do[b, :, :, h]
            dv[b, :, :, h // grp] += np.matmul(np.swapaxes(p, -1, -2), g)
            dp = np.matmul(g, np.swapaxes(vv, -1, -2))
            dz = p * (dp - (p * dp).sum(-1, keepdims=True))
            dq[b, :, :, h] = scale * np.matmul(dz, kk)
            dk[b, :, :, h // grp] += scale * np.matmul(np.swapaxes(dz, -1, -2), q[b, :, :, h])
    flat = lambda t: t.reshape(*t.shape[:3], -1)  # noqa: E731
    if do is None:
        return flat(o), lse
    return flat(o), lse, flat(dq), flat(dk), flat(dv)


def e4m3(x):
    """The nearest of the values (-1)^s 2^e (1 + m / 8), e from -6 (and the multiples of
    2^-9 below it) to 8, ties to even m; what is not finite is NaN."""
    x = np.asarray(x, np.float64)
    with np.errstate(invalid="ignore", divide="ignore"):
        e = np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6)))
        step = 2.0 ** (np.where(np.isfinite(e), e, 0) - 3)
        return np.where(np.isfinite(x), np.round(x / step) * step, np.nan)


def scale_of(top):
    """The least power of two s >= 2^LEAST_EXP with top <= 448 s."""
    s = 2.0 ** LEAST_EXP
    while s * E4M3_MAX < top:
        s *= 2.0
    return s


def append(x, cache, table, q_start, kv_len, scales=None, cos=None, sin=None, pos=None, interleaved=False,
           round_to=lambda t: t):
    """Writes rows x [T, Hkv, D] into cache [pages, page, Hkv, D] (float64, in place), turned
    where cos is given.  scales [pages, Hkv]: the cache holds e4m3 values over them;
    otherwise values pass through round_to."""
    pages, page = cache.shape[:2]
    for n in range(len(kv_len)):
        a, b = int(q_start[n]), int(q_start[n + 1])
        p0 = int(kv_len[n]) - (b - a)
        fresh = {}
        for t in range(a, b):
            at = p0 + t - a
            if at < 0 or at // page >= table.shape[1]:
                continue
            g = int(table[n][at // page])
            if not 0 <= g < pages:
                continue
            row = turned(x[t:t + 1], [at if pos is None else int(pos[t])], cos, sin, interleaved)[0]
            if scales is None:
                cache[g, at % page] = round_to(row)
            else:
                fresh.setdefault(g, []).append((at % page, row))
        for g, rows in fresh.items():
            first = rows[0][0]
            for h in range(cache.shape[2]):
                mags = [np.abs(r[h][np.isfinite(r[h])]).max(initial=0.0) for _, r in rows]
                s = scale_of(max(mags))
                if first > 0:
                    old = scales[g, h]
                    if old > s:
                        s = old
                    elif old > 0:
                        cache[g, :first, h] = e4m3(cache[g, :first, h] * (old / s))
                scales[g, h] = s
                for slot, r in rows:
                    cache[g, slot, h] = e4m3(r[h] / s)


def turned(x, at, cos, sin, interleaved):
    """Rows x [T, heads, D] turned by the table's rows `at`."""
    x = np.asarray(x, np.float64)
    if cos is None:
        return x.copy()
    u = x.reshape(1, 1, x.shape[0], *x.shape[1:])
    return rotate(u, cos, sin, np.asarray(at)[None], interleaved).reshape(x.shape)


def attention_paged(q, k_cache, v_cache, table, q_start, kv_len, H, left=-1, right=0, sinks=0, scale=None,
                    k_scale=None, v_scale=None, max_q=None):
    """{row: (o [H, D], lse [H])} of the packed rows q [T, H, D] that belong to a sequence."""
    pages, page, Hkv, D = k_cache.shape
    scale = 1.0 / math.sqrt(D) if scale is None else scale
    out = {}
    for n in range(len(kv_len)):
        a, b = int(q_start[n]), int(q_start[n + 1])
        cap = table.shape[1] * page
        held = min(max(int(kv_len[n]), 0), cap)
        ok = visible(b - a, held, int(kv_len[n]) - (b - a), held, left, right, sinks)
        k, v = np.zeros((held, Hkv, D)), np.zeros((held, Hkv, D))
        for j in range(held):
            g = int(table[n][j // page])
            if not 0 <= g < pages:
                ok[:, j] = False
            elif ok[:, j].any():
                k[j] = k_cache[g, j % page] * (1.0 if k_scale is None else k_scale[g][:, None])
                v[j] = v_cache[g, j % page] * (1.0 if v_scale is None else v_scale[g][:, None])
        for i in range(b - a if max_q is None else min(b - a, max_q)):
            o, lse = np.zeros((H, D)), np.full(H, -np.inf)
            for h in range(H):
                z = np.where(ok[i], (k[:, h // (H // Hkv)] @ q[a + i, h]) * scale, -np.inf)
                p, lse[h] = _softmax(z)
                o[h] = p @ v[:, h // (H // Hkv)]
            out[a + i] = (o, lse)
    return out
