"""Results and tolerances for windowed attention and attention over pages, from
oracle/window.py's definitions in 64 bits.

With u half a step of the type (bf16 2^-8, fp32 2^-24):
 * a score is an fp32 sum of D products and a scaling: off by at most
   eta = (D + 16) 2^-24 (1 + S), S the largest sum of magnitudes in it, and so are the
   exponent and, relative, each probability and the row's sum;
 * the probabilities enter P v rounded once (u), o is rounded once:
       |do| <= (u + 3 eta) sum_j P |v| + u |o|;
 * Delta is taken from the rounded o: off by dD = sum_d |dO| |do|, plus eta of its terms;
   dZ = P (dP - Delta) is rounded once (u) for dq and dk:
       |d(dZ)| <= (u + 4 eta) P (|dO| |v| + |Delta|) + P dD;
 * sums over N terms add at most N 2^-24 of the terms' magnitudes.
"""
import numpy as np

import synth
from oracle import window as ow

N24 = 2.0 ** -24


def draw(shape, dtype, rng, scale=1.0):
    a = (rng.standard_normal(shape) * scale).astype(np.float32)
    return synth.bf16_round(a) if dtype == "bf16" else a


def case(B, X, Lq, Lk, H, Hkv, D, dtype, seed=0):
    r = np.random.default_rng(seed)
    q = draw((B, X, Lq, H * D), dtype, r)
    k, v = (draw((B, X, Lk, Hkv * D), dtype, r) for _ in range(2))
    return dict(q=q, k=k, v=v, do=draw(q.shape, dtype, r), H=H, Hkv=Hkv)


def row_bounds(q, k, v, p, o, lse, scale, u):
    """(bound of o, bound of lse, eta) of rows q [.., Lq, D] over the n keys k, v [.., n, D]."""
    n, D = k.shape[-2], k.shape[-1]
    S = float((np.abs(q) @ np.abs(k).swapaxes(-1, -2)).max(initial=0.0) * scale)
    eta = (D + 16) * N24 * (1 + S) + n * N24
    t_o = (u + 3 * eta) * (p @ np.abs(v)) + u * np.abs(o)
    return t_o, eta * 2 + 2.0 ** -22 * np.abs(np.where(np.isneginf(lse), 0.0, lse)), eta


def wanted(c, dtype, left=-1, right=-1, sinks=0, q_pos=None, kv_len=None, scale=None, grads=True):
    """{name: (value, tolerance)} of o, lse and the gradients."""
    H, Hkv = c["H"], c["Hkv"]
    q, k, v, do = (ow._heads(c[n], h) for n, h in (("q", H), ("k", Hkv), ("v", Hkv), ("do", H)))
    B, X, Lq, _, D = q.shape
    Lk, grp = k.shape[2], H // Hkv
    scale = D ** -0.5 if scale is None else scale
    u = 2.0 ** -8 if dtype == "bf16" else N24
    got = ow.attention_window(c["q"], c["k"], c["v"], H, Hkv, left, right, sinks, q_pos, kv_len, scale,
                              c["do"] if grads else None)
    names = ["o", "lse", "dq", "dk", "dv"][:len(got)]
    val, tol = dict(zip(names, got)), {n: np.zeros_like(g) for n, g in zip(names, got)}
    hd = lambda t, h: t.reshape(*t.shape[:3], h, D)  # noqa: E731
    for b in range(B):
        n = Lk if kv_len is None else int(min(max(kv_len[b], 0), Lk))
        ok = ow.visible(Lq, Lk, 0 if q_pos is None else q_pos[b], n, left, right, sinks)
        used = ok.any(0)[:, None]
        for h in range(H):
            qq, g = q[b, :, :, h], do[b, :, :, h]
            kk, vv = (np.where(used, t[b, :, :, h // grp], 0.0) for t in (k, v))
            lse = val["lse"][b, :, h]
            z = np.where(ok, qq @ kk.swapaxes(-1, -2) * scale, -np.inf)
            p = np.where(np.isneginf(lse)[..., None], 0.0, np.exp(z - np.where(np.isneginf(lse), 0.0, lse)[..., None]))
            o = hd(val["o"], H)[b, :, :, h]
            t_o, t_lse, eta = row_bounds(qq, kk, vv, p, o, lse, scale, u)
            hd(tol["o"], H)[b, :, :, h] = t_o
            tol["lse"][b, :, h] = t_lse
            if not grads:
                continue
            dp = g @ vv.swapaxes(-1, -2)
            dl = (p * dp).sum(-1, keepdims=True)
            dd = (np.abs(g) * t_o).sum(-1, keepdims=True) + D * N24 * (np.abs(g) * np.abs(o)).sum(-1, keepdims=True)
            mag = p * (np.abs(g) @ np.abs(vv).swapaxes(-1, -2) + np.abs(dl))
            e_dz = p * dd + 4 * eta * mag + u * np.abs(p * (dp - dl)) * (1 + u)
            add = 2.0 ** -22 + max(n, Lq) * N24       # the accumulation
            hd(tol["dq"], H)[b, :, :, h] = scale * ((e_dz + add * mag) @ np.abs(kk)) + u * np.abs(hd(val["dq"], H)[b, :, :, h])
            hd(tol["dk"], Hkv)[b, :, :, h // grp] += scale * ((e_dz + add * mag).swapaxes(-1, -2) @ np.abs(qq))
            hd(tol["dv"], Hkv)[b, :, :, h // grp] += ((u + 3 * eta + add) * p).swapaxes(-1, -2) @ np.abs(g)
    for n in ("dk", "dv") if grads else ():
        tol[n] += u * np.abs(val[n])
    return {n: (val[n], tol[n]) for n in names}


def compare(got, want, say=print):
    """Every element of every output within its tolerance; infinities in the same places."""
    for name, (val, tol) in want.items():
        g = np.asarray(got[name], np.float64).reshape(val.shape)
        same_inf = np.isinf(val) & (g == val)
        assert np.array_equal(np.isinf(val), same_inf), f"{name}: infinities"
        ok = ~np.isinf(val)
        assert np.isfinite(g[ok]).all(), f"{name}: not finite"
        err = np.abs(g[ok] - val[ok]) / (tol[ok] + 1e-30 + 2.0 ** -40 * np.abs(val[ok]).max(initial=0))
        worst = float(err.max(initial=0.0))
        say(f"  {name}: {worst:.3f} of its tolerance")
        assert worst <= 1.0, name
