"""Results and tolerances for attention with a relative position bias, from
oracle/position.py's definitions in 64 bits.

With u half a step of the type (bf16 2^-8, fp32 2^-24):
 * a score is an fp32 sum of D products, a scaling and a bias: off by at most
   eta = (D + 16) 2^-24 (1 + S), S the largest sum of magnitudes in it, and so are
   the exponent and, relative, each probability and the row's sum;
 * the probabilities enter P v rounded once (u), o is rounded once:
       |do| <= (u + 3 eta) sum_j P |v| + u |o|;
 * Delta is taken from the rounded o: off by dD = sum_d |dO| |do|, plus eta of its
   terms; dZ = P (dP - Delta) is rounded once (u) for dq and dk, not for dbias:
       |d(dZ)| <= (u + 4 eta) P (|dO| |v| + |Delta|) + P dD;
 * in dbias the roundings (u) of different rows, keys and columns are independent, so
   there they count as a root of squares, six times over: a row's Delta is off by
   u sqrt(sum_j (P dP)^2 + sum_d (dO o)^2), and a bucket weighs a row by its share of P;
 * sums over N terms add at most N 2^-24 of the terms' magnitudes.
"""
import numpy as np

import synth
from oracle import position as po


def draw(shape, dtype, rng, scale=1.0):
    a = (rng.standard_normal(shape) * scale).astype(np.float32)
    return synth.bf16_round(a) if dtype == "bf16" else a


def case(B, X, Lq, Lk, H, Hkv, D, M, nb, dtype, seed=0, bias_scale=1.0):
    r = np.random.default_rng(seed)
    q = draw((B, X, Lq, H * D), dtype, r)
    k, v = (draw((B, X, Lk, Hkv * D), dtype, r) for _ in range(2))
    return dict(q=q, k=k, v=v, do=draw(q.shape, dtype, r), bias=draw((nb, H), dtype, r, bias_scale),
                buckets=r.integers(0, nb, 2 * M + 1).astype(np.int32), H=H, Hkv=Hkv)


def wanted(c, dtype, causal=False, q_pos=None, kv_len=None, scale=None, grads=True):
    """{name: (value, tolerance)} of o, lse and the gradients."""
    H, Hkv = c["H"], c["Hkv"]
    q, k, v, do = (po._heads(c[n], h) for n, h in (("q", H), ("k", Hkv), ("v", Hkv), ("do", H)))
    B, X, Lq, _, D = q.shape
    Lk = k.shape[2]
    scale = D ** -0.5 if scale is None else scale
    grp, u = H // Hkv, 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    n24 = 2.0 ** -24
    got = po.attention_relpos(c["q"], c["k"], c["v"], H, Hkv, c["bias"], c["buckets"], causal, q_pos, kv_len, scale,
                              c["do"] if grads else None)
    names = ["o", "lse", "dq", "dk", "dv", "dbias"][:len(got)]
    tol = {n: np.zeros_like(g) for n, g in zip(names, got)}
    val = dict(zip(names, got))
    hd = lambda t, h: t.reshape(*t.shape[:3], h, D)  # noqa: E731
    known = np.abs(np.where(np.asarray(c["bias"], np.float64) <= po.MASKED, 0.0, c["bias"]))
    var = np.zeros(np.shape(c["bias"]))
    for b in range(B):
        for h in range(H):
            z, n, which = po._scores(q, k, c["bias"], c["buckets"], b, h, grp, causal, q_pos, kv_len, scale)
            if n == 0 or Lq == 0:
                continue
            kk, vv, qq, g = k[b, :, :n, h // grp], v[b, :, :n, h // grp], q[b, :, :, h], do[b, :, :, h]
            S = float((np.abs(qq) @ np.abs(kk).swapaxes(-1, -2)).max() * scale + known.max())
            eta = (D + 16) * n24 * (1 + S) + n * n24
            lse = val["lse"][b, :, h]
            p = np.where(np.isneginf(lse)[..., None], 0.0, np.exp(z - np.where(np.isneginf(lse), 0.0, lse)[..., None]))
            o = hd(val["o"], H)[b, :, :, h]
            t_o = (u + 3 * eta) * (p @ np.abs(vv)) + u * np.abs(o)
            hd(tol["o"], H)[b, :, :, h] = t_o
            tol["lse"][b, :, h] = eta * 2 + 2.0 ** -22 * np.abs(np.where(np.isneginf(lse), 0.0, lse))
            if not grads:
                continue
            dp = g @ vv.swapaxes(-1, -2)
            dl = (p * dp).sum(-1, keepdims=True)
            dd = (np.abs(g) * t_o).sum(-1, keepdims=True) + D * n24 * (np.abs(g) * np.abs(o)).sum(-1, keepdims=True)
            mag = p * (np.abs(g) @ np.abs(vv).swapaxes(-1, -2) + np.abs(dl))
            e_sum = p * dd + 4 * eta * mag            # what dbias sums
            e_dz = e_sum + u * np.abs(p * (dp - dl)) * (1 + u)
            add = 2.0 ** -22 + max(n, Lq) * n24       # the accumulation
            tq = scale * ((e_dz + add * mag) @ np.abs(kk)) + u * np.abs(hd(val["dq"], H)[b, :, :, h])
            hd(tol["dq"], H)[b, :, :, h] = tq
            hd(tol["dk"], Hkv)[b, :, :n, h // grp] += scale * ((e_dz + add * mag).swapaxes(-1, -2) @ np.abs(qq))
            hd(tol["dv"], Hkv)[b, :, :n, h // grp] += ((u + 3 * eta + add) * p).swapaxes(-1, -2) @ np.abs(g)
            per = ((4 * eta + add + X * B * n24) * mag).sum(0)
            sd = u * np.sqrt(((p * dp) ** 2).sum(-1) + ((g * o) ** 2).sum(-1))      # [X, Lq]
            for t in range(len(c["bias"])):
                tol["dbias"][t, h] += per[which == t].sum()
                var[t, h] += (((p * (which == t)).sum(-1) * sd) ** 2).sum()
    if grads:
        tol["dbias"] += 6 * np.sqrt(var)
        for n in ("dk", "dv", "dbias"):
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
