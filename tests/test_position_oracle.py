"""Pins of the position oracle (oracle/position.py), on the CPU."""
import math

import numpy as np
import pytest

import oracle
from oracle import position as po


def _rng(seed):
    return np.random.default_rng(seed)


def _table(P, rot):
    ang = np.arange(P)[:, None] * 100.0 ** (-np.arange(rot // 2) * 2 / max(rot, 1))
    return np.cos(ang), np.sin(ang)


@pytest.mark.parametrize("interleaved", [False, True])
def test_norm_and_rotation_identities(interleaved):
    x = _rng(0).standard_normal((2, 3, 5, 4 * 6))
    cos, sin = _table(9, 4)
    n = po.qk_norm_rope(x, 4, eps=0.0).reshape(2, 3, 5, 4, 6)
    assert np.allclose((n ** 2).mean(-1), 1.0)
    assert np.allclose(po.qk_norm_rope(7 * x, 4, eps=0.0), n.reshape(x.shape))
    y = po.qk_norm_rope(x, 4, None, cos, sin, interleaved=interleaved, eps=0.0).reshape(n.shape)
    ia, ib = po.pairs(4, interleaved)
    assert np.allclose(y[..., ia] ** 2 + y[..., ib] ** 2, n[..., ia] ** 2 + n[..., ib] ** 2)
    assert np.array_equal(y[:, :, 0], n[:, :, 0]) and np.array_equal(y[..., 4:], n[..., 4:])
    # q at p, k at p + 3: the product is the same for every p
    q, k = _rng(1).standard_normal((2, 1, 1, 1, 6))
    dots = []
    for p in range(6):
        a, b = (po.qk_norm_rope(t, 1, None, cos, sin, pos=np.array([[at]]), interleaved=interleaved)
                for t, at in ((q, p), (k, p + 3)))
        dots.append((a * b).sum())
    assert np.allclose(dots, dots[0])
    bad = po.qk_norm_rope(x, 4, None, cos, sin, pos=np.full((2, 5), 9), interleaved=interleaved).reshape(n.shape)
    assert np.isnan(bad[..., :4]).all() and np.isfinite(bad[..., 4:]).all()


@pytest.mark.parametrize("interleaved", [False, True])
def test_norm_gradient_differences(interleaved):
    r = _rng(2)
    x, dy, g = r.standard_normal((2, 1, 3, 2 * 6)), r.standard_normal((2, 1, 3, 2 * 6)), r.standard_normal(6)
    cos, sin = _table(3, 4)
    f = lambda x, g: (dy * po.qk_norm_rope(x, 2, g, cos, sin, interleaved=interleaved, eps=1e-3)).sum()
    dx, dg = po.qk_norm_rope_bwd(x, dy, 2, g, cos, sin, interleaved=interleaved, eps=1e-3)
    for t, dt, which in ((x, dx, 0), (g, dg, 1)):
        for at in np.ndindex(t.shape):
            up, dn = t.copy(), t.copy()
            up[at] += 1e-6
            dn[at] -= 1e-6
            num = (f(*(up, g) if which == 0 else (x, up)) - f(*(dn, g) if which == 0 else (x, dn))) / 2e-6
            assert abs(num - dt[at]) < 1e-7 * max(1, abs(num)) + 1e-8


def test_buckets():
    b = po.relpos_buckets(128, 32, True)
    at = lambda d: b[d + 128]
    assert [at(-d) for d in (0, 1, 7, 8, 11, 12, 127, 128)] == [0, 1, 7, 8, 8, 9, 15, 15]
    assert [at(d) for d in (1, 7, 8, 128)] == [17, 23, 24, 31]
    assert at(-16) == 10 and at(-32) == 12 and at(-64) == 14 and at(-63) == 13   # exact powers of the step
    c = po.relpos_buckets(128, 32, False)
    assert c[128:].max() == 0 and c[0] == 31 and c[128 - 15] == 15 and c[128 - 16] == 16
    for bi in (True, False):
        for nb, M in ((4, 8), (15, 40), (33, 200)):
            t = po.relpos_buckets(M, nb, bi)
            assert t.min() == 0 and t.max() < nb and (np.diff(t[:M + 1]) <= 0).all()


def _attn(seed, B=2, X=2, Lq=5, Lk=7, H=4, Hkv=2, d=3, nb=5, M=3):
    r = _rng(seed)
    q, k, v = r.standard_normal((B, X, Lq, H * d)), *r.standard_normal((2, B, X, Lk, Hkv * d))
    return q, k, v, r.standard_normal((nb, H)), r.integers(0, nb, 2 * M + 1).astype(np.int32), r


def test_relpos_zero_bias_is_plain_attention():
    q, k, v, bias, bk, _ = _attn(3)
    o, _ = po.attention_relpos(q, k, v, 4, 2, 0 * bias, bk)
    assert np.allclose(o, oracle.attention_grouped(q, k, v, 4, 2))
    o2, l2 = po.attention_relpos(q, k, v, 4, 2, 0 * bias + 2.5, bk)   # a shift of every score
    assert np.allclose(o, o2)


def test_relpos_selects_a_distance():
    """A large bias at distance -1 alone: row i is v of key i - 1."""
    q, k, v, _, _, _ = _attn(4, Lq=6, Lk=6, H=1, Hkv=1)
    bk = np.array([0, 0, 1, 0, 0, 0, 0], np.int32)
    o, _ = po.attention_relpos(q, k, v, 1, 1, np.array([[0.0], [800.0]]), bk)
    assert np.allclose(o[:, :, 1:], v[:, :, :-1])


@pytest.mark.parametrize("causal", [False, True])
def test_relpos_explicit_loops(causal):
    q, k, v, bias, bk, r = _attn(5)
    bias[1, 2] = -np.inf
    bias[3, 0] = -3e38
    bk[0] = 9                                # outside the table: adds nothing
    qp, kl = np.array([2, -3]), np.array([7, 3])
    o, lse = po.attention_relpos(q, k, v, 4, 2, bias, bk, causal, qp, kl, scale=0.7)
    for b in range(2):
        for x in range(2):
            for h in range(4):
                for i in range(5):
                    w, acc = 0.0, np.zeros(3)
                    for j in range(kl[b]):
                        d = j - (i + qp[b])
                        c = bk[min(max(d, -3), 3) + 3]
                        a = bias[c, h] if c < 5 else 0.0
                        if (causal and d > 0) or a <= -1e30:
                            continue
                        e = math.exp(0.7 * float(q[b, x, i, 3 * h:3 * h + 3] @ k[b, x, j, 3 * (h // 2):3 * (h // 2) + 3]) + a)
                        w, acc = w + e, acc + e * v[b, x, j, 3 * (h // 2):3 * (h // 2) + 3]
                    want = acc / w if w else acc
                    assert np.allclose(o[b, x, i, 3 * h:3 * h + 3], want)
                    assert np.isclose(lse[b, x, h, i], math.log(w)) if w else lse[b, x, h, i] == -np.inf
    assert causal is False or np.isneginf(lse[1]).any()   # rows before the first key


@pytest.mark.parametrize("causal", [False, True])
def test_relpos_gradient_differences(causal):
    q, k, v, bias, bk, r = _attn(6, B=2, X=1, Lq=3, Lk=4, H=2, Hkv=1, d=2, nb=3, M=2)
    do = r.standard_normal(q.shape)
    qp, kl = np.array([0, -1]), np.array([4, 2])
    args = [q, k, v, bias]
    f = lambda a: (do * po.attention_relpos(*a[:3], 2, 1, a[3], bk, causal, qp, kl)[0]).sum()
    _, _, dq, dk, dv, db = po.attention_relpos(*args[:3], 2, 1, bias, bk, causal, qp, kl, dout=do)
    for n, g in enumerate((dq, dk, dv, db)):
        for at in np.ndindex(g.shape):
            two = []
            for e in (1e-6, -1e-6):
                a = [t.copy() for t in args]
                a[n][at] += e
                two.append(f(a))
            num = (two[0] - two[1]) / 2e-6
            assert abs(num - g[at]) < 1e-7
