"""Attention with a relative position bias where the choice of kernel, the positions and
the precision of the gradients can go wrong: work-groups of 128 keys in the gradient of
dK and dV, positions at the ends of 32 bits, gradients to the roundings that they make.

Tolerances of dq and dk beyond tests/relpos_util.py, whose notation this follows.  Delta is
a sum in 32 bits, from P and dP or, in fp32, from an o of that precision:
 * P is off by e_p = 3 eta + 2^-22 (1 + |lse|), relative: its exponent by eta, the row's
   log-sum-exp by 2 eta and its own rounding, the exponential by 2^-22;
 * with a = |dO| |v|, dP is off by eta a, Delta by (e_p + 2 eta) sum_j P a, so dZ before
   its rounding by e = P (eta a + that) + e_p |dZ|;
 * dZ is rounded once (u) as an operand, sums add 2^-22 + N 2^-24 of the magnitudes
   P (a + |Delta|), the results are rounded once."""
import numpy as np
import pytest

from oracle import position as po
from tests import relpos_util as ru
from tests.gpu_util import host, say
from tests.test_gpu_attn_relpos import CASES, _check, _run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


def _tight(c, dtype, causal, q_pos, kv_len):
    """{dq, dk: (value, tolerance)}."""
    H, Hkv = c["H"], c["Hkv"]
    _, lse, dq, dk, *_ = po.attention_relpos(c["q"], c["k"], c["v"], H, Hkv, c["bias"], c["buckets"], causal, q_pos,
                                             kv_len, None, c["do"])
    q, k, v, do = (po._heads(c[n], h) for n, h in (("q", H), ("k", Hkv), ("v", Hkv), ("do", H)))
    B, X, Lq, _, D = q.shape
    scale, grp = D ** -0.5, H // Hkv
    u, n24 = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24, 2.0 ** -24
    tq, tk = u * np.abs(dq).reshape(q.shape), u * np.abs(dk).reshape(k.shape)
    known = np.abs(c["bias"]).max()
    for b in range(B):
        for h in range(H):
            z, n, _ = po._scores(q, k, c["bias"], c["buckets"], b, h, grp, causal, q_pos, kv_len, scale)
            if n == 0 or Lq == 0:
                continue
            kk, vv, qq, g = k[b, :, :n, h // grp], v[b, :, :n, h // grp], q[b, :, :, h], do[b, :, :, h]
            S = float((np.abs(qq) @ np.abs(kk).swapaxes(-1, -2)).max() * scale + known)
            eta = (D + 16) * n24 * (1 + S) + n * n24
            row = np.where(np.isneginf(lse[b, :, h]), 0.0, lse[b, :, h])[..., None]
            p = np.exp(z - row)
            e_p = 3 * eta + 2.0 ** -22 * (1 + np.abs(row))
            a = np.abs(g) @ np.abs(vv).swapaxes(-1, -2)
            dp = g @ vv.swapaxes(-1, -2)
            delta = (p * dp).sum(-1, keepdims=True)
            dz = np.abs(p * (dp - delta))
            e = p * (eta * a + (e_p + 2 * eta) * (p * a).sum(-1, keepdims=True)) + (e_p + u) * dz
            e = e + (2.0 ** -22 + max(n, Lq) * grp * n24) * p * (a + np.abs(delta))
            tq[b, :, :, h] += scale * (e @ np.abs(kk))
            tk[b, :, :n, h // grp] += scale * (e.swapaxes(-1, -2) @ np.abs(qq))
    return dict(dq=(dq, tq.reshape(dq.shape)), dk=(dk, tk.reshape(dk.shape)))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,X,Lq,Lk,H,Hkv,D,M,nb,causal,q_pos,kv_len", CASES)
def test_gradients_to_their_roundings(torch, dtype, B, X, Lq, Lk, H, Hkv, D, M, nb, causal, q_pos, kv_len):
    c = ru.case(B, X, Lq, Lk, H, Hkv, D, M, nb, dtype, seed=Lq + D)
    say("relpos tight", dtype, B, X, Lq, Lk, H, Hkv, D)
    got = _run(torch, c, dtype, causal=causal, q_pos=q_pos, kv_len=kv_len)
    ru.compare({n: host(t) for n, t in got.items()}, _tight(c, dtype, causal, q_pos, kv_len), say)


@pytest.mark.parametrize("X,Lq,Lk,H,Hkv,D,causal,lens", [
    (70, 150, 200, 4, 2, 64, False, False),    # 140 and 280 work-groups of 256 and 128 keys; 256 fill the chip
    (70, 150, 200, 4, 2, 72, False, False),
    (140, 33, 130, 3, 1, 40, False, False),
    (75, 260, 256, 2, 2, 24, False, False),
    (150, 150, 200, 4, 2, 64, True, False),    # causal or ragged: twice as many, 300 and 600
    (75, 129, 220, 4, 2, 72, False, True),
    (75, 300, 200, 8, 2, 40, True, True),
])
def test_work_groups_of_128_keys(torch, X, Lq, Lk, H, Hkv, D, causal, lens):
    B = 2 if lens else 1
    c = ru.case(B, X, Lq, Lk, H, Hkv, D, 30, 12, "bf16", seed=D + X)
    kw = dict(causal=causal, kv_len=[Lk, Lk - 61] if lens else None, q_pos=[Lk - Lq] * B if causal else None)
    got = _check(torch, c, "bf16", f"relpos X{X} {Lq}x{Lk} H{H}/{Hkv} D{D}", **kw)
    ru.compare({n: host(t) for n, t in got.items()}, _tight(c, "bf16", causal, kw["q_pos"], kw["kv_len"]), say)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Lq,Lk,H,Hkv,D", [(20, 40, 2, 2, 64), (70, 90, 4, 2, 72), (1, 600, 4, 2, 40), (150, 300, 2, 2, 24),
                                           (40, 40, 2, 1, 80)])
def test_positions_at_the_ends_of_32_bits(torch, dtype, Lq, Lk, H, Hkv, D):
    """Every key far before the queries of one sequence (causal masks none), far after
    those of another (they mask all)."""
    c = ru.case(3, 2, Lq, Lk, H, Hkv, D, 10, 4, dtype, seed=Lq)
    for causal in (True, False):
        for kv_len in (None, [Lk, Lk - 3, 5]):
            got = _check(torch, c, dtype, f"positions {Lq}x{Lk}", causal=causal, kv_len=kv_len,
                         q_pos=[-2 ** 31, 2 ** 31 - 1, 0])
            if causal:
                assert not any(got[n][0].any() for n in ("o", "dq", "dk", "dv")) and got["lse"][0].isneginf().all()


@pytest.mark.parametrize("X,L,Lk,H,Hkv,D,M,causal", [
    (200, 49, 49, 4, 4, 72, 16, False),        # short units, their own keys and shared ones
    (200, 49, 49, 8, 2, 64, 16, True),
    (4, 384, 384, 4, 4, 64, 16, True),
    (4, 384, 384, 4, 2, 72, 16, True),
    (4, 384, 384, 4, 4, 128, 16, True),
    (4, 700, 116, 4, 4, 72, 200, False),
])
def test_the_bias_gradient_is_rounded_once(torch, X, L, Lk, H, Hkv, D, M, causal):
    """Rows of dZ add up to nothing, so the sums of long buckets cancel: in bf16 they carry
    the rounding of the result, at most 2^-8 of it, and errors of 32 bits.  Those are
    independent from term to term as the terms themselves are, and 100 2^-24 of them
    (sums of 128 products and scores up to 30): far below 2^-12."""
    import paper_2403_10266_amd as dsp
    c = ru.case(1, X, L, Lk, H, Hkv, D, M, 8, "bf16", seed=28)
    c["buckets"] = dsp.dsp_relpos_buckets(M, 8, not causal).numpy()
    got = host(_run(torch, c, "bf16", causal=causal)["dbias"])
    want = ru.wanted(c, "bf16", causal)["dbias"][0]
    err = np.linalg.norm(got - want) / np.linalg.norm(want)
    say(f"dbias: {err:.2e}")
    assert err <= 2.0 ** -8 + 2.0 ** -12
