"""Pins of the window and page oracle (oracle/window.py), on the CPU."""
import math

import numpy as np
import pytest

from oracle import position as po
from oracle import window as ow


def _rng(seed):
    return np.random.default_rng(seed)


def _qkv(seed=0, B=2, X=1, Lq=6, Lk=9, H=4, Hkv=2, D=3):
    r = _rng(seed)
    return r.standard_normal((B, X, Lq, H * D)), *(r.standard_normal((B, X, Lk, Hkv * D)) for _ in range(2))


def test_without_bounds_it_is_attention_with_no_bias():
    q, k, v = _qkv()
    o, lse = ow.attention_window(q, k, v, 4, 2, kv_len=[9, 4])
    w = po.attention_relpos(q, k, v, 4, 2, np.zeros((1, 4)), np.zeros(1, np.int32), kv_len=[9, 4])
    assert np.allclose(o, w[0]) and np.allclose(lse, w[1])
    o, lse = ow.attention_window(q, k, v, 4, 2, right=0, q_pos=[3, -2])
    w = po.attention_relpos(q, k, v, 4, 2, np.zeros((1, 4)), np.zeros(1, np.int32), causal=True, q_pos=[3, -2])
    assert np.allclose(o, w[0]) and np.array_equal(np.isneginf(lse), np.isneginf(w[1]))


@pytest.mark.parametrize("left,right,sinks", [(0, 0, 0), (2, 0, 0), (2, 1, 0), (1, 0, 2), (0, 3, 1), (-1, 2, 3), (3, -1, 2),
                                              (100, 100, 100)])
def test_each_query_by_itself(left, right, sinks):
    q, k, v = _qkv(1)
    pos, lens = [2, 7], [9, 5]
    o, lse = ow.attention_window(q, k, v, 4, 2, left, right, sinks, pos, lens)
    for b in range(2):
        for i in range(6):
            p = i + pos[b]
            see = [j for j in range(lens[b]) if (right < 0 or j <= p + right)
                   and (left < 0 or j >= p - left or j < sinks)]
            for h in range(4):
                sl, kl = slice(3 * h, 3 * h + 3), slice(3 * (h // 2), 3 * (h // 2) + 3)
                w = [math.exp(q[b, 0, i, sl] @ k[b, 0, j, kl] / math.sqrt(3)) for j in see]
                if not see:
                    assert not o[b, 0, i, sl].any() and lse[b, 0, h, i] == -np.inf
                    continue
                want = sum(a * v[b, 0, j, kl] for a, j in zip(w, see)) / math.fsum(w)
                assert np.allclose(o[b, 0, i, sl], want) and math.isclose(lse[b, 0, h, i], math.log(math.fsum(w)))


def test_gradient_differences():
    q, k, v = _qkv(2, B=1, Lq=5, Lk=6)
    do = _rng(3).standard_normal(q.shape)
    kw = dict(left=1, right=1, sinks=1, kv_len=[5], q_pos=[1])
    f = lambda q, k, v: (do * ow.attention_window(q, k, v, 4, 2, **kw)[0]).sum()  # noqa: E731
    grads = ow.attention_window(q, k, v, 4, 2, dout=do, **kw)[2:]
    for which, (t, g) in enumerate(zip((q, k, v), grads)):
        for at in np.ndindex(t.shape):
            ab = []
            for step in (1e-6, -1e-6):
                args = [q, k, v]
                args[which] = t.copy()
                args[which][at] += step
                ab.append(f(*args))
            assert abs((ab[0] - ab[1]) / 2e-6 - g[at]) < 1e-7


def test_e4m3_values():
    codes = [s * (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
             for s in (1, -1) for e in range(16) for m in range(8) if (e, m) != (15, 7)]
    assert max(codes) == 448 and np.array_equal(ow.e4m3(codes), codes)
    grid = np.unique(codes)
    x = _rng(4).uniform(-448, 448, 2000) * 2.0 ** -_rng(5).integers(0, 14, 2000)
    near = grid[np.abs(grid[None] - x[:, None]).argmin(1)]
    assert np.array_equal(np.abs(ow.e4m3(x) - x), np.abs(near - x))
    assert ow.e4m3(17.0) == 16 and ow.e4m3(19.0) == 20 and np.isnan(ow.e4m3(np.inf)) and np.isnan(ow.e4m3(np.nan))
    torch = pytest.importorskip("torch")
    t = torch.from_numpy(x.astype(np.float32))
    assert np.array_equal(t.to(torch.float8_e4m3fn).float().numpy(), ow.e4m3(t.numpy()))


def test_scales():
    assert ow.scale_of(0.0) == 2.0 ** -64 and ow.scale_of(448.0) == 1 and ow.scale_of(448.1) == 2
    assert ow.scale_of(7.0) == 2.0 ** -6 and ow.scale_of(7.1) == 2.0 ** -5


def test_paged_attention_is_windowed_attention():
    r = _rng(6)
    H, Hkv, D, page, lens, new = 4, 2, 8, 4, [11, 6, 3], [3, 6, 0]
    table = np.array([[5, 0, 3], [2, 6, -1], [1, -1, 9]])
    kc, vc = (r.standard_normal((7, page, Hkv, D)) for _ in range(2))
    start = np.concatenate([[0], np.cumsum(new)])
    q = r.standard_normal((start[-1], H, D))
    got = ow.attention_paged(q, kc, vc, table, start, lens, H, 3, 0, 2)
    assert sorted(got) == list(range(9))
    for n in range(2):
        k, v = (c[[table[n][j // page] for j in range(lens[n])], [j % page for j in range(lens[n])]] for c in (kc, vc))
        o, lse = ow.attention_window(q[start[n]:start[n + 1]].reshape(1, 1, new[n], -1), k.reshape(1, 1, lens[n], -1),
                                     v.reshape(1, 1, lens[n], -1), H, Hkv, 3, 0, 2, [lens[n] - new[n]])
        for i in range(new[n]):
            assert np.allclose(got[start[n] + i][0].reshape(-1), o[0, 0, i])
            assert np.allclose(got[start[n] + i][1], lse[0, 0, :, i])
    # a missing page takes its keys out
    got = ow.attention_paged(q, kc, vc, np.array([[5, -1, 3]]), [0, 1], [11], H)
    keep = [0, 1, 2, 3, 8, 9, 10]
    k, v = (c[[5] * 4 + [3] * 3, [0, 1, 2, 3, 0, 1, 2]] for c in (kc, vc))
    o, _ = ow.attention_window(q[:1].reshape(1, 1, 1, -1), k.reshape(1, 1, 7, -1), v.reshape(1, 1, 7, -1), H, Hkv)
    assert len(keep) == 7 and np.allclose(got[0][0].reshape(-1), o[0, 0, 0])


def test_append_then_read():
    """What was appended, in chunks of any size, is found at its position, turned by it;
    8-bit pages hold every token to half a step of the largest one's scale."""
    r = _rng(7)
    page, Hkv, D, L = 4, 2, 4, 11
    x = r.standard_normal((L, Hkv, D)) * np.exp(r.uniform(-3, 3, (L, 1, 1)))
    ang = np.arange(L)[:, None] * np.array([1.0, 0.1])
    cos, sin = np.cos(ang), np.sin(ang)
    want = ow.turned(x, np.arange(L), cos, sin, False)
    table = np.array([[3, 1, 4]])
    for bits8 in (False, True):
        for cuts in ([L], [1] * L, [3, 5, 3]):
            cache, scales = r.standard_normal((5, page, Hkv, D)), np.full((5, Hkv), 2.0) if bits8 else None
            at = 0
            for n in cuts:
                ow.append(x[at:at + n], cache, table, [0, n], [at + n], scales, cos, sin)
                at += n
            got = np.stack([cache[table[0][j // page], j % page] for j in range(L)])
            if not bits8:
                assert np.allclose(got, want)
                continue
            s = np.stack([scales[table[0][j // page]] for j in range(L)])[..., None]
            top = np.stack([np.abs(want[j // page * page:j // page * page + page]).max((0, 2)) for j in range(L)])
            assert (top <= 448 * s[..., 0]).all() and (top > 224 * s[..., 0]).all()
            # one rounding, and one more for each time that the scale grew (a lost bit near 0)
            assert (np.abs(got * s - want) <= 2.0 ** -4 * np.abs(want) + 4 * 2.0 ** -10 * s).all()
    assert np.array_equal(want, ow.turned(x, np.arange(L), cos, sin, False))


def test_append_drops_what_has_no_place():
    cache = np.zeros((2, 4, 1, 2))
    ow.append(np.ones((6, 1, 2)), cache, np.array([[1, 7]]), [0, 6], [6])
    assert cache[1].all() and not cache[0].any()
    ow.append(np.full((3, 1, 2), 5.0), cache, np.array([[0]]), [0, 3], [2])    # positions -1, 0, 1
    assert (cache[0, :2] == 5).all() and not cache[0, 2:].any()
