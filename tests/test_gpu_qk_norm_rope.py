"""Norm of queries and keys with the position rotation on the GPU, and its gradient,
against oracle/position.py in 64 bits.

Tolerances: the arithmetic between loads and stores is fp32.  An output is a sum of
a few products, each off by a few roundings of 2^-24 of the row's size A (the
largest normalised element, or for the gradient the largest term), and the sums over
a row add at most D = 256 roundings to the factor r, relative: within 2^-17 A in
all.  bf16 adds the one rounding of the result, at most 2^-8 of it.  A gain's
gradient is a sum of such terms: within 2^-17 of the sum of their magnitudes."""
import numpy as np
import pytest

import synth
from oracle import position as po
from tests.gpu_util import dev, host, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


def _draw(shape, dtype, seed, scale=1.0):
    a = (np.random.default_rng(seed).standard_normal(shape) * scale).astype(np.float32)
    return synth.bf16_round(a) if dtype == "bf16" else a


def _table(P, rot):
    ang = np.arange(P)[:, None] * 1000.0 ** (-np.arange(rot // 2) * 2 / max(rot, 1))
    return np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)


def _within(got, want, size, dtype, what):
    """|got - want| <= 2^-17 size (+ 2^-8 |want| in bf16), element by element."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape and np.isfinite(got).all(), what
    tol = 2.0 ** -17 * size + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0.0) + 1e-30
    worst = float((np.abs(got - want) / tol).max()) if got.size else 0.0
    say(f"  {what}: {worst:.3f} of its tolerance")
    assert worst <= 1.0, what


def _row_size(t, heads):
    """Largest magnitude of each head's row, spread over its elements."""
    B, X, L, C = t.shape
    m = np.abs(t.reshape(B, X, L, heads, -1)).max(-1, keepdims=True)
    return np.broadcast_to(m, (B, X, L, heads, C // heads)).reshape(t.shape)


def _check(torch, dtype, B, X, L, H, Hkv, D, rot, interleaved, pos=None, gain=True, views=None, seed=0, P=None):
    import paper_2403_10266_amd as dsp
    say(f"qk_norm {dtype} B={B} X={X} L={L} H={H} Hkv={Hkv} D={D} rot={rot} adj={interleaved}")
    q, k = _draw((B, X, L, H * D), dtype, seed, 1.5), _draw((B, X, L, Hkv * D), dtype, seed + 1, 0.3)
    dq, dk = _draw(q.shape, dtype, seed + 2), _draw(k.shape, dtype, seed + 3)
    gq, gk = ((1 + _draw((D,), "f32", seed + s, 0.2)) if gain else None for s in (4, 5))
    if gain and dtype == "bf16":
        gq, gk = synth.bf16_round(gq), synth.bf16_round(gk)
    cos, sin = _table(P or max(L, 1), rot) if rot else (None, None)
    put = views or (lambda t, name: dev(t, dtype))
    on = lambda t: None if t is None else torch.from_numpy(t).cuda()
    gain_t = [None if g is None else dev(g, dtype) for g in (gq, gk)]
    kw = dict(pos=on(pos), interleaved=interleaved)
    qt, kt = put(q, "q"), put(k, "k") if Hkv else None
    yq, yk = dsp.dsp_qk_norm_rope(qt, kt, H, Hkv, *gain_t, on(cos), on(sin), **kw)
    g = dsp.dsp_qk_norm_rope_bwd(qt, kt, put(dq, "dq"), put(dk, "dk") if Hkv else None, H, Hkv, *gain_t, on(cos),
                                 on(sin), **kw)
    torch.cuda.synchronize()
    for name, x, dy, heads, gn, y, dx, dg in (("q", q, dq, H, gq, yq, g[0], g[2]), ("k", k, dk, Hkv, gk, yk, g[1], g[3])):
        if not heads:
            assert y is None and dx is None and dg is None
            continue
        want = po.qk_norm_rope(x, heads, gn, cos, sin, pos, interleaved)
        n = po.qk_norm_rope(x, heads, gn)
        _within(host(y), want, _row_size(n, heads), dtype, "y" + name)
        wx, wg = po.qk_norm_rope_bwd(x, dy, heads, gn, cos, sin, pos, interleaved)
        # the gradient's terms: r w, and u r^3 mean(w u), with |w| up to the pair's size
        u = np.asarray(x, np.float64).reshape(B, X, L, heads, D)
        r = 1 / np.sqrt((u ** 2).mean(-1, keepdims=True) + 1e-6)
        w = np.sqrt(2) * np.abs(dy.reshape(u.shape)).max(-1, keepdims=True) * (np.abs(gn).max() if gn is not None else 1)
        size = r * w * (1 + np.abs(u).max(-1, keepdims=True) * r * r * np.abs(u).mean(-1, keepdims=True))
        _within(host(dx), wx, np.broadcast_to(size, u.shape).reshape(x.shape), dtype, "d" + name)
        dn = po.rotate(dy.astype(np.float64).reshape(u.shape), cos, None if sin is None else -sin, pos, interleaved)
        mag = (np.abs(np.sqrt(2) * np.abs(dy.reshape(u.shape)).max(-1, keepdims=True) * u * r)).sum((0, 1, 2, 3))
        _within(host(dg), wg, mag, "f32", "dg" + name)


CASES = [
    # B, X, L, H, Hkv, D, rot, adjacent
    (2, 3, 17, 4, 4, 72, 72, False),
    (1, 5, 33, 16, 16, 72, 72, True),
    (2, 2, 9, 8, 2, 64, 64, False),
    (1, 1, 1, 16, 16, 72, 72, False),        # one token
    (3, 1, 1, 1, 1, 128, 64, True),
    (1, 7, 40, 6, 2, 40, 16, False),         # part of the head turns
    (1, 2, 50, 3, 1, 80, 40, False),         # half of it, in bf16 in runs of 8 bytes
    (1, 2, 13, 5, 5, 96, 0, False),          # no rotation
    (1, 1, 12, 2, 2, 256, 256, False),
    (1, 2, 11, 3, 2, 200, 200, True),
    (1, 2, 21, 2, 1, 44, 22, True),          # pairs that no 16-byte chunk holds
    (1, 2, 21, 2, 1, 44, 22, False),
    (2, 1, 5, 2, 2, 7, 6, False),            # odd width
    (2, 1, 5, 2, 2, 7, 2, True),
    (1, 1, 3, 2, 2, 1, 0, False),            # width 1
    (1, 3, 1000, 2, 1, 16, 16, False),       # many work-groups
    (1, 1, 130, 40, 0, 24, 24, True),        # queries alone
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,X,L,H,Hkv,D,rot,adj", CASES)
def test_against_the_formula(torch, dtype, B, X, L, H, Hkv, D, rot, adj):
    _check(torch, dtype, B, X, L, H, Hkv, D, rot, adj)


def test_many_rows_per_group_of_lanes(torch):
    """More rows than the gradient's work-groups hold in one pass."""
    _check(torch, "bf16", 2, 40, 330, 16, 4, 72, 72, False, seed=3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_positions_of_each_sequence(torch, dtype):
    pos = np.array([[5, 0, 99, 7], [98, 98, 1, 2]], np.int32)
    _check(torch, dtype, 2, 3, 4, 4, 2, 72, 72, False, pos=pos, P=100)
    _check(torch, dtype, 2, 3, 4, 4, 2, 72, 72, True, pos=pos, P=100, gain=False)


@pytest.mark.parametrize("D,rot", [(72, 72), (44, 22)])
def test_position_without_a_row_is_nan(torch, D, rot):
    import paper_2403_10266_amd as dsp
    x = torch.randn(2, 2, 3, 2 * D, device="cuda")
    cos, sin = (torch.from_numpy(t).cuda() for t in _table(10, rot))
    pos = torch.tensor([[0, 10, 2], [-1, 9, 2 ** 31 - 1]], dtype=torch.int32, device="cuda")
    y, _ = dsp.dsp_qk_norm_rope(x, None, 2, 0, cos=cos, sin=sin, pos=pos)
    dx, _, _, _ = dsp.dsp_qk_norm_rope_bwd(x, None, x, None, 2, 0, cos=cos, sin=sin, pos=pos)
    torch.cuda.synchronize()
    bad = torch.tensor([[False, True, False], [True, False, True]], device="cuda")[:, None].expand(2, 2, 3)
    y, dx = y.view(2, 2, 3, 2, D), dx.view(2, 2, 3, 2, D)
    assert y[bad][..., :rot].isnan().all() and not y[bad][..., rot:].isnan().any() and not y[~bad].isnan().any()
    assert dx[bad].isnan().any(-1).all() and not dx[~bad].isnan().any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("off", [0, 1])
def test_packed_and_permuted_views(torch, dtype, off):
    """Columns of a wider buffer, an order of (b, l, x), an offset off 16 bytes."""
    def views(t, name):
        B, X, L, C = t.shape
        wide = torch.zeros(B, L, X, C + 40, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
        v = wide.permute(0, 2, 1, 3)[..., 8 + off:8 + off + C]
        v.copy_(dev(t, dtype))
        return v
    _check(torch, dtype, 2, 3, 19, 4, 2, 72, 72, False, views=views)


@pytest.mark.parametrize("D,rot,adj", [(72, 72, False), (64, 32, True), (44, 22, False)])
def test_in_place_and_packed_columns(torch, D, rot, adj):
    """In place of q and k inside [Q | K | V]: the bits of the call with new outputs,
    V and the padding as they were; the gradient in place of dyq and dyk."""
    import paper_2403_10266_amd as dsp
    H, B, X, L = 4, 2, 3, 21
    qkv = torch.randn(B, X, L, 3 * H * D, device="cuda").bfloat16()
    cos, sin = (torch.from_numpy(t).cuda() for t in _table(L, rot))
    cut = lambda t: (t[..., :H * D], t[..., H * D:2 * H * D])
    q, k = cut(qkv)
    kw = dict(cos=cos, sin=sin, interleaved=adj)
    yq, yk = dsp.dsp_qk_norm_rope(q, k, H, H, **kw)
    dy = torch.randn_like(qkv)
    want = dsp.dsp_qk_norm_rope_bwd(q, k, *cut(dy), H, H, **kw)
    dy2, v0 = dy.clone(), dy[..., 2 * H * D:].clone()
    got = dsp.dsp_qk_norm_rope_bwd(q, k, *cut(dy2), H, H, dq=cut(dy2)[0], dk=cut(dy2)[1], **kw)
    buf = qkv.clone()
    dsp.dsp_qk_norm_rope(*cut(buf), H, H, out_q=cut(buf)[0], out_k=cut(buf)[1], **kw)
    torch.cuda.synchronize()
    assert torch.equal(cut(buf)[0], yq) and torch.equal(cut(buf)[1], yk)
    assert torch.equal(buf[..., 2 * H * D:], qkv[..., 2 * H * D:]) and torch.equal(dy2[..., 2 * H * D:], v0)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_empty(torch):
    import paper_2403_10266_amd as dsp
    e = torch.empty(2, 0, 4, 72, device="cuda")
    yq, yk = dsp.dsp_qk_norm_rope(e, e, 1, 1)
    dq, dk, dgq, dgk = dsp.dsp_qk_norm_rope_bwd(e, e, e, e, 1, 1)
    torch.cuda.synchronize()
    assert yq.shape == e.shape and not dgq.any() and not dgk.any()


def test_graph_replays(torch):
    """The serving step's call in a captured graph: positions move between replays."""
    import paper_2403_10266_amd as dsp
    H, D, P = 16, 72, 50
    q, k = (torch.randn(8, 1, 1, H * D, device="cuda").bfloat16() for _ in range(2))
    cos, sin = (torch.from_numpy(t).cuda() for t in _table(P, D))
    pos = torch.zeros(8, 1, dtype=torch.int32, device="cuda")
    oq, ok = torch.empty_like(q), torch.empty_like(k)
    dy = torch.randn_like(q)
    step = lambda: (*dsp.dsp_qk_norm_rope(q, k, H, H, cos=cos, sin=sin, pos=pos, out_q=oq, out_k=ok),
                    *dsp.dsp_qk_norm_rope_bwd(q, k, dy, dy, H, H, cos=cos, sin=sin, pos=pos))
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for t in range(4):
        pos.copy_(torch.arange(8, device="cuda").view(8, 1) + 9 * t)
        g.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in out]
        for a, b in zip(got, step()):
            assert torch.equal(a, b)


def test_side_stream(torch):
    import paper_2403_10266_amd as dsp
    s = torch.cuda.Stream()
    q = torch.randn(1, 4, 500, 16 * 72, device="cuda").bfloat16()
    want, _ = dsp.dsp_qk_norm_rope(q, None, 16, 0)
    s.wait_stream(torch.cuda.current_stream())
    got, _ = dsp.dsp_qk_norm_rope(q, None, 16, 0, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)
    torch.cuda.synchronize()


def test_infinite_and_nan_rows_stay_alone(torch):
    """A NaN or infinity in one head of one token reaches no other row."""
    import paper_2403_10266_amd as dsp
    for D in (72, 44):
        q = torch.randn(1, 2, 9, 5 * D, device="cuda").bfloat16()
        clean, _ = dsp.dsp_qk_norm_rope(q, None, 5, 0)
        bad = q.clone()
        bad[0, 1, 4, 2 * D + 3] = float("nan")
        bad[0, 0, 2, 0] = float("inf")
        y, _ = dsp.dsp_qk_norm_rope(bad, None, 5, 0)
        torch.cuda.synchronize()
        same = (y == clean).view(2, 9, 5, D).all(-1)
        hit = torch.zeros_like(same)
        hit[1, 4, 2] = hit[0, 2, 0] = True
        assert torch.equal(same, ~hit)


@pytest.mark.parametrize("D", [72, 44])
def test_offsets_past_32_bits_and_broadcast_rows(torch, D):
    """Tokens 2 MB apart in 4.6 GB, and one row for every token: the bits of the same
    rows side by side, forward and gradient."""
    import paper_2403_10266_amd as dsp
    L, H, gap = 2200, 2, 1 << 20
    q, dy = (torch.randn(1, 1, L, H * D, device="cuda").bfloat16() for _ in range(2))
    cos, sin = (torch.from_numpy(t).cuda() for t in _table(L, D // 2 * 2))
    def far(t):
        wide = torch.empty(L * gap, dtype=t.dtype, device="cuda").as_strided(t.shape, (0, 0, gap, 1))
        wide.copy_(t)
        return wide
    both = lambda x, g, **kw: (dsp.dsp_qk_norm_rope(x, None, H, 0, cos=cos, sin=sin, out_q=kw.get("y"))[0],  # noqa: E731
                               *dsp.dsp_qk_norm_rope_bwd(x, None, g, None, H, 0, cos=cos, sin=sin, dq=kw.get("dq"))[::2])
    want = both(q, dy)
    got = both(far(q), far(dy), y=far(torch.zeros_like(q)), dq=far(torch.zeros_like(q)))
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    one, g1 = q[:, :, :1].expand_as(q), dy[:, :, :1].expand_as(dy)
    for a, b in zip(both(one, g1), both(one.contiguous(), g1.contiguous())):
        assert torch.equal(a, b)
    torch.cuda.synchronize()
