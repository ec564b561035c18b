"""Norm with rotation and attention with a relative position bias as they are used
together: a packed projection through both and its gradient back, a cache that grows
token by token, many units at once, streams side by side.

Each call is held to the oracle at its own inputs, with the tolerances of
tests/relpos_util.py and tests/test_gpu_qk_norm_rope.py.  The fp32 chain from end to
end: a normalised row is off by 2^-17 of its size, so a score by 2^-16 of its sum of
magnitudes S; with S <= 32 (heads of 16 to 24 elements of about 1, scale D^-1/2) a
probability is off by 2^-11 and a gradient, a sum of two such products, by 2^-10 of
its largest element."""
import numpy as np
import pytest

from oracle import position as po
from tests import relpos_util as ru
from tests import test_gpu_qk_norm_rope as nr
from tests.gpu_util import dev, host, say
from tests.test_gpu_attn_relpos import _check, _run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


def _held(got, want):
    ru.compare({n: host(t) for n, t in got.items()}, want, say)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,X,L,H,D,rot,causal", [(1, 6, 32, 4, 24, 24, False), (2, 1, 150, 3, 16, 8, True),
                                                  (2, 2, 70, 2, 72, 72, True)])
def test_packed_projection_and_back(torch, dtype, B, X, L, H, D, rot, causal):
    """[Q | K | V] of one buffer: norm and rotation in place, attention, and the
    gradients back into one buffer, in place again."""
    import paper_2403_10266_amd as dsp
    C = H * D
    u = ru.draw((B, X, L, 3 * C), dtype, np.random.default_rng(7))
    gq, gk = (ru.draw((D,), dtype, np.random.default_rng(8 + i), 0.2) + np.float32(1) for i in range(2))
    c = ru.case(B, X, L, L, H, H, D, 12, 6, dtype, seed=3)
    if dtype == "bf16":
        gq, gk = (ru.synth.bf16_round(g) for g in (gq, gk))
    cos, sin = nr._table(L, rot)
    cut = lambda t: [t[..., i * C:(i + 1) * C] for i in range(3)]  # noqa: E731
    raw, buf, gbuf = dev(u, dtype), dev(u, dtype), dev(np.zeros_like(u), dtype)
    norm = dict(gq=dev(gq, dtype), gk=dev(gk, dtype), cos=torch.from_numpy(cos).cuda(), sin=torch.from_numpy(sin).cuda())
    q, k, v = cut(buf)
    dsp.dsp_qk_norm_rope(q, k, H, H, out_q=q, out_k=k, **norm)
    bias, bk, do = dev(c["bias"], dtype), torch.from_numpy(c["buckets"]).cuda(), dev(c["do"], dtype)
    o, lse = dsp.dsp_attn_relpos(q, k, v, H, H, bias, bk, causal=causal, with_lse=True)
    dq, dk, dv = cut(gbuf)
    *_, db = dsp.dsp_attn_relpos_bwd(q, k, v, o, do, lse, H, H, bias, bk, causal=causal, dq=dq, dk=dk, dv=dv)
    at_attn = {n: t.clone() for n, t in (("dq", dq), ("dk", dk), ("dv", dv))}
    rq, rk, rv = cut(raw)
    _, _, dgq, dgk = dsp.dsp_qk_norm_rope_bwd(rq, rk, dq, dk, H, H, dq=dq, dk=dk, **norm)
    torch.cuda.synchronize()
    assert torch.equal(v, rv) and torch.equal(dv, at_attn["dv"])
    for x, y, g in ((rq, q, gq), (rk, k, gk)):
        x = host(x)
        nr._within(host(y), po.qk_norm_rope(x, H, g, cos, sin), nr._row_size(po.qk_norm_rope(x, H, g), H), dtype, "y")
    at = dict(c, **{n: host(t).astype(np.float32) for n, t in (("q", q), ("k", k), ("v", v))})
    _held(dict(o=o, lse=lse, dbias=db, **at_attn), ru.wanted(at, dtype, causal))
    for x, dy, dx, dg, g in ((rq, at_attn["dq"], dq, dgq, gq), (rk, at_attn["dk"], dk, dgk, gk)):
        x, dy = host(x), host(dy)
        wx, wg = po.qk_norm_rope_bwd(x, dy, H, g, cos, sin)
        row = lambda t: t.reshape(B, X, L, H, D)  # noqa: E731
        r = 1 / np.sqrt((row(x).astype(np.float64) ** 2).mean(-1, keepdims=True) + 1e-6)
        w = np.sqrt(2) * np.abs(row(dy)).max(-1, keepdims=True)
        size = r * w * np.abs(g).max() * (1 + np.abs(row(x)).max(-1, keepdims=True) * r * r
                                          * np.abs(row(x)).mean(-1, keepdims=True))
        nr._within(host(dx), wx, np.broadcast_to(size, row(x).shape).reshape(x.shape), dtype, "dx")
        nr._within(host(dg), wg, np.abs(w * row(x) * r).sum((0, 1, 2, 3)), "f32", "dg")
    if dtype == "bf16" or D > 24:
        return
    # from end to end
    uq, uk, uv = (t.astype(np.float64) for t in cut(u))
    yq, yk = po.qk_norm_rope(uq, H, gq, cos, sin), po.qk_norm_rope(uk, H, gk, cos, sin)
    wo, _, wq, wk, wv, wb = po.attention_relpos(yq, yk, uv, H, H, c["bias"], c["buckets"], causal, None, None,
                                                D ** -0.5, c["do"])
    wq, wgq = po.qk_norm_rope_bwd(uq, wq, H, gq, cos, sin)
    wk, wgk = po.qk_norm_rope_bwd(uk, wk, H, gk, cos, sin)
    for name, a, b in (("o", o, wo), ("dq", dq, wq), ("dk", dk, wk), ("dv", dv, wv), ("dbias", db, wb),
                       ("dgq", dgq, wgq), ("dgk", dgk, wgk)):
        assert np.abs(host(a) - b).max() <= 2.0 ** -10 * np.abs(b).max(), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_cache_that_grows(torch, dtype):
    """A prefill, then tokens one at a time: keys go through the norm straight into
    their place in the cache; each step as the oracle has it on that cache, the cache
    as one call over the whole sequence writes it."""
    import paper_2403_10266_amd as dsp
    B, H, Hkv, D, room, n0, steps = 3, 6, 2, 64, 700, 290, 3
    lens0 = [n0, 33, 1]                                      # of the prefill; the batch is padded
    u = lambda *s, seed: dev(ru.draw(s, dtype, np.random.default_rng(seed)), dtype)  # noqa: E731
    q, k, v = (u(B, 1, n0 + steps, h * D, seed=i) for i, h in enumerate((H, Hkv, Hkv)))
    cos, sin = (torch.from_numpy(t).cuda() for t in nr._table(room, D))
    c = ru.case(1, 1, 1, 1, H, Hkv, D, 50, 12, dtype, seed=5)
    bias, bk = dev(c["bias"], dtype), torch.from_numpy(c["buckets"]).cuda()
    kc, vc = (torch.full((B, 1, room, Hkv * D), float("nan"), dtype=q.dtype, device="cuda") for _ in range(2))
    yq, _ = dsp.dsp_qk_norm_rope(q[:, :, :n0], k[:, :, :n0], H, Hkv, cos=cos, sin=sin, out_k=kc[:, :, :n0])
    vc[:, :, :n0] = v[:, :, :n0]
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731

    def held(got, y, lens, q_pos):
        torch.cuda.synchronize()
        at = dict(c, q=host(y), k=host(kc), v=host(vc), do=None)
        at = {n: np.nan_to_num(t) if n in "kv" else t for n, t in at.items()}
        at["do"] = at["q"]
        _held(dict(o=got[0], lse=got[1]), ru.wanted(at, dtype, True, q_pos, lens, grads=False))

    kw = dict(causal=True, with_lse=True)
    got = dsp.dsp_attn_relpos(yq, kc, vc, H, Hkv, bias, bk, kv_len=i32(lens0), **kw)
    held(got, yq, lens0, None)
    for t in range(steps):
        lens = [n + t + 1 for n in lens0]
        for b, n in enumerate(lens):                         # the token's own inputs, at its own place
            y1, _ = dsp.dsp_qk_norm_rope(q[b:b + 1, :, n - 1:n], k[b:b + 1, :, n - 1:n], H, Hkv, cos=cos, sin=sin,
                                         pos=i32([[n - 1]]), out_k=kc[b:b + 1, :, n - 1:n])
            yq = y1 if b == 0 else torch.cat([yq, y1])
            vc[b, :, n - 1] = v[b, :, n - 1]
        pos = [n - 1 for n in lens]
        got = dsp.dsp_attn_relpos(yq, kc, vc, H, Hkv, bias, bk, q_pos=i32(pos), kv_len=i32(lens), **kw)
        held(got, yq, lens, pos)
    _, whole = dsp.dsp_qk_norm_rope(None, k, 0, Hkv, cos=cos, sin=sin)
    torch.cuda.synchronize()
    for b, n in enumerate(lens0):
        assert torch.equal(kc[b, :, :n + steps], whole[b, :, :n + steps])


MANY = [
    # B, X, Lq, Lk, H, Hkv, D, causal, q_pos, kv_len, grads: units, rows or keys enough for
    # each way of sharing out the work
    (1, 130, 100, 100, 2, 2, 32, False, None, None, True),
    (2, 66, 90, 200, 2, 2, 24, False, None, None, True),
    (2, 130, 70, 90, 2, 2, 40, True, [20, -3], [90, 50], True),
    (1, 130, 80, 100, 2, 2, 96, False, None, None, True),
    (2, 700, 33, 33, 3, 3, 16, False, [0, 9], [33, 20], True),
    (2, 900, 20, 28, 3, 3, 72, True, [8, 3], None, True),
    (2, 300, 33, 40, 6, 2, 64, True, [7, -5], [40, 31], True),
    (2, 700, 3, 3, 8, 2, 128, True, None, [3, 2], True),
    (3, 50, 64, 50, 4, 1, 24, False, [0, -70, 70], [50, 0, 1], True),
    (2, 130, 32, 30, 8, 4, 72, False, None, None, True),
    (1, 3, 2, 64, 5, 1, 96, True, [60], None, True),
    (3, 120, 64, 64, 2, 2, 128, False, [0, -70, 70], [64, 0, 1], True),
    (2, 900, 3, 75, 4, 2, 64, True, [72, 40], [75, 43], False),
    (1, 1700, 1, 150, 4, 2, 72, False, None, None, False),
    (2, 40, 2, 60, 6, 2, 72, True, [58, 1], [60, 3], False),
    (2, 40, 1024, 130, 2, 2, 72, False, [0, -900], None, False),
    (1, 70, 1025, 70, 2, 1, 64, True, [-990], None, False),
    (1, 40, 1030, 70, 2, 2, 128, False, None, [69], False),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,X,Lq,Lk,H,Hkv,D,causal,q_pos,kv_len,grads", MANY)
def test_many_units(torch, dtype, B, X, Lq, Lk, H, Hkv, D, causal, q_pos, kv_len, grads):
    c = ru.case(B, X, Lq, Lk, H, Hkv, D, 25, 9, dtype, seed=X)
    _check(torch, c, dtype, f"relpos X{X} {Lq}x{Lk} D{D}", causal=causal, q_pos=q_pos, kv_len=kv_len, grads=grads)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_short_units_with_long_tables(torch, dtype):
    """Groups whose tables are past what the short units' kernel keeps."""
    for M, H, Hkv in ((1024, 8, 2), (1024, 2, 2), (900, 4, 2)):
        c = ru.case(2, 5, 20, 30, H, Hkv, 64, M, 30, dtype, seed=M)
        _check(torch, c, dtype, f"relpos M{M} H{H}/{Hkv}", q_pos=[0, 950])


def test_two_streams_at_once(torch):
    """Training steps on two streams that run side by side, workspaces and outputs of
    their own: the bits of each alone."""
    import paper_2403_10266_amd as dsp
    H, D = 4, 72
    cos, sin = (torch.from_numpy(t).cuda() for t in nr._table(200, D))
    bias, bk = torch.randn(8, H, device="cuda").bfloat16(), dsp.dsp_relpos_buckets(40, 8).cuda()
    data = [[torch.randn(2, X, L, H * D, device="cuda").bfloat16() for _ in range(4)] for X, L in ((40, 33), (2, 200))]

    def step(q, k, v, do):
        yq, yk = dsp.dsp_qk_norm_rope(q, k, H, H, cos=cos, sin=sin)
        o, lse = dsp.dsp_attn_relpos(yq, yk, v, H, H, bias, bk, with_lse=True)
        g = dsp.dsp_attn_relpos_bwd(yq, yk, v, o, do, lse, H, H, bias, bk)
        return [o, lse, *g[2:], *dsp.dsp_qk_norm_rope_bwd(q, k, g[0], g[1], H, H, cos=cos, sin=sin)]

    alone = [step(*d) for d in data]
    streams = [torch.cuda.Stream() for _ in data]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    kept = []
    for _ in range(6):
        for s, d in zip(streams, data):
            with torch.cuda.stream(s):
                kept.append(step(*d))
    torch.cuda.synchronize()
    for i, got in enumerate(kept):
        for a, b in zip(got, alone[i % 2]):
            assert torch.equal(a, b), i
