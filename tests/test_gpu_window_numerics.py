"""Windowed attention and attention over pages in bf16 at the ends of their numbers."""
import numpy as np
import pytest

from oracle import window as ow
from tests import window_util as wu
from tests.gpu_util import dev, host, say
from tests.test_gpu_attn_window import _i32, _run, torch  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("exp", [100, 60, -60, -80, -100])
@pytest.mark.parametrize("Lq,Lk,left,kv_len", [(300, 300, -1, 300), (900, 1000, 300, 960), (200, 1400, 500, 1390), (20, 3000, -1, 2900),
                                               (2, 3000, -1, 3000), (100, 100, 30, 90)])
def test_values_of_any_magnitude(torch, exp, Lq, Lk, left, kv_len):  # noqa: F811
    """Values times a power of two give outputs times that power, at the tolerances of values
    around 1: every form of the kernel, scores that climb among them."""
    import paper_2403_10266_amd as dsp
    c = wu.case(1, 1, Lq, Lk, 4, 2, 64, "bf16", seed=50)
    for climb in (0.0, 30.0):       # nats, over the keys
        c["q"][..., 0::64] = 8.0
        c["k"][..., 0::64] = wu.synth.bf16_round(np.linspace(0, climb, Lk, dtype=np.float32))[:, None]
        kw = dict(left=left, right=0, sinks=3)
        want = wu.wanted(c, "bf16", q_pos=[kv_len - Lq], kv_len=[kv_len], grads=False, **kw)
        v = dev(c["v"], "bf16") * 2.0 ** exp
        assert torch.isfinite(v).all()
        o, lse = dsp.dsp_attn_window(dev(c["q"], "bf16"), dev(c["k"], "bf16"), v, 4, 2, q_pos=_i32(torch, [kv_len - Lq]),
                                     kv_len=_i32(torch, [kv_len]), with_lse=True, **kw)
        say(f"2^{exp}, climb {climb}")
        wu.compare(dict(o=host(o) * 2.0 ** -exp, lse=host(lse)), want, say)


@pytest.mark.parametrize("new", [1, 200])
def test_8_bit_values_of_the_least_scale(torch, new):  # noqa: F811
    """Scales of 2^-64 and 2^-40: values down to 2^-73 keep their bits."""
    import paper_2403_10266_amd as dsp
    r = np.random.default_rng(51)
    H, Hkv, D, page, kv = 4, 2, 64, 32, 320
    k = ow.e4m3(wu.draw((10, page, Hkv, D), "bf16", r) * 8)
    v = np.clip(ow.e4m3(wu.draw((10, page, Hkv, D), "bf16", r)), -448, 448)
    q = wu.draw((new, H * D), "bf16", r)
    table = r.permutation(10)[None]
    put = lambda t: torch.from_numpy(t.astype(np.float32)).cuda().to(torch.float8_e4m3fn)  # noqa: E731
    ks = torch.full((10, Hkv), 0.125, device="cuda")
    call = lambda e: dsp.dsp_attn_paged(dev(q, "bf16"), put(k), put(v), _i32(torch, table), _i32(torch, [0, new]),  # noqa: E731
                                        _i32(torch, [kv]), H, max_q=new, k_scale=ks, v_scale=torch.full_like(ks, 2.0 ** e))
    rows = lambda t: t[table[0]].reshape(1, 1, kv, Hkv * D)  # noqa: E731
    c = dict(q=q[None, None], k=rows(k) * 0.125, v=rows(v), do=q[None, None], H=H, Hkv=Hkv)
    want = wu.wanted(c, "bf16", right=0, q_pos=[kv - new], grads=False)
    for e in (0, -40, -64):
        wu.compare(dict(o=host(call(e)) * 2.0 ** -e), dict(o=want["o"]), say)


@pytest.mark.parametrize("rise", [15.5, 63.5, 300.0])
def test_scores_under_the_reference_cost_nothing(torch, rise):  # noqa: F811
    """Keys whose scores lie well above the first tile's, all on one level (a reference may sit
    just above it), take the time of keys that all score alike, and give their mean."""
    import paper_2403_10266_amd as dsp
    L, H, D = 4096, 16, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.zeros(1, 1, L, H * D, device="cuda", dtype=torch.bfloat16)
    q[..., 0::D] = 8.0
    v = torch.randn(1, 1, L, H * D, device="cuda", generator=g).bfloat16()
    out = torch.empty_like(q)
    times, ks = [[], []], []
    for up in (0.0, rise):
        k = torch.zeros_like(q)
        k[..., 64:, 0::D] = up * np.log(2.0)      # q.k / sqrt(D) = k
        ks.append(k)
    ev = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
    for i in range(12):
        for t, k in zip(times, ks):
            ev[0].record()
            for _ in range(10):
                dsp.dsp_attn_window(q, k, v, H, H, out=out)
            ev[1].record()
            torch.cuda.synchronize()
            t.append(ev[0].elapsed_time(ev[1]))
    say(f"{min(times[0]) * 100:.0f} us alike, {min(times[1]) * 100:.0f} us {rise} above the first tile")
    # weights 1 and 2^rise (of the rounded keys): D terms of at most 2^-24 each way and n rounded weights (2^-8)
    w = torch.exp((ks[1][0, 0, :, 0].double() - ks[1][0, 0, -1, 0].double()))
    vd = v.double().view(L, H * D)
    want = (w[:, None] * vd).sum(0) / w.sum()
    tol = (2.0 ** -8 + 2.0 ** -16) * (w[:, None] * vd.abs()).sum(0) / w.sum() + 2.0 ** -8 * want.abs()
    assert ((out[0, 0].double() - want).abs() <= tol).all()
    # steps of the pass are alike in number and kind; half as much again is a step taken twice
    assert min(times[1]) < 1.5 * min(times[0])


def _tight(c, left, right, sinks, q_pos, kv_len, scale):
    """{name: (value, tolerance)} of dq and dk with Delta in fp32.  With e = eta of window_util:
    dZ = P (dP - Delta) is off by 4 e P (|dO| |v| + |Delta|), and by u |dZ| where it is rounded as
    an operand (twice u P dD, dD the o's rounding in Delta, where a correction of it meets
    rounded operands); the sum by as much and the result by u."""
    H, Hkv, u = c["H"], c["Hkv"], 2.0 ** -8
    q, k, v, do = (ow._heads(c[n], h) for n, h in (("q", H), ("k", Hkv), ("v", Hkv), ("do", H)))
    D = q.shape[-1]
    _, lse, dq, dk, _ = ow.attention_window(c["q"], c["k"], c["v"], H, Hkv, left, right, sinks, q_pos, kv_len, scale, c["do"])
    tq, tk = np.zeros_like(dq), np.zeros_like(dk)
    hd = lambda t, h: t.reshape(*t.shape[:3], h, D)  # noqa: E731
    Lq, Lk = q.shape[2], k.shape[2]
    for b in range(q.shape[0]):
        ok = ow.visible(Lq, Lk, q_pos[b], kv_len[b], left, right, sinks)
        for h in range(H):
            qq, g, kk, vv = q[b, :, :, h], do[b, :, :, h], k[b, :, :, h // (H // Hkv)], v[b, :, :, h // (H // Hkv)]
            ll = lse[b, :, h][..., None]
            p = np.where(ok & ~np.isneginf(ll), np.exp(qq @ kk.swapaxes(-1, -2) * scale - np.where(np.isneginf(ll), 0, ll)), 0.0)
            S = float((np.abs(qq) @ np.abs(kk).swapaxes(-1, -2)).max() * scale)
            eta = (D + 16) * wu.N24 * (1 + S) + Lk * wu.N24
            dp = g @ vv.swapaxes(-1, -2)
            dl = (p * dp).sum(-1, keepdims=True)
            dd = u * (np.abs(g) * np.abs(p @ vv)).sum(-1, keepdims=True)
            mag = p * (np.abs(g) @ np.abs(vv).swapaxes(-1, -2) + np.abs(dl))
            e = (4 * eta + 2.0 ** -22 + max(Lk, Lq) * wu.N24) * mag + u * np.abs(p * (dp - dl)) * (1 + u) + 2 * u * p * dd
            hd(tq, H)[b, :, :, h] = scale * (e @ np.abs(kk))
            hd(tk, Hkv)[b, :, :, h // (H // Hkv)] += scale * (e.swapaxes(-1, -2) @ np.abs(qq))
    return dict(dq=(dq, tq + u * np.abs(dq)), dk=(dk, tk + u * np.abs(dk)))


@pytest.mark.parametrize("B,Lq,Lk,H,Hkv,D,left,right,sinks,kv_len", [
    (1, 200, 200, 2, 2, 64, 3, 0, 0, [200]),
    (2, 150, 150, 4, 2, 72, 1, 1, 2, [150, 40]),       # later queries see two sinks only
    (1, 300, 300, 2, 1, 128, -1, 0, 0, [300]),
    (1, 140, 260, 3, 3, 40, 9, 0, 4, [250]),
    (1, 700, 700, 2, 1, 96, 40, 0, 4, [700]),          # sinks in parts
    (3, 140, 140, 8, 4, 80, 2, 0, 1, [140, 70, 0]),
    (1, 190, 190, 2, 2, 16, 2, 2, 0, [190]),
])
def test_gradients_do_not_see_the_rounding_of_o(torch, B, Lq, Lk, H, Hkv, D, left, right, sinks, kv_len):  # noqa: F811
    """Values 64 and a little: o is rounded to halves, and dP - Delta is of that size.  Delta has to be that of
    the probabilities, not of the rounded o."""
    import paper_2403_10266_amd as dsp
    r = np.random.default_rng(Lq + D)
    c = wu.case(B, 1, Lq, Lk, H, Hkv, D, "bf16", seed=Lq)
    c["v"] = (64.0 + 0.5 * r.integers(0, 5, c["v"].shape)).astype(np.float32)
    q_pos = [n - Lq if Lq < Lk else 0 for n in kv_len]
    want = _tight(c, left, right, sinks, q_pos, kv_len, D ** -0.5)
    q, k, v, do = (dev(c[n], "bf16") for n in ("q", "k", "v", "do"))
    kw = dict(left=left, right=right, sinks=sinks, q_pos=_i32(torch, q_pos), kv_len=_i32(torch, kv_len))
    o, lse = dsp.dsp_attn_window(q, k, v, H, Hkv, with_lse=True, **kw)
    dq, dk, _ = dsp.dsp_attn_window_bwd(q, k, v, o, do, lse, H, Hkv, **kw)
    wu.compare(dict(dq=host(dq), dk=host(dk)), want, say)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("X,L,H,Hkv,D,left,sinks", [(1, 1100, 2, 1, 40, 30, 3), (90, 560, 4, 2, 16, 9, 1), (150, 800, 2, 2, 8, 5, 140),
                                                    (300, 520, 2, 2, 16, 3, 4)])
def test_sinks_of_few_and_many_units(torch, dtype, X, L, H, Hkv, D, left, sinks):
    """First tokens' gradients in many parts, in a few and in one: some units against the oracle."""
    import paper_2403_10266_amd as dsp
    r = np.random.default_rng(X)
    q, do = (wu.draw((1, X, L, H * D), dtype, r) for _ in range(2))
    k, v = (wu.draw((1, X, L, Hkv * D), dtype, r) for _ in range(2))
    kw = dict(left=left, right=0, sinks=sinks)
    n = L - 7
    put = dict(kv_len=_i32(torch, [n]))
    dq, dk, dv, dg = (dev(t, dtype) for t in (q, k, v, do))
    o, lse = dsp.dsp_attn_window(dq, dk, dv, H, Hkv, with_lse=True, **put, **kw)
    got = dict(zip(("dq", "dk", "dv"), dsp.dsp_attn_window_bwd(dq, dk, dv, o, dg, lse, H, Hkv, **put, **kw)))
    for x in {0, X // 2, X - 1}:
        c = dict(q=q[:, x:x + 1], k=k[:, x:x + 1], v=v[:, x:x + 1], do=do[:, x:x + 1], H=H, Hkv=Hkv)
        want = wu.wanted(c, dtype, kv_len=[n], **kw)
        say(f"unit {x} of {X}")
        wu.compare({m: host(t[:, x:x + 1]) for m, t in got.items()}, {m: want[m] for m in got}, say)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Lq,sinks", [(300, 3), (3, 0)])
def test_rows_far_apart(torch, dtype, Lq, sinks):  # noqa: F811
    """Rows whose offsets inside one unit pass 32 bits, q, k and v columns of one buffer, and
    their gradients of another: the bits of compact rows."""
    import paper_2403_10266_amd as dsp
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of free GPU memory")
    L, H, D = 300, 2, 64
    step, C = (1 << 22 if dtype == "f32" else 1 << 23), H * D
    c = wu.case(1, 1, Lq, L, H, H, D, dtype, seed=60)
    q, k, v, do = (dev(c[n], dtype) for n in ("q", "k", "v", "do"))
    kw = dict(left=40, right=0, sinks=sinks, q_pos=_i32(torch, [L - Lq]))

    def views():
        base = torch.empty(L * step, dtype=q.dtype, device="cuda")
        assert (L - 1) * step * base.element_size() > 2 ** 32
        return [base.as_strided((1, 1, n, C), (n * step, n * step, step, 1), i * C) for i, n in enumerate((Lq, L, L))]

    far, grads, got = views(), views(), []
    for t, x in zip(far, (q, k, v)):
        t.copy_(x)
    for t, g in (((q, k, v), [torch.empty_like(x) for x in (q, k, v)]), (far, grads)):
        o, lse = dsp.dsp_attn_window(*t, H, H, with_lse=True, **kw)
        got.append([o, lse, *dsp.dsp_attn_window_bwd(*t, o, do, lse, H, H, dq=g[0], dk=g[1], dv=g[2], **kw)])
    assert torch.isfinite(got[0][0].float()).all()
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Lq,Lk", [(2, 600), (40, 50), (150, 200)])
def test_positions_at_the_ends_of_32_bits(torch, dtype, Lq, Lk):  # noqa: F811
    """First queries at positions of any size, with windows that reach back to the keys, that just
    do and that do not."""
    far = 2 ** 31 - 1
    c = wu.case(1, 1, Lq, Lk, 2, 1, 64, dtype, seed=70)
    for q_pos, left, right in ((far, 2 ** 30 + 5, 0), (far, far - 30, 0), (far, far, -1), (-far - 1, -1, 2 ** 30 + 5),
                               (-far - 1, 7, far), (-far - 1 + Lq, -1, far - 20), (2 ** 30 + 9, 2 ** 30, 3)):
        kw = dict(left=left, right=right, sinks=0, q_pos=[q_pos])
        say(kw)
        got = _run(torch, c, dtype, **kw)
        wu.compare({n: host(t) for n, t in got.items()}, wu.wanted(c, dtype, **kw), say)
