"""Attention with a learned relative position bias on the GPU, forward and gradients,
against the oracle with the tolerances of tests/relpos_util.py."""
import numpy as np
import pytest

from tests import relpos_util as ru
from tests.gpu_util import dev, host, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


def _i32(torch, a):
    return None if a is None else torch.tensor(a, dtype=torch.int32, device="cuda")


def _run(torch, c, dtype, causal=False, q_pos=None, kv_len=None, scale=0.0, grads=True, put=None):
    import paper_2403_10266_amd as dsp
    put = put or (lambda t, n: dev(t, dtype))
    q, k, v = (put(c[n], n) for n in "qkv")
    bias, bk = dev(c["bias"], dtype), torch.from_numpy(c["buckets"]).cuda()
    kw = dict(causal=causal, q_pos=_i32(torch, q_pos), kv_len=_i32(torch, kv_len), scale=scale)
    o, lse = dsp.dsp_attn_relpos(q, k, v, c["H"], c["Hkv"], bias, bk, with_lse=True, **kw)
    got = dict(o=o, lse=lse)
    if grads:
        g = dsp.dsp_attn_relpos_bwd(q, k, v, o, dev(c["do"], dtype), lse, c["H"], c["Hkv"], bias, bk, **kw,
                                    **({} if q.is_contiguous() else dict(dq=torch.empty_strided(
                                        q.shape, q.stride(), dtype=q.dtype, device="cuda"))))
        got |= dict(zip(("dq", "dk", "dv", "dbias"), g))
    torch.cuda.synchronize()
    return got


def _check(torch, c, dtype, what, scale=None, **kw):
    say(what, dtype, kw)
    got = _run(torch, c, dtype, scale=scale or 0.0, **kw)
    want = ru.wanted(c, dtype, kw.get("causal", False), kw.get("q_pos"), kw.get("kv_len"), scale,
                     kw.get("grads", True))
    ru.compare({n: host(t) for n, t in got.items()}, want, say)
    return got


CASES = [
    # B, X, Lq, Lk, H, Hkv, D, M, nb, causal, q_pos, kv_len
    (1, 2, 64, 64, 2, 2, 72, 20, 8, False, None, None),
    (2, 3, 32, 32, 4, 4, 72, 128, 32, False, None, None),
    (1, 4, 17, 17, 2, 2, 64, 5, 4, True, None, None),
    (2, 1, 150, 150, 2, 1, 72, 16, 8, True, None, [150, 61]),
    (3, 1, 70, 90, 4, 2, 64, 30, 9, False, None, [0, 90, 33]),     # no keys at all; odd lengths
    (2, 1, 40, 200, 2, 2, 80, 64, 16, True, [160, 30], [200, 70]),  # positions inside a cache
    (1, 2, 33, 65, 2, 1, 128, 10, 3, False, [-40], None),           # queries before the keys
    (2, 1, 65, 33, 2, 2, 32, 3, 5, True, [-20, 5], None),           # rows before the first key
    (1, 1, 300, 300, 2, 2, 40, 40, 12, False, None, None),          # blocks past both ends of the table
    (1, 1, 260, 260, 1, 1, 96, 100, 20, True, None, None),
    (1, 2, 129, 257, 2, 2, 16, 0, 1, False, None, None),            # one bias for every distance
    (1, 3, 1, 1, 2, 1, 72, 4, 2, False, None, None),
    (1, 2, 5, 1, 2, 2, 64, 4, 9, False, None, None),
    (1, 1, 100, 40, 3, 1, 24, 1000, 33, False, None, None),         # a table longer than the sequence
    (1, 1, 40, 300, 8, 2, 48, 200, 300, True, [260], None),         # a bias of nearly every distance's own
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,X,Lq,Lk,H,Hkv,D,M,nb,causal,q_pos,kv_len", CASES)
def test_against_the_oracle(torch, dtype, B, X, Lq, Lk, H, Hkv, D, M, nb, causal, q_pos, kv_len):
    c = ru.case(B, X, Lq, Lk, H, Hkv, D, M, nb, dtype, seed=Lq + D)
    _check(torch, c, dtype, f"relpos B{B} X{X} {Lq}x{Lk} H{H}/{Hkv} D{D} M{M} nb{nb}", causal=causal, q_pos=q_pos,
           kv_len=kv_len)


@pytest.mark.parametrize("D", [1, 3, 20, 70])
def test_odd_widths_f32(torch, D):
    c = ru.case(1, 2, 37, 45, 2, 1, D, 12, 7, "f32", seed=D)
    _check(torch, c, "f32", f"relpos D{D}")


TOKENS = [
    # B, X, Lq, Lk, H, Hkv, D, lens
    (3, 1, 1, 900, 4, 4, 72, [900, 1, 0]),
    (2, 1, 1, 2500, 8, 2, 64, [2500, 1300]),
    (2, 3, 2, 700, 8, 1, 72, [700, 259]),
    (1, 1, 5, 1025, 6, 1, 128, [1025]),       # 30 rows in one block
    (2, 40, 1, 120, 8, 2, 72, [120, 77]),
    (1, 1, 32, 600, 2, 2, 80, [600]),
    (2, 1, 8, 513, 4, 1, 40, [513, 5]),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,X,Lq,Lk,H,Hkv,D,lens", TOKENS)
def test_tokens_against_a_cache(torch, dtype, B, X, Lq, Lk, H, Hkv, D, lens):
    """The last Lq positions of each sequence against its keys so far."""
    c = ru.case(B, X, Lq, Lk, H, Hkv, D, 60, 16, dtype, seed=Lk)
    _check(torch, c, dtype, f"relpos tokens {Lq}x{Lk}", causal=True, q_pos=[n - Lq for n in lens], kv_len=lens,
           grads=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masks_in_the_table(torch, dtype):
    """-inf, the type's lowest value and -1e30 take distances out, a row left with
    nothing among them; entries outside the table add nothing."""
    lowest = -3.3895313892515355e38 if dtype == "bf16" else -3.4028234663852886e38
    for low in (-np.inf, lowest, -2e30):
        c = ru.case(1, 2, 50, 60, 2, 2, 72, 10, 4, dtype, seed=3)
        c["bias"][1, 0] = c["bias"][2, 1] = low
        c["buckets"][0], c["buckets"][5], c["buckets"][-1] = 7, -1, 2 ** 30
        _check(torch, c, dtype, f"masked by {low}")
        c["bias"][:, 0] = low                         # head 0 keeps only what has no bias
        c["buckets"][:] = np.where(np.arange(21) < 8, 0, 3)
        got = _check(torch, c, dtype, "a head with nothing")
        assert not host(got["o"])[..., :72].any() and np.isneginf(host(got["lse"])[:, :, 0]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_lies_past_the_length(torch, dtype):
    """NaN and infinities in keys and values past kv_len change no bit."""
    import paper_2403_10266_amd as dsp
    for Lq, causal, pos in ((70, False, None), (1, True, [49, 20])):
        c = ru.case(2, 2, Lq, 90, 4, 2, 72, 20, 8, dtype, seed=9)
        lens = [50, 21]
        a = _run(torch, c, dtype, causal=causal, q_pos=pos, kv_len=lens)
        for b, n in enumerate(lens):
            c["k"][b, :, n:] = np.nan
            c["v"][b, :, n:, ::2] = np.inf
            c["v"][b, :, n:, 1::2] = np.nan
        bad = _run(torch, c, dtype, causal=causal, q_pos=pos, kv_len=lens)
        for n in a:
            assert torch.equal(a[n], bad[n]), n
        assert not a["dk"][1, :, 21:].any() and not a["dv"][1, :, 21:].any()


def test_lengths_outside_the_cache(torch):
    """kv_len past Lk or negative is clamped, positions of any size are taken."""
    c = ru.case(3, 1, 20, 40, 2, 2, 64, 10, 4, "bf16", seed=2)
    a = _run(torch, c, "bf16", kv_len=[40, 0, 7])
    b = _run(torch, c, "bf16", kv_len=[2 ** 31 - 1, -5, 7])
    for n in a:
        assert torch.equal(a[n], b[n]), n
    far = _run(torch, c, "bf16", q_pos=[2 ** 31 - 1, -2 ** 31, 0])
    end = dict(c, buckets=np.concatenate([np.full(10, c["buckets"][0]), c["buckets"][:1], np.full(10, c["buckets"][-1])]).astype(np.int32))
    near = _run(torch, end, "bf16", q_pos=[1000, -1000, 0])
    assert torch.equal(far["o"][:2], near["o"][:2])
    out = _run(torch, c, "bf16", causal=True, q_pos=[-2 ** 31, 2 ** 31 - 1, 0])
    assert not out["o"][0].any() and torch.equal(out["o"][1], far["o"][0] * 0 + out["o"][1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_scores(torch, dtype):
    """Scores whose running maximum moves many times, and rows of one key each."""
    c = ru.case(1, 1, 70, 600, 2, 2, 64, 300, 40, dtype, seed=5, bias_scale=30.0)
    ramp = np.linspace(0, 4, 600, dtype=np.float32)[None, None, :, None]
    c["k"] = c["k"] * (ru.synth.bf16_round(np.broadcast_to(ramp, c["k"].shape).copy()))
    if dtype == "bf16":
        c["k"] = ru.synth.bf16_round(c["k"])
    _check(torch, c, dtype, "ramp", scale=0.5)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_views_and_packed_buffers(torch, dtype):
    """q, k, v and the gradients as columns of packed buffers, (B, L, X) order; keys
    and values shared by every x (stride 0) in the forward."""
    import paper_2403_10266_amd as dsp
    H, D, B, X, L = 4, 72, 2, 3, 45
    c = ru.case(B, X, L, L, H, H, D, 16, 8, dtype, seed=11)
    tt = torch.bfloat16 if dtype == "bf16" else torch.float32
    buf, gbuf = (torch.zeros(B, L, X, 3 * H * D + 16, dtype=tt, device="cuda") for _ in range(2))
    cut = lambda t: [t.permute(0, 2, 1, 3)[..., i * H * D:(i + 1) * H * D] for i in range(3)]
    for view, n in zip(cut(buf), "qkv"):
        view.copy_(dev(c[n], dtype))
    q, k, v = cut(buf)
    bias, bk = dev(c["bias"], dtype), torch.from_numpy(c["buckets"]).cuda()
    o, lse = dsp.dsp_attn_relpos(q, k, v, H, H, bias, bk, with_lse=True)
    dq, dk, dv = cut(gbuf)
    gbuf[..., 3 * H * D:] = 7
    *_, db = dsp.dsp_attn_relpos_bwd(q, k, v, o, dev(c["do"], dtype), lse, H, H, bias, bk, dq=dq, dk=dk, dv=dv)
    torch.cuda.synchronize()
    ru.compare({n: host(t) for n, t in dict(o=o, lse=lse, dq=dq, dk=dk, dv=dv, dbias=db).items()},
               ru.wanted(c, dtype), say)
    assert (gbuf[..., 3 * H * D:] == 7).all()
    one = {n: dev(c[n][:, :1], dtype).expand(B, X, L, H * D) for n in "kv"}
    got = dsp.dsp_attn_relpos(dev(c["q"], dtype), one["k"], one["v"], H, H, bias, bk)
    want = dsp.dsp_attn_relpos(dev(c["q"], dtype), one["k"].contiguous(), one["v"].contiguous(), H, H, bias, bk)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_f32_off_16_bytes(torch):
    """fp32 rows that start anywhere, of a width that 16 bytes do not divide."""
    c = ru.case(1, 2, 40, 50, 2, 2, 22, 9, 5, "f32", seed=8)
    def put(t, n):
        wide = torch.zeros(*t.shape[:3], t.shape[3] + 7, device="cuda")
        view = wide[..., 3:3 + t.shape[3]]
        view.copy_(dev(t, "f32"))
        return view
    got = _run(torch, c, "f32", put=put, grads=False)
    ru.compare({n: host(t) for n, t in got.items()}, ru.wanted(c, "f32", grads=False), say)


def test_zero_bias_equals_plain_attention(torch):
    """With a table of zeros, the framework's plain attention to its tolerance."""
    import paper_2403_10266_amd as dsp
    from tests.gpu_util import assert_close
    c = ru.case(1, 3, 200, 200, 4, 2, 72, 30, 8, "bf16", seed=1)
    c["bias"][:] = 0
    o = _run(torch, c, "bf16", grads=False)["o"]
    q, k, v = (dev(c[n], "bf16") for n in "qkv")
    p = dsp.dsp_attn_general(q, k, v, 4, 2)
    torch.cuda.synchronize()
    assert_close(host(o), host(p), "bf16", "zero bias")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradient_against_differences(torch, dtype):
    """The bias gradient against central differences of the forward in 64 bits, on the
    GPU's rounded inputs (the differences' own error is 1e-6 of the loss's terms)."""
    from oracle import position as po
    c = ru.case(1, 2, 33, 40, 2, 1, 24, 6, 4, dtype, seed=21)
    got = _run(torch, c, dtype)
    tol = ru.wanted(c, dtype)["dbias"][1]
    f = lambda b: (c["do"] * po.attention_relpos(c["q"], c["k"], c["v"], 2, 1, b, c["buckets"])[0]).sum()
    for at in np.ndindex(4, 2):
        e = np.zeros((4, 2))
        e[at] = 1e-4
        num = (f(c["bias"] + e) - f(c["bias"] - e)) / 2e-4
        assert abs(host(got["dbias"])[at] - num) <= tol[at] + 1e-5 * np.abs(c["do"]).sum(), at


def test_same_bits_every_time(torch):
    """Repeated calls give identical bits, between other work on the chip."""
    c = ru.case(2, 3, 333, 333, 4, 2, 72, 50, 16, "bf16", seed=4)
    first = _run(torch, c, "bf16", causal=True, kv_len=[333, 200])
    for _ in range(3):
        torch.randn(4096, 4096, device="cuda") @ torch.randn(4096, 4096, device="cuda")
        again = _run(torch, c, "bf16", causal=True, kv_len=[333, 200])
        for n in first:
            assert torch.equal(first[n], again[n]), n


def test_graph_replays_and_streams(torch):
    """A token's step (split keys among it) and a training step in captured graphs:
    replays with moved positions, between eager calls; two graphs with workspaces of
    their own."""
    import paper_2403_10266_amd as dsp
    H, Hkv, D, M, nb = 8, 2, 64, 40, 8
    r = lambda *s: torch.randn(*s, device="cuda").bfloat16()
    k, v, q = r(2, 1, 3000, Hkv * D), r(2, 1, 3000, Hkv * D), r(2, 1, 1, H * D)
    bias, bk = r(nb, H), dsp.dsp_relpos_buckets(M, nb, False).cuda()
    lens = torch.tensor([10, 20], dtype=torch.int32, device="cuda")
    pos = lens - 1
    token = lambda: [dsp.dsp_attn_relpos(q, k, v, H, Hkv, bias, bk, causal=True, q_pos=pos, kv_len=lens)]
    tq, tk, tv, do = r(1, 4, 90, H * D), r(1, 4, 90, Hkv * D), r(1, 4, 90, Hkv * D), r(1, 4, 90, H * D)
    def train():
        o, lse = dsp.dsp_attn_relpos(tq, tk, tv, H, Hkv, bias, bk, with_lse=True)
        return [o, lse, *dsp.dsp_attn_relpos_bwd(tq, tk, tv, o, do, lse, H, Hkv, bias, bk)]
    graphs = []
    for fn in (token, train):
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            fn()
        torch.cuda.current_stream().wait_stream(s)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = fn()
        graphs.append((g, out, fn))
    for t in range(4):
        lens.copy_(torch.tensor([10 + 900 * t, 2999 - t], dtype=torch.int32, device="cuda"))
        pos.copy_(lens - 1)
        tq.mul_(0.9)
        for g, out, fn in graphs:
            g.replay()
        torch.cuda.synchronize()
        for g, out, fn in graphs:
            got = [x.clone() for x in out]
            for a, b in zip(got, fn()):
                assert torch.equal(a, b), t
    side = torch.cuda.Stream()
    want = token()[0]
    side.wait_stream(torch.cuda.current_stream())
    got = dsp.dsp_attn_relpos(q, k, v, H, Hkv, bias, bk, causal=True, q_pos=pos, kv_len=lens, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_empty(torch):
    import paper_2403_10266_amd as dsp
    z = lambda *s: torch.zeros(*s, device="cuda")
    bias, bk = z(4, 2), dsp.dsp_relpos_buckets(3, 4).cuda()
    o, lse = dsp.dsp_attn_relpos(z(1, 2, 0, 16), z(1, 2, 5, 16), z(1, 2, 5, 16), 2, 2, bias, bk, with_lse=True)
    assert o.numel() == 0 and lse.numel() == 0
    o, lse = dsp.dsp_attn_relpos(z(1, 2, 3, 16) + 1, z(1, 2, 0, 16), z(1, 2, 0, 16), 2, 2, bias, bk, with_lse=True)
    torch.cuda.synchronize()
    assert not o.any() and lse.isneginf().all()
    for Lq, Lk in ((0, 5), (3, 0), (0, 0)):
        q, k = z(1, 2, Lq, 16), z(1, 2, Lk, 16)
        dq, dk, dv, db = dsp.dsp_attn_relpos_bwd(q, k, k, q, q, z(1, 2, 2, Lq), 2, 2, bias, bk)
        torch.cuda.synchronize()
        assert not any(t.any() for t in (dq, dk, dv, db))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Lq,Lk", [(1, 200), (3, 50), (32, 32), (60, 60), (70, 150)])
def test_rows_of_any_stride(torch, dtype, Lq, Lk):
    """One key for every position (stride 0), key rows that overlap, one query for
    every row: as with the same rows in their own places."""
    import paper_2403_10266_amd as dsp
    H, D = 2, 24
    c = ru.case(1, 3, Lq, Lk, H, H, D, 9, 5, dtype, seed=Lq)
    bias, bk = dev(c["bias"], dtype), torch.from_numpy(c["buckets"]).cuda()
    q, k, v = (dev(c[n], dtype) for n in "qkv")
    flat = [t.reshape(-1) for t in (k, v)]
    views = dict(one=[t[:, :, :1].expand_as(t) for t in (k, v)],
                 close=[t.as_strided(k.shape, (0, Lk * 8, 8, 1)) for t in flat])
    for kind, (a, b) in views.items():
        got = dsp.dsp_attn_relpos(q, a, b, H, H, bias, bk)
        want = dsp.dsp_attn_relpos(q, a.contiguous(), b.contiguous(), H, H, bias, bk)
        torch.cuda.synchronize()
        assert torch.equal(got, want), kind
    one = q[:, :, -1:].expand_as(q)
    assert torch.equal(dsp.dsp_attn_relpos(one, k, v, H, H, bias, bk),
                       dsp.dsp_attn_relpos(one.contiguous(), k, v, H, H, bias, bk))
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_tables_of_wide_heads_and_groups(torch, dtype):
    """The longest table with the widest heads, and with groups whose tables do not fit
    a work-group together (with the keys cut among work-groups, and not)."""
    import paper_2403_10266_amd as dsp
    for Lq, Lk, H, Hkv, D in ((60, 60, 2, 2, 128), (150, 1300, 2, 2, 128), (1300, 150, 2, 1, 80)):
        c = ru.case(1, 1, Lq, Lk, H, Hkv, D, 1024, 40, dtype, seed=D)
        _check(torch, c, dtype, f"M1024 D{D}")
    for D, H, Lq, lens in ((128, 32, 1, [2100, 1, 0]), (64, 30, 1, [2100, 2000, 7]), (72, 6, 5, [1800, 5, 900])):
        c = ru.case(3, 1, Lq, max(lens), H, 1, D, 1024, 40, dtype, seed=H)
        _check(torch, c, dtype, f"M1024 group {H}", causal=True, q_pos=[n - Lq for n in lens], kv_len=lens, grads=False)
    c = ru.case(1, 2, 1, 2400, 32, 1, 32, 1024, 40, dtype, seed=6)
    q, k, v = (dev(c[n], dtype) for n in "qkv")
    many = lambda t: t[:, :1].expand(1, 2100, *t.shape[2:])  # noqa: E731
    pos = torch.tensor([1200], dtype=torch.int32, device="cuda")
    o, lse = dsp.dsp_attn_relpos(many(q), many(k), many(v), 32, 1, dev(c["bias"], dtype),
                                 torch.from_numpy(c["buckets"]).cuda(), q_pos=pos, with_lse=True)
    torch.cuda.synchronize()
    assert (o == o[:, :1]).all() and (lse == lse[:, :1]).all()
    c = {n: t[:, :1] if n in ("q", "k", "v", "do") else t for n, t in c.items()}
    ru.compare(dict(o=host(o[:, :1]), lse=host(lse[:, :1])), ru.wanted(c, dtype, False, [1200], None, grads=False), say)


def test_offsets_past_32_bits(torch):
    """Rows of keys 2 MB apart, 4.6 GB of them: the bits of the same rows side by side."""
    import paper_2403_10266_amd as dsp
    H, D, Lk, gap = 2, 64, 2200, 1 << 20
    def far(t):
        wide = torch.empty(Lk * gap, dtype=t.dtype, device="cuda").as_strided(t.shape, (0, 0, gap, 1))
        wide.copy_(t)
        return wide
    c = ru.case(1, 1, 100, Lk, H, H, D, 30, 8, "bf16", seed=1)
    near = {n: dev(c[n], "bf16") for n in "qkv"}
    k, v = far(near["k"]), far(near["v"])
    bias, bk, do = dev(c["bias"], "bf16"), torch.from_numpy(c["buckets"]).cuda(), dev(c["do"], "bf16")
    at = torch.tensor([Lk - 100], dtype=torch.int32, device="cuda")
    for n in (1, 100):
        q = near["q"][:, :, -n:].contiguous()
        kw = dict(causal=True, q_pos=at + 100 - n, with_lse=True)
        a = dsp.dsp_attn_relpos(q, k, v, H, H, bias, bk, **kw)
        b = dsp.dsp_attn_relpos(q, near["k"], near["v"], H, H, bias, bk, **kw)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(a, b)), n
    kw = dict(causal=True, q_pos=at)
    dk, dv = far(torch.zeros_like(near["k"])), far(torch.zeros_like(near["k"]))
    got = dsp.dsp_attn_relpos_bwd(q, k, v, a[0], do, a[1], H, H, bias, bk, dk=dk, dv=dv, **kw)
    want = dsp.dsp_attn_relpos_bwd(q, near["k"], near["v"], a[0], do, a[1], H, H, bias, bk, **kw)
    torch.cuda.synchronize()
    for x, y in zip(got, want):
        assert torch.equal(x, y)


def test_no_units(torch):
    import paper_2403_10266_amd as dsp
    z = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    bias, bk = z(4, 2) + 1, dsp.dsp_relpos_buckets(3, 4).cuda()
    for B, X in ((0, 2), (2, 0)):
        q, k = z(B, X, 3, 16), z(B, X, 5, 16)
        o, lse = dsp.dsp_attn_relpos(q, k, k, 2, 2, bias, bk, with_lse=True)
        *_, db = dsp.dsp_attn_relpos_bwd(q, k, k, q, q, lse, 2, 2, bias, bk, dbias=z(4, 2) + 9)
        torch.cuda.synchronize()
        assert o.shape == q.shape and not db.any()


@pytest.mark.parametrize("L,Lk,M,causal", [(384, 384, 16, True), (700, 116, 200, False)])
def test_the_bias_gradient_is_rounded_once(torch, L, Lk, M, causal):
    """The rows of dZ add up to nothing, so the sums of long buckets cancel: in bf16 they
    still carry the rounding of the result, at most 2^-8 of it, and fp32 errors (2^-12)
    alone."""
    import paper_2403_10266_amd as dsp
    c = ru.case(1, 4, L, Lk, 4, 4, 40, M, 8, "bf16", seed=28)
    c["buckets"] = dsp.dsp_relpos_buckets(M, 8, not causal).numpy()
    got = host(_run(torch, c, "bf16", causal=causal)["dbias"])
    want = ru.wanted(c, "bf16", causal)["dbias"][0]
    assert np.linalg.norm(got - want) <= (2.0 ** -8 + 2.0 ** -12) * np.linalg.norm(want)
