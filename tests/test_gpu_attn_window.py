"""Windowed attention on the GPU, forward and gradients, against the oracle with the
tolerances of tests/window_util.py."""
import numpy as np
import pytest

from tests import window_util as wu
from tests.gpu_util import dev, host, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


def _i32(torch, a):
    return None if a is None else torch.tensor(a, dtype=torch.int32, device="cuda")


def _run(torch, c, dtype, left=-1, right=-1, sinks=0, q_pos=None, kv_len=None, scale=0.0, grads=True, put=None):
    import paper_2403_10266_amd as dsp
    put = put or (lambda t, n: dev(t, dtype))
    q, k, v = (put(c[n], n) for n in "qkv")
    kw = dict(left=left, right=right, sinks=sinks, q_pos=_i32(torch, q_pos), kv_len=_i32(torch, kv_len), scale=scale)
    o, lse = dsp.dsp_attn_window(q, k, v, c["H"], c["Hkv"], with_lse=True, **kw)
    got = dict(o=o, lse=lse)
    if grads:
        got |= dict(zip(("dq", "dk", "dv"), dsp.dsp_attn_window_bwd(q, k, v, o, dev(c["do"], dtype), lse, c["H"], c["Hkv"],
                                                                    **kw)))
    torch.cuda.synchronize()
    return got


def _check(torch, c, dtype, what, scale=None, **kw):
    say(what, dtype, kw)
    got = _run(torch, c, dtype, scale=scale or 0.0, **kw)
    kw.pop("put", None)
    want = wu.wanted(c, dtype, scale=scale, **kw)
    wu.compare({n: host(t) for n, t in got.items()}, want, say)
    return got


CASES = [
    # B, X, Lq, Lk, H, Hkv, D, left, right, sinks, q_pos, kv_len
    (1, 2, 64, 64, 2, 2, 72, 16, 16, 1, None, None),
    (2, 3, 32, 32, 4, 4, 72, 5, 0, 0, None, None),
    (1, 4, 17, 17, 2, 2, 64, 3, 2, 4, None, None),
    (2, 1, 150, 150, 2, 1, 72, 40, 0, 3, None, [150, 61]),
    (3, 1, 70, 90, 4, 2, 64, 30, 30, 2, None, [0, 90, 33]),       # no keys at all; odd lengths
    (2, 1, 40, 200, 2, 2, 80, 64, 0, 7, [160, 30], [200, 70]),    # positions inside a cache
    (1, 2, 33, 65, 2, 1, 128, 10, 10, 0, [-40], None),            # queries before the keys: rows that see nothing
    (2, 1, 65, 33, 2, 2, 32, 8, 0, 2, [-20, 25], None),           # rows before the first key, and past the last
    (1, 1, 300, 300, 4, 2, 40, 100, 0, 40, None, None),           # sinks past a tile
    (1, 1, 260, 260, 1, 1, 96, -1, 0, 0, None, None),             # causal without a window
    (1, 2, 129, 257, 2, 2, 16, -1, -1, 0, None, None),            # no bounds
    (1, 1, 129, 257, 2, 2, 16, -1, 30, 5, [60], None),
    (1, 3, 1, 1, 2, 1, 72, 4, 0, 1, None, None),
    (1, 2, 5, 1, 2, 2, 64, 1, 1, 0, None, None),
    (1, 1, 100, 40, 3, 1, 24, 0, 0, 0, None, None),               # each query its own key, and then none
    (1, 1, 40, 300, 8, 2, 48, 20, 0, 300, [260], None),           # sinks are all keys
    (1, 1, 700, 700, 2, 1, 64, 64, 0, 4, None, None),             # sinks' gradients in parts
    (2, 1, 1500, 1500, 3, 1, 32, 33, 5, 130, None, [1500, 1400]),  # two blocks of sinks in parts
    (1, 1, 90, 500, 2, 2, 64, 7, 3, 2, [300], None),              # keys before every window
    (1, 1, 50, 50, 6, 1, 56, 2147483647, 2147483647, 2147483647, None, None),
    (1, 2, 3, 40, 4, 4, 64, 12, 0, 2, [37], None),                # few queries
    (2, 1, 2, 3000, 8, 2, 72, -1, 0, 0, [2998, 1499], [3000, 1501]),
    (2, 1, 1, 2500, 8, 2, 128, 1000, 0, 4, [2499, 700], [2500, 701]),
    (1, 1, 1, 9000, 32, 1, 64, -1, -1, 0, None, None),            # many parts, 32 heads in a block
    (1, 1, 2, 200, 40, 1, 64, 50, 0, 0, [198], None),             # a group of more heads than a block has columns
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,X,Lq,Lk,H,Hkv,D,left,right,sinks,q_pos,kv_len", CASES)
def test_against_the_oracle(torch, dtype, B, X, Lq, Lk, H, Hkv, D, left, right, sinks, q_pos, kv_len):
    c = wu.case(B, X, Lq, Lk, H, Hkv, D, dtype, seed=Lq + D)
    _check(torch, c, dtype, f"window B{B} X{X} {Lq}x{Lk} H{H}/{Hkv} D{D}", left=left, right=right, sinks=sinks, q_pos=q_pos,
           kv_len=kv_len)


@pytest.mark.parametrize("D", [1, 3, 20, 70])
def test_odd_widths_f32(torch, D):
    c = wu.case(1, 2, 37, 45, 2, 1, D, "f32", seed=D)
    _check(torch, c, "f32", f"window D{D}", left=9, right=3, sinks=2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("seed", range(4))
def test_every_edge(torch, dtype, seed):
    """Windows whose edges fall on, before and after the tiles' and groups' borders."""
    r = np.random.default_rng(100 + seed)
    for _ in range(6):
        L, D = int(r.integers(1, 200)), int(r.choice([16, 40, 72]))
        left, right = (int(r.choice([-1, 0, 1, 14, 15, 16, 17, 31, 32, 33, 63, 64, 65])) for _ in range(2))
        sinks, pos = int(r.choice([0, 1, 15, 16, 17, 33])), int(r.integers(-40, 200))
        c = wu.case(1, 1, L, 190, 2, 1, D, dtype, seed=L)
        _check(torch, c, dtype, f"window {L}x190 D{D}", left=left, right=right, sinks=sinks, q_pos=[pos],
               kv_len=[int(r.integers(1, 191))])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Lq,Lk", [(2, 150), (90, 150)])
def test_what_no_query_sees_may_hold_anything(torch, dtype, Lq, Lk):
    """NaN and infinities behind kv_len, before the first window and after the last change
    nothing; their gradients are 0."""
    kw = dict(left=20, right=3, sinks=2, q_pos=[50], kv_len=[Lk - 8])
    c = wu.case(1, 2, Lq, Lk, 4, 2, 72, dtype, seed=3)
    want = _run(torch, c, dtype, **kw)
    last = min(50 + Lq - 1 + 3, Lk - 9)
    gone = [j for j in range(Lk) if j > last or (2 <= j < 30)]
    d = {n: t.copy() for n, t in c.items() if isinstance(t, np.ndarray)} | dict(H=4, Hkv=2)
    for i, j in enumerate(gone):
        d["k"][:, :, j] = (np.nan, np.inf, -np.inf)[i % 3]
        d["v"][:, :, j] = (np.inf, np.nan)[i % 2]
    got = _run(torch, d, dtype, **kw)
    for n in want:
        assert torch.equal(got[n], want[n]), n
    for n in ("dk", "dv"):
        assert not got[n][:, :, gone].any()


@pytest.mark.parametrize("Lq", [2, 70])
def test_a_query_that_is_not_finite_keeps_to_its_row(torch, Lq):
    import paper_2403_10266_amd as dsp
    c = wu.case(1, 2, Lq, 100, 4, 2, 72, "bf16", seed=4)
    kw = dict(left=30, right=0, sinks=1, q_pos=_i32(torch, [60]))
    q, k, v = (dev(c[n], "bf16") for n in "qkv")
    o, lse = dsp.dsp_attn_window(q, k, v, 4, 2, with_lse=True, **kw)
    q[0, 1, 1, 72:144] = float("nan")
    p, lsp = dsp.dsp_attn_window(q, k, v, 4, 2, with_lse=True, **kw)
    assert p[0, 1, 1, 72:144].isnan().all() and lsp[0, 1, 1, 1].isnan()
    p[0, 1, 1, 72:144], lsp[0, 1, 1, 1] = o[0, 1, 1, 72:144], lse[0, 1, 1, 1]
    assert torch.equal(p, o) and torch.equal(lsp, lse)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scores_of_any_size(torch, dtype):
    """Scores that climb along the keys, so that the softmax's reference moves at every tile,
    and ones far above those that a later window keeps."""
    c = wu.case(1, 1, 200, 200, 2, 2, 64, dtype, seed=5)
    ramp = np.linspace(0, 40, 200)
    for sign in (1, -1):
        c["q"][..., 0] = c["q"][..., 64] = 8.0
        c["k"][..., 0] = c["k"][..., 64] = wu.synth.bf16_round((sign * ramp).astype(np.float32))
        _check(torch, c, dtype, "ramp", left=50, right=0, sinks=1)


def _strided(torch, dtype):
    """Puts tensors into views: rows with gaps, units in another order."""
    def put(t, n):
        t = dev(t, dtype)
        B, X, L, C = t.shape
        if n == "q":       # columns of wider rows
            wide = torch.full((B, X, L, C + 64), 9.0, dtype=t.dtype, device="cuda")
            wide[..., 16:16 + C] = t
            return wide[..., 16:16 + C]
        return t.permute(1, 2, 0, 3).contiguous().permute(2, 0, 1, 3)
    return put


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Lq", [3, 100])
def test_views(torch, dtype, Lq):
    c = wu.case(2, 3, Lq, 130, 4, 2, 40, dtype, seed=6)
    _check(torch, c, dtype, "views", left=17, right=2, sinks=2, q_pos=[10, 60], put=_strided(torch, dtype))


@pytest.mark.parametrize("Lq", [2, 80])
def test_broadcast_keys(torch, Lq):
    """One text sequence for every unit: strides of 0, forward only."""
    import paper_2403_10266_amd as dsp
    c = wu.case(1, 1, 1, 60, 2, 2, 72, "bf16", seed=7)
    q = dev(wu.draw((2, 3, Lq, 144), "bf16", np.random.default_rng(1)), "bf16")
    k, v = (dev(c[n], "bf16").expand(2, 3, 60, 144) for n in "kv")
    o = dsp.dsp_attn_window(q, k, v, 2, 2, 9, 9, 1)
    assert torch.equal(o, dsp.dsp_attn_window(q, k.contiguous(), v.contiguous(), 2, 2, 9, 9, 1))
    with pytest.raises(ValueError, match="broadcasts"):
        dsp.dsp_attn_window_bwd(q, k, v, o, o, torch.zeros(2, 3, 2, Lq, device="cuda"), 2, 2, 9, 9, 1)


def test_packed_projection_gradients(torch):
    """q, k and v as columns of one projection: new gradients are columns of one buffer."""
    import paper_2403_10266_amd as dsp
    c = wu.case(1, 2, 60, 60, 2, 2, 72, "bf16", seed=8)
    kw = dict(left=11, right=4, sinks=1)
    want = _run(torch, c, "bf16", **kw)
    qkv = torch.cat([dev(c[n], "bf16") for n in "qkv"], -1)
    q, k, v = qkv.split(144, -1)
    o, lse = dsp.dsp_attn_window(q, k, v, 2, 2, with_lse=True, **kw)
    dq, dk, dv = dsp.dsp_attn_window_bwd(q, k, v, o, dev(c["do"], "bf16"), lse, 2, 2, **kw)
    assert dq.stride() == q.stride() and len({t.untyped_storage().data_ptr() for t in (dq, dk, dv)}) == 1
    for n, t in dict(o=o, lse=lse, dq=dq, dk=dk, dv=dv).items():
        assert torch.equal(t, want[n]), n


def test_far_positions(torch):
    """A cache whose offsets pass 32 bits: 9 units of 2^28 elements, the last one's keys read
    at the end of a long sequence; memory is shared by strides, so little of it is touched."""
    import paper_2403_10266_amd as dsp
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB of free GPU memory")
    L, C = 1 << 21, 128
    k = torch.empty(9, 1, L, C, dtype=torch.bfloat16, device="cuda")
    assert k.numel() > 2 ** 31
    c = wu.case(1, 1, 3, 200, 2, 2, 64, "bf16", seed=9)
    k[8, 0, L - 200:] = dev(c["k"], "bf16")[0, 0]
    v = k                                    # one tensor for both: values are the keys
    c["v"] = c["k"]
    pos, lens = [0] * 8 + [L - 3], [0] * 8 + [L]
    q = torch.zeros(9, 1, 3, C, dtype=torch.bfloat16, device="cuda")
    q[8] = dev(c["q"], "bf16")[0]
    o, lse = dsp.dsp_attn_window(q, k, v, 2, 2, 150, 0, 0, _i32(torch, pos), _i32(torch, lens), with_lse=True)
    want = wu.wanted(c, "bf16", 150, 0, 0, [197], [200], grads=False)
    wu.compare(dict(o=host(o[8:]), lse=host(lse[8:])), want, say)
    assert not o[:8].any() and (lse[:8] == -np.inf).all()


def test_same_bits_again(torch):
    c = wu.case(2, 1, 900, 900, 4, 2, 64, "bf16", seed=10)
    kw = dict(left=70, right=0, sinks=4, kv_len=[900, 700])
    a, b = (_run(torch, c, "bf16", **kw) for _ in range(2))
    assert all(torch.equal(a[n], b[n]) for n in a)


def test_no_queries_give_zero_gradients(torch):
    import paper_2403_10266_amd as dsp
    k = torch.randn(1, 2, 30, 128, device="cuda").bfloat16()
    q = k.new_empty(1, 2, 0, 128)
    dq, dk, dv = dsp.dsp_attn_window_bwd(q, k, k.clone(), q, q, torch.empty(1, 2, 2, 0, device="cuda"), 2, 2, 5, 0, 1)
    assert not dk.any() and not dv.any() and dq.numel() == 0


@pytest.mark.parametrize("Lq,Lk", [(1, 3000), (150, 150)])
def test_captured_and_on_another_stream(torch, Lq, Lk):
    """A graph of the forward (and gradients) replays with changed inputs, with eager calls of
    other inputs between the replays; the same call on a stream of its own."""
    import paper_2403_10266_amd as dsp
    cs = [wu.case(1, 2, Lq, Lk, 4, 2, 72, "bf16", seed=20 + i) for i in range(3)]
    kw = dict(left=-1 if Lq == 1 else 40, right=0, sinks=3)
    pos = _i32(torch, [Lk - Lq])
    put = lambda c: [dev(c[n], "bf16") for n in ("q", "k", "v", "do")]  # noqa: E731

    def call(t, stream=None):
        o, lse = dsp.dsp_attn_window(t[0], t[1], t[2], 4, 2, q_pos=pos, with_lse=True, stream=stream, **kw)
        if Lq == 1:
            return [o, lse]
        return [o, lse, *dsp.dsp_attn_window_bwd(t[0], t[1], t[2], o, t[3], lse, 4, 2, q_pos=pos, stream=stream, **kw)]

    want = [[x.clone() for x in call(put(c))] for c in cs]
    t = put(cs[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = call(t, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want[0]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call(t)
    for i in (1, 2, 0, 1):
        for x, y in zip(t, put(cs[i])):
            x.copy_(y)
        graph.replay()
        call(put(cs[(i + 1) % 3]))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want[i])), i


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Lq,Lk,at", [(3, 900, 700), (100, 100, 70), (400, 400, 250)])
def test_a_key_that_is_not_finite_shows(torch, dtype, Lq, Lk, at):
    """A NaN in a key, wherever the pass over the keys meets it, is in every query that sees the
    key, and not in another unit."""
    import paper_2403_10266_amd as dsp
    c = wu.case(1, 2, Lq, Lk, 4, 2, 72, dtype, seed=30)
    q, k, v = (dev(c[n], dtype) for n in "qkv")
    kw = dict(left=-1, right=0, q_pos=_i32(torch, [Lk - Lq]), with_lse=True)
    o, lse = dsp.dsp_attn_window(q, k, v, 4, 2, **kw)
    k[0, 1, at, 3] = float("nan")
    p, lsp = dsp.dsp_attn_window(q, k, v, 4, 2, **kw)
    first = max(at - (Lk - Lq), 0)
    seen = p.reshape(2, Lq, 2, 2, 72)[1, first:, 0]       # heads of the key's head
    assert seen.isnan().all() and lsp[0, 1, :2, first:].isnan().all()
    assert torch.equal(p[0, 0], o[0, 0]) and torch.equal(lsp[0, 0], lse[0, 0])
    assert torch.equal(p[0, 1, :, 144:], o[0, 1, :, 144:]) and torch.equal(lsp[0, 1, 2:], lse[0, 1, 2:])


SHORT = [
    # B, X, Lq, Lk, H, Hkv, D, left, right, sinks, q_pos, kv_len
    (1, 5, 32, 32, 2, 2, 64, 8, 0, 0, None, None),                # one wave, full
    (2, 3, 8, 31, 4, 1, 72, -1, 0, 2, [23, -3], [31, 7]),         # a group of 4 heads in a block
    (1, 4, 33, 20, 2, 2, 40, 5, 5, 1, None, None),                # more columns than keys
    (2, 2, 16, 64, 8, 2, 96, 30, 2, 3, [40, 60], [64, 0]),        # a unit without keys
    (1, 3, 64, 64, 2, 2, 128, 16, 16, 0, None, None),
    (1, 3, 32, 100, 4, 1, 64, 20, 0, 5, [68], None),              # 128 columns
    (1, 2, 128, 128, 1, 1, 72, 16, 16, 1, None, None),
    (1, 2, 128, 128, 2, 2, 16, -1, -1, 0, None, None),
    (1, 2, 1, 128, 6, 2, 48, 40, 0, 130, [127], None),
    (1, 2, 127, 1, 2, 2, 80, 3, 200, 0, [-90], None),
    (1, 2, 129, 128, 2, 2, 72, 16, 16, 1, None, None),            # one more than fits
    (1, 2, 43, 128, 3, 1, 32, 60, 0, 0, [80], None),              # 129 columns of a group
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,X,Lq,Lk,H,Hkv,D,left,right,sinks,q_pos,kv_len", SHORT)
def test_short_units(torch, dtype, B, X, Lq, Lk, H, Hkv, D, left, right, sinks, q_pos, kv_len):
    c = wu.case(B, X, Lq, Lk, H, Hkv, D, dtype, seed=Lq + Lk)
    _check(torch, c, dtype, f"short B{B} X{X} {Lq}x{Lk} H{H}/{Hkv} D{D}", left=left, right=right, sinks=sinks, q_pos=q_pos,
           kv_len=kv_len)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,X,L,H,Hkv,D", [(2, 3, 600, 4, 2, 64), (1, 5, 641, 3, 3, 72), (1, 1, 900, 2, 1, 128),
                                           (3, 1, 530, 4, 4, 96), (1, 9, 257, 8, 8, 8)])
def test_blocks_in_runs(torch, dtype, B, X, L, H, Hkv, D):
    """Enough blocks of a narrow window that neighbouring ones go to one place together."""
    c = wu.case(B, X, L, L, H, Hkv, D, dtype, seed=L)
    _check(torch, c, dtype, f"runs B{B} X{X} {L} H{H}/{Hkv} D{D}", left=33, right=20, sinks=2)


def test_two_at_once(torch):
    """Two streams, and two graphs replayed in turn and together, with workspaces of their own."""
    import paper_2403_10266_amd as dsp
    cs = [wu.case(1, 1, L, n, 8, 2, 64, "bf16", seed=40 + i) for i, (L, n) in enumerate([(2, 5000), (300, 300)])]
    kw = [dict(left=-1, right=0, q_pos=_i32(torch, [4998])), dict(left=30, right=0, sinks=2)]
    ts = [[dev(c[n], "bf16") for n in ("q", "k", "v", "do")] for c in cs]

    def call(i, stream=None):
        q, k, v, do = ts[i]
        o, lse = dsp.dsp_attn_window(q, k, v, 8, 2, with_lse=True, stream=stream, **kw[i])
        return [o, lse, *dsp.dsp_attn_window_bwd(q, k, v, o, do, lse, 8, 2, stream=stream, **kw[i])]

    want = [[x.clone() for x in call(i)] for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(4):
        got = [call(i, streams[i]) for i in range(2)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))
    graphs, outs = [], []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(call(i))
        graphs.append(g)
    for together in (False, True, False, True):
        for o in outs:
            for x in o:
                x.fill_(7)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s if together else streams[0]):
                g.replay()
        call(0)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(outs, want) for a, b in zip(g, w))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,Lq,Lk,H,Hkv,D,left,right,sinks", [
    (1, 16, 3000, 8, 2, 64, -1, 0, 0), (2, 33, 1500, 4, 2, 72, -1, 0, 0), (1, 3, 2500, 40, 1, 40, 1200, 0, 5),
    (1, 129, 2200, 2, 2, 128, -1, 3, 0), (1, 9, 1025, 4, 1, 96, 700, 40, 2)])
def test_several_blocks_of_columns_against_many_keys(torch, dtype, B, Lq, Lk, H, Hkv, D, left, right, sinks):
    c = wu.case(B, 1, Lq, Lk, H, Hkv, D, dtype, seed=Lq)
    _check(torch, c, dtype, f"blocks B{B} {Lq}x{Lk} H{H}/{Hkv} D{D}", left=left, right=right, sinks=sinks,
           q_pos=[Lk - Lq - 7 * b for b in range(B)], kv_len=[Lk - 7 * b for b in range(B)])
