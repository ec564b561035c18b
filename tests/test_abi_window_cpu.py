"""Refusals of windowed attention and of the paged cache, without a GPU: only calls that
fail validation (or launch nothing) are made."""
import ctypes

import pytest

import paper_2403_10266_amd as dsp

A = [0x10000000 + i * 0x10000000 for i in range(24)]   # far apart, never dereferenced
BF, F32, E4 = dsp.DSP_BF16, dsp.DSP_F32, dsp.DSP_E4M3


def _st(*v):
    return (ctypes.c_int64 * len(v))(*v)


@pytest.fixture(scope="module")
def lib():
    return dsp.lib()


def _window(lib, bwd=False, **kw):
    """A valid call (B2 X3, 5 queries, 7 keys, 4 and 2 heads of 72) with some arguments
    replaced; every test replaces one by something refused."""
    d = dict(q=A[0], k=A[1], v=A[2], o=A[3], lse=A[4], q_pos=None, kv_len=None, left=3, right=0, sinks=1, ws=A[7],
             nws=1 << 30, B=2, X=3, Lq=5, Lk=7, H=4, Hkv=2, D=72, qs=_st(15 * 288, 5 * 288, 288),
             ks=_st(21 * 144, 7 * 144, 144), os=None, scale=0.0, dt=BF, do=A[8], dq=A[9], dk=A[10], dv=A[11])
    assert set(kw) <= set(d)
    d |= kw
    os_ = d["os"] if d["os"] is not None or "os" in kw else d["qs"]
    tail = [d["q_pos"], d["kv_len"], d["left"], d["right"], d["sinks"], d["ws"], d["nws"], d["B"], d["X"], d["Lq"], d["Lk"],
            d["H"], d["Hkv"], d["D"], d["qs"], d["ks"], os_, d["scale"], d["dt"], None]
    if not bwd:
        return lib.dsp_attn_window(d["q"], d["k"], d["v"], d["o"], d["lse"], *tail)
    return lib.dsp_attn_window_bwd(d["q"], d["k"], d["v"], d["o"], d["do"], d["lse"], d["dq"], d["dk"], d["dv"], *tail)


@pytest.mark.parametrize("bwd", [False, True])
@pytest.mark.parametrize("status,kw", [
    (dsp.DSP_ERR_DTYPE, dict(dt=7)),
    (dsp.DSP_ERR_DTYPE, dict(dt=E4)),
    (dsp.DSP_ERR_NULL, dict(q=None)),
    (dsp.DSP_ERR_NULL, dict(v=None)),
    (dsp.DSP_ERR_NULL, dict(o=None)),
    (dsp.DSP_ERR_NULL, dict(ks=None)),
    (dsp.DSP_ERR_NULL, dict(os=None)),
    (dsp.DSP_ERR_SHAPE, dict(X=-1)),
    (dsp.DSP_ERR_SHAPE, dict(Hkv=3)),
    (dsp.DSP_ERR_SHAPE, dict(H=1 << 15, Hkv=1)),
    (dsp.DSP_ERR_SHAPE, dict(Hkv=0)),
    (dsp.DSP_ERR_SHAPE, dict(D=132)),
    (dsp.DSP_ERR_SHAPE, dict(D=68)),
    (dsp.DSP_ERR_SHAPE, dict(D=0)),
    (dsp.DSP_ERR_SHAPE, dict(Lk=1 << 30)),
    (dsp.DSP_ERR_SHAPE, dict(Lq=(1 << 30) - 1, H=8, Hkv=1)),
    (dsp.DSP_ERR_SHAPE, dict(qs=_st(-8, 5 * 288, 288))),
    (dsp.DSP_ERR_SHAPE, dict(qs=_st(15 * 288, 5 * 288, 1 << 24))),
    (dsp.DSP_ERR_ARG, dict(sinks=-1)),
    (dsp.DSP_ERR_ARG, dict(scale=float("nan"))),
    (dsp.DSP_ERR_ARG, dict(scale=float("inf"))),
    (dsp.DSP_ERR_ALIGN, dict(q=A[0] + 8)),
    (dsp.DSP_ERR_ALIGN, dict(k=A[1] + 2)),
    (dsp.DSP_ERR_ALIGN, dict(ks=_st(21 * 148, 7 * 148, 148))),
    (dsp.DSP_ERR_ALIGN, dict(lse=A[4] + 2)),
    (dsp.DSP_ERR_ALIGN, dict(q_pos=A[13] + 1)),
    (dsp.DSP_ERR_ALIGN, dict(kv_len=A[13] + 1)),
])
def test_window_refusals(lib, bwd, status, kw):
    assert _window(lib, bwd, **kw) == status


def test_window_overlaps(lib):
    for name in ("o", "lse"):
        for at in [A[0], A[1], A[2], A[13], A[14]] + ([A[4]] if name == "o" else []):
            assert _window(lib, q_pos=A[13], kv_len=A[14], **{name: at}) == dsp.DSP_ERR_ARG, (name, hex(at))
    assert _window(lib, os=_st(15 * 288, 5 * 288, 280)) == dsp.DSP_ERR_ARG          # output rows overlap
    for name in ("dq", "dk", "dv"):
        for at in (A[0], A[1], A[2], A[3], A[4], A[8], A[13], A[14], *(A[i] for i in (9, 10, 11))):
            if {"dq": A[9], "dk": A[10], "dv": A[11]}[name] != at:
                assert _window(lib, True, q_pos=A[13], kv_len=A[14], **{name: at}) == dsp.DSP_ERR_ARG, (name, hex(at))
    assert _window(lib, True, ks=_st(0, 7 * 144, 144)) == dsp.DSP_ERR_ARG           # broadcast keys have no gradient


LONG = dict(X=1, Lq=1, Lk=5000, H=8, Hkv=2, qs=_st(576, 576, 576), ks=_st(5000 * 144, 5000 * 144, 144), left=-1, sinks=0)


def test_window_workspaces(lib):
    need = lib.dsp_attn_window_workspace_bytes(2, 1, 1, 5000, 8, 2, 72, -1, 0, 0, BF)
    assert need > 0
    for kw in (dict(ws=None), dict(nws=need - 1), dict(ws=A[7] + 8)):
        assert _window(lib, **LONG, **kw) == dsp.DSP_ERR_WORKSPACE
    for at in (A[0], A[1], A[2], A[3], A[4], A[3] - need + 16):
        assert _window(lib, **LONG, ws=at) == dsp.DSP_ERR_ARG, hex(at)
    assert lib.dsp_attn_window_bwd_workspace_bytes(2, 3, 5, 7, 4, 2, 72, 3, 0, 1, BF) == 0     # short units need none
    need = lib.dsp_attn_window_bwd_workspace_bytes(2, 3, 5, 150, 4, 2, 72, 3, 0, 1, BF)
    assert need > 0
    more = dict(Lk=150, ks=_st(450 * 144, 150 * 144, 144))
    for kw in (dict(ws=None), dict(nws=need - 1), dict(ws=A[7] + 8)):
        assert _window(lib, True, **more, **kw) == dsp.DSP_ERR_WORKSPACE
    for at in (A[0], A[1], A[2], A[3], A[4], A[8], A[9], A[10], A[11]):
        assert _window(lib, True, **more, ws=at) == dsp.DSP_ERR_ARG, hex(at)
    assert lib.dsp_attn_window_workspace_bytes(-1, 1, 1, 5000, 8, 2, 72, -1, 0, 0, BF) == 0
    assert lib.dsp_attn_window_bwd_workspace_bytes(2, 3, 5, 7, 4, 3, 72, 3, 0, 1, BF) == 0
    # long windows and short ones; sinks that every query sees ask for partial sums
    far = [lib.dsp_attn_window_bwd_workspace_bytes(1, 1, 8000, 8000, 8, 2, 64, 200, 0, s, BF) for s in (0, 1)]
    assert far[1] > far[0] == 8 * 8000 * 4


def test_window_of_nothing(lib):
    none = dict(q=None, k=None, v=None, o=None, lse=None)
    assert _window(lib, B=0, **none) == dsp.DSP_OK
    assert _window(lib, Lq=0, **none) == dsp.DSP_OK
    assert _window(lib, True, X=0, **none, do=None, dq=None, dk=None, dv=None) == dsp.DSP_OK


def _cache_args(**kw):
    """64 pages of 32 slots, 2 heads of 72, N 3 sequences, T 10 rows, tables of 20 pages."""
    d = dict(q=A[0], k=A[1], v=A[2], o=A[3], kc=A[4], vc=A[5], ks=None, vs=None, table=A[8], start=A[9], lens=A[10],
             cos=A[11], sin=A[12], pos=None, P=700, rot=72, flags=0, N=3, T=10, n_pages=64, max_pages=20, page=32, H=4, Hkv=2,
             D=72, row=288, krow=144, vrow=144, orow=288, cs=_st(32 * 144, 144, 72), cdt=BF, dt=BF, left=-1, right=0, sinks=0,
             ws=A[13], nws=1 << 30, max_q=1, scale=0.0, lse=A[14])
    assert set(kw) <= set(d)
    return d | kw


def _append(lib, **kw):
    d = _cache_args(**kw)
    return lib.dsp_kv_append(d["k"], d["v"], d["q"], d["o"], d["kc"], d["vc"], d["ks"], d["vs"], d["table"], d["start"],
                             d["lens"], d["cos"], d["sin"], d["pos"], d["P"], d["rot"], d["flags"], d["N"], d["T"],
                             d["n_pages"], d["max_pages"], d["page"], d["H"], d["Hkv"], d["D"], d["krow"], d["vrow"],
                             d["row"], d["orow"], d["cs"], d["cdt"], d["dt"], None)


def _paged(lib, **kw):
    d = _cache_args(**kw)
    return lib.dsp_attn_paged(d["q"], d["kc"], d["vc"], d["o"], d["lse"], d["ks"], d["vs"], d["table"], d["start"],
                              d["lens"], d["left"], d["right"], d["sinks"], d["ws"], d["nws"], d["N"], d["T"], d["max_q"],
                              d["n_pages"], d["max_pages"], d["page"], d["H"], d["Hkv"], d["D"], d["row"], d["cs"],
                              d["orow"], d["scale"], d["cdt"], d["dt"], None)


COMMON = [
    (dsp.DSP_ERR_DTYPE, dict(dt=9)),
    (dsp.DSP_ERR_DTYPE, dict(cdt=F32)),
    (dsp.DSP_ERR_DTYPE, dict(dt=F32, cdt=E4)),
    (dsp.DSP_ERR_DTYPE, dict(dt=E4, cdt=E4)),
    (dsp.DSP_ERR_NULL, dict(q=None)),
    (dsp.DSP_ERR_NULL, dict(o=None)),
    (dsp.DSP_ERR_NULL, dict(kc=None)),
    (dsp.DSP_ERR_NULL, dict(vc=None)),
    (dsp.DSP_ERR_NULL, dict(table=None)),
    (dsp.DSP_ERR_NULL, dict(start=None)),
    (dsp.DSP_ERR_NULL, dict(lens=None)),
    (dsp.DSP_ERR_NULL, dict(cs=None)),
    (dsp.DSP_ERR_NULL, dict(cdt=E4)),                                   # no scales
    (dsp.DSP_ERR_NULL, dict(cdt=E4, ks=A[15])),
    (dsp.DSP_ERR_SHAPE, dict(page=24)),
    (dsp.DSP_ERR_SHAPE, dict(page=8)),
    (dsp.DSP_ERR_SHAPE, dict(page=2048)),
    (dsp.DSP_ERR_SHAPE, dict(N=-1)),
    (dsp.DSP_ERR_SHAPE, dict(N=(1 << 20) + 1)),
    (dsp.DSP_ERR_SHAPE, dict(T=-1)),
    (dsp.DSP_ERR_SHAPE, dict(T=1 << 29)),
    (dsp.DSP_ERR_SHAPE, dict(n_pages=-1)),
    (dsp.DSP_ERR_SHAPE, dict(max_pages=1 << 26)),
    (dsp.DSP_ERR_SHAPE, dict(Hkv=0)),
    (dsp.DSP_ERR_SHAPE, dict(D=0)),
    (dsp.DSP_ERR_SHAPE, dict(row=-288)),
    (dsp.DSP_ERR_SHAPE, dict(cs=_st(32 * 144, -144, 72))),
    (dsp.DSP_ERR_SHAPE, dict(cs=_st(0, 144, 72))),                      # pages over one another
    (dsp.DSP_ERR_ARG, dict(cs=_st(32 * 144, 144, 64))),                 # heads over one another
    (dsp.DSP_ERR_ARG, dict(cs=_st(31 * 144, 144, 72))),
    (dsp.DSP_ERR_ARG, dict(orow=280)),
    (dsp.DSP_ERR_ALIGN, dict(q=A[0] + 1)),
    (dsp.DSP_ERR_ALIGN, dict(kc=A[4] + 1)),
    (dsp.DSP_ERR_ALIGN, dict(table=A[8] + 2)),
    (dsp.DSP_ERR_ALIGN, dict(start=A[9] + 2)),
    (dsp.DSP_ERR_ALIGN, dict(lens=A[10] + 2)),
    (dsp.DSP_ERR_ALIGN, dict(cdt=E4, ks=A[15] + 2, vs=A[16])),
    (dsp.DSP_ERR_ARG, dict(o=A[4])),                                    # over the cache, the table, the lengths
    (dsp.DSP_ERR_ARG, dict(o=A[8])),
    (dsp.DSP_ERR_ARG, dict(o=A[9])),
    (dsp.DSP_ERR_ARG, dict(o=A[10])),
    (dsp.DSP_ERR_ARG, dict(o=A[0] + 32)),                               # over q, not in place
]


@pytest.mark.parametrize("call", [_append, _paged])
@pytest.mark.parametrize("status,kw", COMMON)
def test_page_refusals(lib, call, status, kw):
    assert call(lib, **kw) == status


@pytest.mark.parametrize("status,kw", [
    (dsp.DSP_ERR_NULL, dict(k=None)),
    (dsp.DSP_ERR_NULL, dict(v=None)),
    (dsp.DSP_ERR_NULL, dict(cos=None)),
    (dsp.DSP_ERR_SHAPE, dict(rot=3)),
    (dsp.DSP_ERR_SHAPE, dict(rot=74)),
    (dsp.DSP_ERR_SHAPE, dict(P=0)),
    (dsp.DSP_ERR_SHAPE, dict(H=-1)),
    (dsp.DSP_ERR_SHAPE, dict(D=260)),
    (dsp.DSP_ERR_SHAPE, dict(H=2044, row=2044 * 72, orow=2044 * 72)),
    (dsp.DSP_ERR_SHAPE, dict(krow=-1)),
    (dsp.DSP_ERR_ARG, dict(flags=4)),
    (dsp.DSP_ERR_ALIGN, dict(sin=A[12] + 2)),
    (dsp.DSP_ERR_ALIGN, dict(pos=A[13] + 2)),
    (dsp.DSP_ERR_ARG, dict(kc=A[1])),                                   # the cache over the new keys
    (dsp.DSP_ERR_ARG, dict(vc=A[4])),                                   # over each other
    (dsp.DSP_ERR_ARG, dict(vc=A[4] + 16)),
    (dsp.DSP_ERR_ARG, dict(vc=A[8])),
    (dsp.DSP_ERR_ARG, dict(kc=A[11])),
    (dsp.DSP_ERR_ARG, dict(cdt=E4, ks=A[4], vs=A[15])),
    (dsp.DSP_ERR_ARG, dict(cdt=E4, ks=A[15], vs=A[15] + 4)),
    (dsp.DSP_ERR_ARG, dict(o=A[0], orow=296)),                          # in place with other strides
    (dsp.DSP_ERR_ARG, dict(o=A[1])),
])
def test_append_refusals(lib, status, kw):
    assert _append(lib, **kw) == status


def test_caches_in_one_buffer(lib):
    """Keys and values that interleave, by pages, slots or heads, are apart; a launch without
    a GPU fails later than validation."""
    per = 32 * 144
    for off, cs in ((per, _st(2 * per, 144, 72)), (144, _st(2 * per, 288, 72)), (72, _st(2 * per, 288, 144))):
        assert _append(lib, N=0, vc=A[4] + 2 * off, cs=cs) == dsp.DSP_OK
        assert _append(lib, vc=A[4] + 2 * off - 16, cs=cs) == dsp.DSP_ERR_ARG
        assert _append(lib, vc=A[4] + 2 * off + 16, cs=cs) == dsp.DSP_ERR_ARG
    assert _append(lib, vc=A[4] + 2 * 63 * per, cs=_st(per, 144, 72)) == dsp.DSP_ERR_ARG


@pytest.mark.parametrize("status,kw", [
    (dsp.DSP_ERR_SHAPE, dict(H=3)),
    (dsp.DSP_ERR_SHAPE, dict(H=0)),
    (dsp.DSP_ERR_SHAPE, dict(D=68)),
    (dsp.DSP_ERR_SHAPE, dict(D=136)),
    (dsp.DSP_ERR_SHAPE, dict(max_q=-1)),
    (dsp.DSP_ERR_ARG, dict(sinks=-1)),
    (dsp.DSP_ERR_ARG, dict(scale=float("inf"))),
    (dsp.DSP_ERR_ALIGN, dict(q=A[0] + 8)),
    (dsp.DSP_ERR_ALIGN, dict(row=292, orow=296)),
    (dsp.DSP_ERR_ALIGN, dict(kc=A[4] + 8)),
    (dsp.DSP_ERR_ALIGN, dict(cs=_st(32 * 148, 148, 72))),
    (dsp.DSP_ERR_ALIGN, dict(cdt=E4, ks=A[15], vs=A[16], kc=A[4] + 4)),
    (dsp.DSP_ERR_ALIGN, dict(lse=A[14] + 2)),
    (dsp.DSP_ERR_ARG, dict(lse=A[3])),
    (dsp.DSP_ERR_ARG, dict(lse=A[4])),
    (dsp.DSP_ERR_ARG, dict(cdt=E4, ks=A[15], vs=A[16], o=A[15])),
])
def test_paged_refusals(lib, status, kw):
    assert _paged(lib, **kw) == status


def test_paged_workspace(lib):
    args = (3, 10, 1, 64, 20, 32, 4, 2, 72, -1, 0, 0, BF)
    need = lib.dsp_attn_paged_workspace_bytes(*args)
    assert need > 0
    for kw in (dict(ws=None), dict(nws=need - 1), dict(ws=A[13] + 8)):
        assert _paged(lib, **kw) == dsp.DSP_ERR_WORKSPACE
    for at in (A[0], A[3], A[4], A[5], A[8], A[9], A[10], A[14]):
        assert _paged(lib, ws=at) == dsp.DSP_ERR_ARG, hex(at)
    assert lib.dsp_attn_paged_workspace_bytes(3, 10, 1, 64, 20, 33, 4, 2, 72, -1, 0, 0, BF) == 0


def test_pages_of_nothing(lib):
    none = dict(q=None, k=None, v=None, o=None, kc=None, vc=None, table=None, start=None, lens=None, lse=None, ws=None, nws=0)
    for call in (_append, _paged):
        assert call(lib, N=0, **none) == dsp.DSP_OK
        assert call(lib, T=0, **none) == dsp.DSP_OK
    assert _paged(lib, max_q=0, **none) == dsp.DSP_OK


def test_binding_refusals():
    import torch
    x = torch.zeros(1, 1, 2, 144)
    with pytest.raises(ValueError, match="device tensor"):
        dsp.dsp_attn_window(x, x, x, 2, 2, 1, 0)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="device tensor"):
        dsp.dsp_kv_append(x[0, 0], x[0, 0], torch.zeros(3, 16, 2, 72), torch.zeros(3, 16, 2, 72), i[None], i, i[:1])
    with pytest.raises(ValueError, match="device tensor"):
        dsp.dsp_attn_paged(x[0, 0], torch.zeros(3, 16, 2, 72), torch.zeros(3, 16, 2, 72), i[None], i, i[:1], 2)


@pytest.mark.parametrize("call", [_append, _paged])
def test_a_cache_of_no_pages(lib, call):
    """No pages are a size like any other: with nothing to do the calls return, other
    arguments are checked as ever."""
    none = dict(q=None, k=None, v=None, o=None, kc=None, vc=None, table=None, start=None, lens=None, lse=None, ws=None, nws=0)
    for more in (dict(N=0), dict(T=0)):
        assert call(lib, n_pages=0, **more, **none) == dsp.DSP_OK
        assert call(lib, n_pages=0, **more, **none, cs=_st(0, 0, 0)) == dsp.DSP_ERR_SHAPE   # slots over one another
    bare = dict(n_pages=0, kc=None, vc=None)
    assert call(lib, **bare, q=None) == dsp.DSP_ERR_NULL
    assert call(lib, **bare, lens=None) == dsp.DSP_ERR_NULL
    assert call(lib, **bare, o=A[9]) == dsp.DSP_ERR_ARG
    assert call(lib, **bare, page=24) == dsp.DSP_ERR_SHAPE


def test_sinks_of_many_units_keep_no_sums(lib):
    """The partial sums of first tokens fill the chip and no more, however many units there are."""
    need = lambda X, L, left, sinks: lib.dsp_attn_window_bwd_workspace_bytes(1, X, L, L, 16, 16, 72, left, 0, sinks, BF)  # noqa: E731
    for X, L, left in ((1024, 512, 33), (64, 8000, 65)):
        assert need(X, L, left, 1) == need(X, L, left, 4) == need(X, L, left, 0) == X * 16 * L * 4
    most = 512 * 2 * 128 * 72 * 4                       # work-groups, dK and dV, keys, columns
    for X in range(1, 40):
        for sinks in (1, 300):
            assert 0 <= need(X, 9000, 50, sinks) - X * 16 * 9000 * 4 <= most, X


@pytest.mark.parametrize("Lq", [1, 3, 150])
def test_gradients_of_unequal_lengths_in_one_buffer(lib, Lq):
    """dq, dk and dv as columns of one buffer's rows where queries are fewer than keys: apart (the
    call goes on to its workspace), and refused where columns meet."""
    row, L = 288 + 2 * 144, 150
    st = _st(2 * L * row, L * row, row)
    kw = dict(B=2, X=2, Lq=Lq, Lk=L, ws=None, os=_st(2 * Lq * 288, Lq * 288, 288))
    packed = dict(qs=st, ks=st, q=A[0], k=A[0] + 2 * 288, v=A[0] + 2 * 432)
    at = lambda q, k, v: _window(lib, True, **kw, **packed, dq=A[9] + 2 * q, dk=A[9] + 2 * k, dv=A[9] + 2 * v)  # noqa: E731
    assert at(0, 288, 432) == at(288, 0, 144) == dsp.DSP_ERR_WORKSPACE
    assert at(0, 280, 432) == at(8, 288, 440) == at(296, 0, 144) == dsp.DSP_ERR_ARG
    assert at(row, 288, 432) == dsp.DSP_ERR_WORKSPACE      # a row on the columns are as far apart
    assert at(row + 8, 288, 432) == at(row + 288, 288, 432) == dsp.DSP_ERR_ARG
