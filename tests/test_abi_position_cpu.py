"""Refusals of the position operators, without a GPU: only calls that fail
validation (or launch nothing) are made."""
import ctypes

import pytest

import paper_2403_10266_amd as dsp

A = [0x10000000 + i * 0x10000000 for i in range(24)]   # far apart, never dereferenced
BF, F32 = dsp.DSP_BF16, dsp.DSP_F32


def _st(*v):
    return (ctypes.c_int64 * len(v))(*v)


@pytest.fixture(scope="module")
def lib():
    return dsp.lib()


def _norm(lib, bwd=False, **kw):
    """A valid call on fake pointers (B2 X3 L5, 4 and 2 heads of 72) with some
    arguments replaced; every test replaces one by something refused."""
    d = dict(q=A[0], k=A[1], yq=A[2], yk=A[3], gq=A[4], gk=A[5], cos=A[6], sin=A[7], pos=None, P=5, rot=72, flags=0,
             B=2, X=3, L=5, H=4, Hkv=2, D=72, qs=_st(15 * 288, 5 * 288, 288), ks=_st(15 * 144, 5 * 144, 144), yqs=None,
             yks=None, eps=1e-6, dt=BF, dyq=A[8], dyk=A[9], dgq=A[10], dgk=A[11], ws=A[12], nws=1 << 30)
    assert set(kw) <= set(d)
    d |= kw
    yqs, yks = (d[n] if d[n] is not None or n in kw else d[m] for n, m in (("yqs", "qs"), ("yks", "ks")))
    tail = [d["cos"], d["sin"], d["pos"], d["P"], d["rot"], d["flags"]]
    size = [d["B"], d["X"], d["L"], d["H"], d["Hkv"], d["D"]]
    if not bwd:
        return lib.dsp_qk_norm_rope(d["q"], d["k"], d["yq"], d["yk"], d["gq"], d["gk"], *tail, *size, d["qs"], d["ks"],
                                    yqs, yks, d["eps"], d["dt"], None)
    return lib.dsp_qk_norm_rope_bwd(d["q"], d["k"], d["dyq"], d["dyk"], d["yq"], d["yk"], d["dgq"], d["dgk"], d["gq"],
                                    d["gk"], *tail, d["ws"], d["nws"], *size, d["qs"], d["ks"], d["qs"], d["ks"], yqs,
                                    yks, d["eps"], d["dt"], None)


@pytest.mark.parametrize("bwd", [False, True])
@pytest.mark.parametrize("status,kw", [
    (dsp.DSP_ERR_DTYPE, dict(dt=5)),
    (dsp.DSP_ERR_NULL, dict(q=None)),
    (dsp.DSP_ERR_NULL, dict(yk=None)),
    (dsp.DSP_ERR_NULL, dict(qs=None)),
    (dsp.DSP_ERR_NULL, dict(cos=None)),
    (dsp.DSP_ERR_NULL, dict(sin=None)),
    (dsp.DSP_ERR_SHAPE, dict(B=-1)),
    (dsp.DSP_ERR_SHAPE, dict(H=0, Hkv=0)),
    (dsp.DSP_ERR_SHAPE, dict(H=-1)),
    (dsp.DSP_ERR_SHAPE, dict(D=0)),
    (dsp.DSP_ERR_SHAPE, dict(D=257)),
    (dsp.DSP_ERR_SHAPE, dict(rot=7)),
    (dsp.DSP_ERR_SHAPE, dict(rot=74)),
    (dsp.DSP_ERR_SHAPE, dict(rot=-2)),
    (dsp.DSP_ERR_SHAPE, dict(P=4)),
    (dsp.DSP_ERR_SHAPE, dict(P=0, pos=A[13])),
    (dsp.DSP_ERR_SHAPE, dict(L=1 << 31, P=1 << 31)),
    (dsp.DSP_ERR_SHAPE, dict(qs=_st(15 * 288, -1, 288))),
    (dsp.DSP_ERR_SHAPE, dict(qs=_st(1 << 62, 5 * 288, 288))),
    (dsp.DSP_ERR_ARG, dict(eps=-1.0)),
    (dsp.DSP_ERR_ARG, dict(eps=float("inf"))),
    (dsp.DSP_ERR_ARG, dict(eps=float("nan"))),
    (dsp.DSP_ERR_ARG, dict(flags=2)),
    (dsp.DSP_ERR_ALIGN, dict(q=A[0] + 1)),
    (dsp.DSP_ERR_ALIGN, dict(gq=A[4] + 1)),
    (dsp.DSP_ERR_ALIGN, dict(cos=A[6] + 2)),
    (dsp.DSP_ERR_ALIGN, dict(pos=A[13] + 2)),
    (dsp.DSP_ERR_ARG, dict(yqs=_st(15 * 288, 5 * 288, 280))),           # output rows overlap
    (dsp.DSP_ERR_ARG, dict(yq=A[0] + 16)),                              # over q, not in place
    (dsp.DSP_ERR_ARG, dict(yq=A[0], yqs=_st(15 * 296, 5 * 296, 296))),  # in place with other strides
    (dsp.DSP_ERR_ARG, dict(yq=A[1])),                                   # over k
    (dsp.DSP_ERR_ARG, dict(yk=A[2] + 144)),                             # over yq
])
def test_norm_refusals(lib, bwd, status, kw):
    assert _norm(lib, bwd, **kw) == status


def test_norm_gradient_refusals(lib):
    assert _norm(lib, True, dyq=None) == dsp.DSP_ERR_NULL
    assert _norm(lib, True, dyk=A[9] + 1) == dsp.DSP_ERR_ALIGN
    assert _norm(lib, True, dgq=A[10] + 2) == dsp.DSP_ERR_ALIGN
    assert _norm(lib, True, yq=A[9]) == dsp.DSP_ERR_ARG                  # dq over dyk
    need = lib.dsp_qk_norm_rope_bwd_workspace_bytes(2, 3, 5, 4, 2, 72)
    assert need > 0
    assert _norm(lib, True, ws=None) == dsp.DSP_ERR_WORKSPACE
    assert _norm(lib, True, nws=need - 1) == dsp.DSP_ERR_WORKSPACE
    assert _norm(lib, True, ws=A[12] + 8) == dsp.DSP_ERR_WORKSPACE
    assert lib.dsp_qk_norm_rope_bwd_workspace_bytes(1 << 40, 1 << 40, 5, 4, 2, 72) == 0
    assert lib.dsp_qk_norm_rope_bwd_workspace_bytes(2, 3, 5, 4, 2, 300) == 0


def test_norm_of_nothing(lib):
    assert _norm(lib, L=0, q=None, k=None, yq=None, yk=None) == dsp.DSP_OK
    assert _norm(lib, True, B=0, q=None, dgq=None, dgk=None, ws=None, nws=0) == dsp.DSP_OK


def test_norm_binding_refusals():
    import torch
    x = torch.zeros(1, 1, 2, 144)
    with pytest.raises(ValueError, match="device tensor"):
        dsp.dsp_qk_norm_rope(x, x, 2, 2)


def _relpos(lib, bwd=False, **kw):
    """A valid call (B2 X3, 5 queries, 7 keys, 4 and 2 heads of 72) with some arguments
    replaced."""
    d = dict(q=A[0], k=A[1], v=A[2], o=A[3], lse=A[4], bias=A[5], bk=A[6], nb=8, M=16, q_pos=None, kv_len=None, flags=0,
             ws=A[7], nws=1 << 30, B=2, X=3, Lq=5, Lk=7, H=4, Hkv=2, D=72, qs=_st(15 * 288, 5 * 288, 288),
             ks=_st(21 * 144, 7 * 144, 144), os=_st(15 * 288, 5 * 288, 288), scale=0.0, dt=BF, do=A[8], dq=A[9], dk=A[10],
             dv=A[11], db=A[12])
    assert set(kw) <= set(d)
    d |= kw
    mid = [d["bias"], d["bk"], d["nb"], d["M"], d["q_pos"], d["kv_len"], d["flags"], d["ws"], d["nws"], d["B"], d["X"],
           d["Lq"], d["Lk"], d["H"], d["Hkv"], d["D"], d["qs"], d["ks"], d["os"], d["scale"], d["dt"], None]
    if not bwd:
        return lib.dsp_attn_relpos(d["q"], d["k"], d["v"], d["o"], d["lse"], *mid)
    return lib.dsp_attn_relpos_bwd(d["q"], d["k"], d["v"], d["o"], d["do"], d["lse"], d["dq"], d["dk"], d["dv"], d["db"],
                                   *mid)


@pytest.mark.parametrize("bwd", [False, True])
@pytest.mark.parametrize("status,kw", [
    (dsp.DSP_ERR_DTYPE, dict(dt=2)),
    (dsp.DSP_ERR_NULL, dict(q=None)),
    (dsp.DSP_ERR_NULL, dict(v=None)),
    (dsp.DSP_ERR_NULL, dict(o=None)),
    (dsp.DSP_ERR_NULL, dict(bias=None)),
    (dsp.DSP_ERR_NULL, dict(bk=None)),
    (dsp.DSP_ERR_NULL, dict(ks=None)),
    (dsp.DSP_ERR_SHAPE, dict(B=-1)),
    (dsp.DSP_ERR_SHAPE, dict(H=0)),
    (dsp.DSP_ERR_SHAPE, dict(Hkv=3)),
    (dsp.DSP_ERR_SHAPE, dict(D=0)),
    (dsp.DSP_ERR_SHAPE, dict(D=136)),
    (dsp.DSP_ERR_SHAPE, dict(D=70)),                        # bf16: multiples of 8
    (dsp.DSP_ERR_SHAPE, dict(D=129, dt=F32)),
    (dsp.DSP_ERR_SHAPE, dict(nb=0)),
    (dsp.DSP_ERR_SHAPE, dict(M=-1)),
    (dsp.DSP_ERR_SHAPE, dict(M=1025)),
    (dsp.DSP_ERR_SHAPE, dict(Lq=1 << 30)),
    (dsp.DSP_ERR_SHAPE, dict(Lk=1 << 30)),
    (dsp.DSP_ERR_SHAPE, dict(B=1 << 20, X=1 << 20)),
    (dsp.DSP_ERR_SHAPE, dict(ks=_st(21 * 144, 7 * 144, -8))),
    (dsp.DSP_ERR_SHAPE, dict(ks=_st(1 << 40, 1 << 30, 1 << 24))),   # 64 rows past 2^31 bytes
    (dsp.DSP_ERR_SHAPE, dict(qs=_st(1 << 40, 1 << 30, 1 << 24))),
    (dsp.DSP_ERR_SHAPE, dict(os=_st(1 << 40, 1 << 30, 1 << 24))),
    (dsp.DSP_ERR_ARG, dict(scale=float("nan"))),
    (dsp.DSP_ERR_ARG, dict(scale=float("inf"))),
    (dsp.DSP_ERR_ARG, dict(flags=2)),
    (dsp.DSP_ERR_ALIGN, dict(q=A[0] + 8)),
    (dsp.DSP_ERR_ALIGN, dict(k=A[1] + 1)),
    (dsp.DSP_ERR_ALIGN, dict(bias=A[5] + 1)),
    (dsp.DSP_ERR_ALIGN, dict(bk=A[6] + 2)),
    (dsp.DSP_ERR_ALIGN, dict(q_pos=A[13] + 2)),
    (dsp.DSP_ERR_ALIGN, dict(kv_len=A[13] + 1)),
    (dsp.DSP_ERR_ALIGN, dict(lse=A[4] + 2)),
    (dsp.DSP_ERR_ALIGN, dict(qs=_st(15 * 288, 5 * 288, 292))),
])
def test_relpos_refusals(lib, bwd, status, kw):
    assert _relpos(lib, bwd, **kw) == status


def test_relpos_output_overlaps(lib):
    assert _relpos(lib, o=A[0]) == dsp.DSP_ERR_ARG
    assert _relpos(lib, o=A[2]) == dsp.DSP_ERR_ARG
    assert _relpos(lib, os=_st(15 * 288, 5 * 288, 280)) == dsp.DSP_ERR_ARG
    for kw in (dict(dq=A[0]), dict(dk=A[1]), dict(dv=A[10]), dict(dq=A[3]), dict(dk=A[8]), dict(db=A[5]),
               dict(ks=_st(21 * 144, 0, 144)), dict(qs=_st(0, 5 * 288, 288))):
        assert _relpos(lib, True, **kw) == dsp.DSP_ERR_ARG, kw


def test_relpos_gradient_refusals(lib):
    for n in ("do", "dq", "dk", "dv", "db", "lse"):
        assert _relpos(lib, True, **{n: None}) == dsp.DSP_ERR_NULL, n
    need = lib.dsp_attn_relpos_bwd_workspace_bytes(2, 3, 5, 7, 4, 2, 72, 16, BF)
    assert need >= 2 * 3 * 4 * 5 * 4
    for kw in (dict(ws=None), dict(nws=need - 1), dict(ws=A[7] + 8)):
        assert _relpos(lib, True, **kw) == dsp.DSP_ERR_WORKSPACE, kw
    assert _relpos(lib, True, qs=_st(15 << 30, 5 << 26, 1 << 26), Lq=5) == dsp.DSP_ERR_SHAPE


def test_relpos_workspaces(lib):
    size = lib.dsp_attn_relpos_workspace_bytes
    assert size(2, 1, 1, 100, 8, 2, 72, BF) == 0 and size(2, 1, 300, 5000, 8, 2, 72, BF) == 0
    need = size(2, 1, 1, 5000, 8, 2, 72, BF)
    assert need > 0
    long = dict(X=1, Lq=1, Lk=5000, H=8, Hkv=2, qs=_st(576, 576, 576), os=_st(576, 576, 576), ks=_st(5000 * 144, 5000 * 144, 144))
    for kw in (dict(ws=None), dict(nws=need - 1)):
        assert _relpos(lib, **long, **kw) == dsp.DSP_ERR_WORKSPACE
    assert size(1, 1, 1, 5000, 8, 3, 72, BF) == 0 and size(-1, 1, 1, 5000, 8, 2, 72, BF) == 0


def test_relpos_of_nothing(lib):
    assert _relpos(lib, Lq=0, q=None, o=None, lse=None) == dsp.DSP_OK
    assert _relpos(lib, B=0, q=None, k=None, v=None, o=None, bias=None, bk=None) == dsp.DSP_OK


def test_buckets_refusals(lib):
    buf = (ctypes.c_int32 * 9)()
    assert lib.dsp_relpos_buckets(None, 4, 8, 1) == dsp.DSP_ERR_NULL
    assert lib.dsp_relpos_buckets(buf, -1, 8, 1) == dsp.DSP_ERR_SHAPE
    assert lib.dsp_relpos_buckets(buf, 1025, 8, 1) == dsp.DSP_ERR_SHAPE
    assert lib.dsp_relpos_buckets(buf, 4, 1, 1) == dsp.DSP_ERR_SHAPE
    assert lib.dsp_relpos_buckets(buf, 4, 0, 0) == dsp.DSP_ERR_SHAPE
    assert lib.dsp_relpos_buckets(buf, 4, 1, 0) == dsp.DSP_OK and not any(buf)
    with pytest.raises(ValueError):
        dsp.dsp_relpos_buckets(-1, 8)


@pytest.mark.parametrize("M,nb", [(8, 4), (128, 32), (128, 8), (40, 15), (200, 33), (1024, 64)])
@pytest.mark.parametrize("both", [False, True])
def test_buckets_follow_the_oracle(M, nb, both):
    from oracle import position as po
    assert dsp.dsp_relpos_buckets(M, nb, both).tolist() == po.relpos_buckets(M, nb, both).tolist()


def test_relpos_binding_refusals():
    import torch
    x = torch.zeros(1, 1, 2, 144)
    with pytest.raises(ValueError, match="device tensor"):
        dsp.dsp_attn_relpos(x, x, x, 2, 2, torch.zeros(3, 2), torch.zeros(5, dtype=torch.int32))


def test_rows_between_rows_of_uneven_pitch(lib):
    """Outputs in the gaps between the inputs' rows share no element only where every
    stride is whole pitches; here x's second run of rows starts inside a gap."""
    uneven, even = _st(10000, 2688, 600), _st(10000, 3000, 600)
    for es, dt in ((2, BF), (4, F32)):
        assert _norm(lib, qs=uneven, yq=A[0] + 300 * es, dt=dt) == dsp.DSP_ERR_ARG
        assert _norm(lib, qs=even, yq=A[0] + 300 * es, dt=dt, cos=None) == dsp.DSP_ERR_NULL
        assert _norm(lib, qs=even, yq=A[0] + 313 * es, dt=dt) == dsp.DSP_ERR_ARG
