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
