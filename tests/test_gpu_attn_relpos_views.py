"""The gradient of attention with a relative position bias on views, with the gradients
that it makes by itself, and with layouts that differ only where a dimension has one
element."""
import pytest

from tests import relpos_util as ru
from tests.gpu_util import dev, host, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


def _case(torch, dtype, B=2, X=3, L=45, H=4, Hkv=4, D=24, seed=0):
    import paper_2403_10266_amd as dsp
    c = ru.case(B, X, L, L, H, Hkv, D, 16, 8, dtype, seed=seed)
    c["buckets"] = dsp.dsp_relpos_buckets(16, 8).numpy()
    return c


def _both(torch, c, q, k, v, do, **kw):
    import paper_2403_10266_amd as dsp
    bias, bk = dev(c["bias"], "bf16" if q.dtype == torch.bfloat16 else "f32"), torch.from_numpy(c["buckets"]).cuda()
    o, lse = dsp.dsp_attn_relpos(q, k, v, c["H"], c["Hkv"], bias, bk, with_lse=True)
    got = dict(zip(("dq", "dk", "dv", "dbias"),
                   dsp.dsp_attn_relpos_bwd(q, k, v, o, do(o), lse, c["H"], c["Hkv"], bias, bk, **kw)))
    torch.cuda.synchronize()
    return dict(o=o, lse=lse, **got)


def _held(c, got, dtype):
    ru.compare({n: host(t) for n, t in got.items()}, ru.wanted(c, dtype), say)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hkv", [(4, 4), (4, 2)])
def test_packed_columns_and_no_gradients_given(torch, dtype, H, Hkv):
    """q, k, v = split columns of a projection: gradients with their strides, the columns
    of one packed gradient."""
    c = _case(torch, dtype, H=H, Hkv=Hkv)
    D = 24
    buf = torch.cat([dev(c[n], dtype) for n in "qkv"], -1)
    for order in ("split", "permuted"):
        t = buf if order == "split" else buf.transpose(1, 2).contiguous().transpose(1, 2)
        q, k, v = t.split([H * D, Hkv * D, Hkv * D], dim=-1)
        got = _both(torch, c, q, k, v, lambda o: dev(c["do"], dtype))
        _held(c, got, dtype)
        for x, g in ((q, "dq"), (k, "dk"), (v, "dv")):
            assert got[g].shape == x.shape and got[g].stride() == x.stride(), g
        base = got["dq"].data_ptr()
        es = buf.element_size()
        assert got["dk"].data_ptr() - base == H * D * es and got["dv"].data_ptr() - base == (H + Hkv) * D * es


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_views_of_other_kinds_and_no_gradients_given(torch, dtype):
    """Some given; views of different buffers; k and v the same tensor; one unit of one
    query, whose strides say nothing."""
    c = _case(torch, dtype, seed=1)
    C = 4 * 24
    do = lambda o: dev(c["do"], dtype)  # noqa: E731
    wide = [torch.cat([dev(c[n], dtype), dev(c[n], dtype)], -1)[..., C:] for n in "qkv"]
    got = _both(torch, c, *wide, do)
    _held(c, got, dtype)
    assert all(got["d" + n].stride() == t.stride() for n, t in zip("qkv", wide))
    buf = torch.cat([dev(c[n], dtype) for n in "qkv"], -1)
    q, k, v = buf.split(C, dim=-1)
    room = torch.zeros_like(buf)
    got = _both(torch, c, q, k, v, do, dk=room[..., :C])
    _held(c, got, dtype)
    assert got["dk"].data_ptr() == room.data_ptr() and not room[..., C:].any()
    one = dict(c, v=c["k"])
    got = _both(torch, one, q, k, k, do)
    _held(one, got, dtype)
    assert got["dk"].data_ptr() != got["dv"].data_ptr()
    c = _case(torch, dtype, B=1, X=1, L=1, seed=2)
    q, k, v = torch.cat([dev(c[n], dtype) for n in "qkv"], -1).split(C, dim=-1)
    _held(c, _both(torch, c, q, k, v, lambda o: dev(c["do"], dtype)), dtype)


def test_broadcast_inputs_have_no_gradient(torch):
    c = _case(torch, "bf16", X=2)
    q, k, v = (dev(c[n], "bf16") for n in "qkv")
    one = lambda t: t[:, :1].expand_as(t)  # noqa: E731
    for args, name in (((one(q), k, v), "q"), ((q, one(k), one(v)), "k")):
        with pytest.raises(ValueError, match=f"{name} broadcasts"):
            _both(torch, c, *args, lambda o: dev(c["do"], "bf16"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,X,L", [(1, 3, 45), (2, 1, 45), (1, 1, 70), (1, 1, 1)])
def test_strides_of_single_elements_say_nothing(torch, dtype, B, X, L):
    """v, dout and the gradients with other strides in dimensions of one element than k,
    o and the inputs."""
    c = _case(torch, dtype, B=B, X=X, L=L, seed=3)

    def odd(t):
        st = [s if n > 1 else 8 * (i + 3) * t.shape[3] for i, (n, s) in enumerate(zip(t.shape[:3], t.stride()))]
        return torch.empty(t.numel(), dtype=t.dtype, device="cuda").as_strided(t.shape, (*st, 1)).copy_(t)

    q, k, v, do = (dev(c[n], dtype) for n in ("q", "k", "v", "do"))
    for a, b, d, g in ((k, odd(v), do, None), (k, v, odd(do), None), (k, v, do, odd), (odd(k), odd(v), odd(do), odd)):
        kw = {} if g is None else dict(dq=g(q), dk=g(k), dv=g(v))
        _held(c, _both(torch, c, q, a, b, lambda o: d, **kw), dtype)
    with pytest.raises(ValueError, match="strides"):
        wide = torch.zeros(2, 3, 45, 192, dtype=q.dtype, device="cuda")[..., :96]
        c = _case(torch, dtype)
        _both(torch, c, *(dev(c[n], dtype) for n in "qkv"), lambda o: wide)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("L", [45, 150])
def test_a_training_step_without_copies(torch, dtype, L):
    """The raw projection [Q | K | V] stays for the norm's gradient: the norm writes into
    the columns of a second buffer of its layout, the values are read where they are, and
    the gradients meet in one packed buffer, the norm's in place.  The bits of the step
    on contiguous copies."""
    import paper_2403_10266_amd as dsp
    B, X, H, D = 2, 3, 4, 24
    C = H * D
    c = _case(torch, dtype, L=L, seed=5)
    raw = torch.cat([dev(c[n], dtype) for n in "qkv"], -1)
    do = dev(c["do"], dtype)
    g = torch.Generator(device="cuda").manual_seed(1)
    gq, gk = ((1 + 0.1 * torch.randn(D, generator=g, device="cuda")).to(raw.dtype) for _ in range(2))
    ang = torch.arange(float(L))[:, None] * 100.0 ** (-torch.arange(D // 2) / 12)
    norm = dict(gq=gq, gk=gk, cos=ang.cos().cuda(), sin=ang.sin().cuda())
    bias, bk = dev(c["bias"], dtype), torch.from_numpy(c["buckets"]).cuda()

    rq, rk, v = raw.split(C, dim=-1)
    q, k, _ = torch.empty_like(raw).split(C, dim=-1)
    dsp.dsp_qk_norm_rope(rq, rk, H, H, out_q=q, out_k=k, **norm)
    o, lse = dsp.dsp_attn_relpos(q, k, v, H, H, bias, bk, causal=True, with_lse=True)
    grad = torch.empty_like(raw)
    dq, dk, dv = grad.split(C, dim=-1)
    *_, db = dsp.dsp_attn_relpos_bwd(q, k, v, o, do, lse, H, H, bias, bk, causal=True, dq=dq, dk=dk, dv=dv)
    _, _, dgq, dgk = dsp.dsp_qk_norm_rope_bwd(rq, rk, dq, dk, H, H, dq=dq, dk=dk, **norm)

    cq, ck, cv = (t.contiguous() for t in (rq, rk, v))
    yq, yk = dsp.dsp_qk_norm_rope(cq, ck, H, H, **norm)
    o2, lse2 = dsp.dsp_attn_relpos(yq, yk, cv, H, H, bias, bk, causal=True, with_lse=True)
    aq, ak, av, db2 = dsp.dsp_attn_relpos_bwd(yq, yk, cv, o2, do, lse2, H, H, bias, bk, causal=True)
    nq, nk, dgq2, dgk2 = dsp.dsp_qk_norm_rope_bwd(cq, ck, aq, ak, H, H, **norm)
    torch.cuda.synchronize()
    for a, b in ((o, o2), (lse, lse2), (dq, nq), (dk, nk), (dv, av), (db, db2), (dgq, dgq2), (dgk, dgk2)):
        assert torch.equal(a, b)
