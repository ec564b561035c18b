"""A query or an output gradient that is not finite stays in its own unit and head: no
other result of attention with a relative position bias loses a bit to it, whichever
units a work-group takes in turn."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


CASES = [
    # X, Lq, Lk, H, Hkv, D: more units to a head than it has work-groups
    (48, 66, 70, 128, 128, 72),    # long rows: 32 work-groups to a head
    (48, 66, 70, 128, 32, 40),
    (24, 150, 70, 128, 128, 24),   # two blocks of queries to a unit
    (60, 49, 49, 64, 64, 72),      # short units: 16
    (60, 30, 32, 64, 64, 40),      # in one block: 32
    (100, 49, 49, 64, 32, 72),     # shared keys: 16, and 32 for dK and dV
    (150, 20, 31, 128, 64, 24),
    (60, 49, 49, 64, 64, 64),      # a width without spare columns
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("X,Lq,Lk,H,Hkv,D", CASES)
def test_other_units_keep_their_bits(torch, dtype, X, Lq, Lk, H, Hkv, D):
    import paper_2403_10266_amd as dsp
    tt = torch.bfloat16 if dtype == "bf16" else torch.float32
    if dtype == "f32":
        H, Hkv, D = H // 2, Hkv // 2, {72: 52, 40: 20}.get(D, D)   # spare columns in fp32 too
        X = 2 * X
    g = torch.Generator(device="cuda").manual_seed(X + D)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(tt)  # noqa: E731
    q, do = r(1, X, Lq, H * D), r(1, X, Lq, H * D)
    k, v = r(1, X, Lk, Hkv * D), r(1, X, Lk, Hkv * D)
    bias, bk = r(8, H), dsp.dsp_relpos_buckets(16, 8).cuda()

    def both(q, do):
        o, lse = dsp.dsp_attn_relpos(q, k, v, H, Hkv, bias, bk, with_lse=True)
        return dict(zip(("o", "lse", "dq", "dk", "dv", "dbias"),
                        (o, lse, *dsp.dsp_attn_relpos_bwd(q, k, v, o, do, lse, H, Hkv, bias, bk))))

    clean = both(q, do)
    # (unit, head, row, what): early units, so that others of their work-groups follow
    hit = [(0, 0, 3, "do", float("nan")), (1, 5, Lq - 1, "do", float("inf")), (2, H - 1, 0, "q", float("nan")),
           (3, 1, 7, "q", float("-inf"))]
    q2, do2 = q.clone(), do.clone()
    for x, h, row, what, value in hit:
        (q2 if what == "q" else do2)[0, x, row, h * D + 2] = value
    bad = both(q2, do2)
    torch.cuda.synchronize()
    grp = H // Hkv
    for name, heads in (("o", H), ("dq", H), ("dk", Hkv), ("dv", Hkv), ("lse", H), ("dbias", H)):
        a, b = clean[name], bad[name]
        if name == "dbias":                                     # a head's sums over its units
            same = (a == b).all(0)[None]
        elif name == "lse":
            same = (a == b).view(X, H, Lq).all(-1)
        else:
            same = (a == b).view(X, -1, heads, D).all(1).all(-1)
        free = torch.ones_like(same)
        for x, h, *_ in hit:
            free[0 if name == "dbias" else x, h if heads == H else h // grp] = False
        assert same[free].all(), (name, (free & ~same).nonzero()[:5].tolist())
    assert bad["dq"].view(X, Lq, H, D)[0, 3, 0].isnan().any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("X,Lq,Lk,H,Hkv,D", [
    (2, 200, 200, 2, 2, 72), (16, 2000, 200, 16, 16, 72), (2, 200, 200, 2, 2, 64), (2, 50, 50, 2, 2, 72),
    (1, 1, 900, 4, 4, 72), (2, 3, 100, 8, 2, 64), (2, 2, 20, 4, 2, 72), (1, 2, 60, 2, 2, 40), (3000, 1, 120, 4, 4, 72),
])
def test_a_query_that_is_not_finite_shows(torch, dtype, X, Lq, Lk, H, Hkv, D):
    """Its row is NaN, its log-sum-exp too (only a row without keys is 0 with -inf), its
    gradient and what it adds to the gradients of its keys as well; other rows stay.
    Those of its wave may be summed from another reference: both results are off by at
    most u of the largest value for P and u for the result, u = 2^-8 in bf16; in fp32 by
    3 (D + 16) 2^-24 (1 + S), S < 60 the largest score: 2^-9 of the largest value."""
    import paper_2403_10266_amd as dsp
    tt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(X + D)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(tt)  # noqa: E731
    q, do = r(1, X, Lq, H * D), r(1, X, Lq, H * D)
    k, v = r(1, X, Lk, Hkv * D), r(1, X, Lk, Hkv * D)
    bias, bk = r(8, H), dsp.dsp_relpos_buckets(16, 8).cuda()
    clean, lse0 = dsp.dsp_attn_relpos(q, k, v, H, Hkv, bias, bk, with_lse=True)
    for value in (float("nan"), float("inf")):
        q2 = q.clone()
        q2[0, 0, Lq - 1, D + 3] = value                         # head 1
        o, lse = dsp.dsp_attn_relpos(q2, k, v, H, Hkv, bias, bk, with_lse=True)
        dq, dk, dv, _ = dsp.dsp_attn_relpos_bwd(q2, k, v, o, do, lse, H, Hkv, bias, bk)
        torch.cuda.synchronize()
        assert o[0, 0, Lq - 1, D:2 * D].isnan().all() and lse[0, 0, 1, Lq - 1].isnan(), value
        assert dq[0, 0, Lq - 1, D:2 * D].isnan().any(), value
        e = 1 // (H // Hkv)                                     # the keys of head 1
        assert all(t[0, 0, :, e * D:(e + 1) * D].isnan().any() for t in (dk, dv)), value
        free = torch.ones(1, X, Lq, H, dtype=torch.bool, device="cuda")
        free[0, 0, Lq - 1, 1] = False
        a, b = (t.float().view(1, X, Lq, H, D)[free] for t in (clean, o))
        most = (4 * 2.0 ** -8 if dtype == "bf16" else 2.0 ** -9) * float(v.abs().max())
        assert (a - b).abs().max() <= most, value
        a, b = (t.transpose(2, 3)[free] for t in (lse0, lse))
        assert (a - b).abs().max() <= 2.0 ** -9, value
        k0 = torch.zeros(1, dtype=torch.int32, device="cuda")
        o, lse = dsp.dsp_attn_relpos(q2, k, v, H, Hkv, bias, bk, kv_len=k0, with_lse=True)
        torch.cuda.synchronize()
        assert not o.any() and lse.isneginf().all()
