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
