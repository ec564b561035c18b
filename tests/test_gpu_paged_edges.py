"""The paged cache on the GPU at the ends of its sizes."""
import numpy as np
import pytest

from tests import window_util as wu
from tests.gpu_util import dev
from tests.test_gpu_paged import _cache, _i32, _rows_of, torch  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("new", [[1, 2], [60, 40]])
def test_no_pages(torch, kind, new):  # noqa: F811
    """A cache of no pages: queries are turned, no key is seen."""
    import paper_2403_10266_amd as dsp
    r = np.random.default_rng(20)
    dtype, H, Hkv, D, T = "f32" if kind == "f32" else "bf16", 4, 2, 72, sum(new) + 1
    q, k, v = (dev(wu.draw((T, n * D), dtype, r), dtype) for n in (H, Hkv, Hkv))
    ct = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}[kind]
    caches = [torch.empty(0, 16, Hkv, D, dtype=ct, device="cuda") for _ in "kv"]
    s = [torch.zeros(0, Hkv, device="cuda") for _ in "kv"] if kind == "e4m3" else [None, None]
    ang = torch.arange(80, device="cuda")[:, None] * 0.3 ** torch.arange(36, device="cuda")
    table, start, kv = _i32(torch, [[0, 1], [-1, 5]]), _i32(torch, _rows_of(new)), _i32(torch, [70, 50])
    got = dsp.dsp_kv_append(k, v, *caches, table, start, kv, *s, cos=ang.cos(), sin=ang.sin(), q=q,
                            out_q=torch.full_like(q, 7.0))
    one = [_cache(torch, np.zeros((6, 16, Hkv, D)), kind, "token") for _ in "kv"]
    s1 = [torch.zeros(6, Hkv, device="cuda") for _ in "kv"] if kind == "e4m3" else [None, None]
    assert torch.equal(got, dsp.dsp_kv_append(k, v, *one, table, start, kv, *s1, cos=ang.cos(), sin=ang.sin(), q=q,
                                              out_q=torch.full_like(q, 7.0)))
    o, lse = dsp.dsp_attn_paged(got, *caches, table, start, kv, H, max_q=max(new), k_scale=s[0], v_scale=s[1],
                                out=torch.full_like(q, 7.0), lse=torch.full((T, H), 7.0, device="cuda"))
    assert not o[:-1].any() and (lse[:-1] == -np.inf).all() and (o[-1] == 7).all() and (lse[-1] == 7).all()


@pytest.mark.parametrize("Hkv,D", [(0, 72), (2, 0)])
def test_caches_without_heads_are_refused(torch, Hkv, D):  # noqa: F811
    import paper_2403_10266_amd as dsp
    x, c = torch.zeros(3, 144, device="cuda"), torch.zeros(4, 16, Hkv, D, device="cuda")
    k, args = torch.zeros(3, Hkv * D, device="cuda"), (_i32(torch, [[0, 1]]), _i32(torch, [0, 3]), _i32(torch, [9]))
    with pytest.raises(ValueError, match="at least one head"):
        dsp.dsp_attn_paged(x, c, c.clone(), *args, 2)
    with pytest.raises(ValueError, match="at least one head"):
        dsp.dsp_kv_append(k, k, c, c.clone(), *args, q=x)
