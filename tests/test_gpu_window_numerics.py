"""Windowed attention and attention over pages in bf16 at the ends of their numbers."""
import numpy as np
import pytest

from tests.gpu_util import say
from tests.test_gpu_attn_window import torch  # noqa: F401

pytestmark = pytest.mark.gpu


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
