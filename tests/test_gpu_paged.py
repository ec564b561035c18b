"""The paged cache on the GPU: appending to it, bit for bit against the oracle where the
arithmetic is exact, and attention over it with the tolerances of tests/window_util.py."""
import numpy as np
import pytest

import synth
from oracle import window as ow
from tests import window_util as wu
from tests.gpu_util import dev, host, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


def _i32(torch, a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def _rows_of(new):
    return np.concatenate([[0], np.cumsum(new)])


def _cache(torch, values, kind, layout):
    """A cache [pages, page, Hkv, D] on the GPU that holds `values`, in some memory layout."""
    t = torch.from_numpy(np.ascontiguousarray(values, np.float32)).cuda()
    t = t.to({"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}[kind])
    if layout == "head":
        return t.transpose(1, 2).contiguous().transpose(1, 2)
    if layout == "both":       # K and V slots side by side: rows with gaps
        two = torch.zeros(t.shape[0], t.shape[1], 2, *t.shape[2:], dtype=torch.float32, device="cuda").to(t.dtype)
        two.view(torch.uint8)[:, :, 1] = t.contiguous().view(torch.uint8)
        return two[:, :, 1]
    return t.contiguous()


def _f64(t):
    return t.float().cpu().numpy().astype(np.float64)


def _table(r, lens, page, extra=2):
    """(table, pages): each sequence's pages at random places, the rest of its row -1."""
    need = [-(-n // page) for n in lens]
    count = sum(need) + extra
    order, width = r.permutation(count), max(need) + 1
    table, at = np.full((len(lens), width), -1), 0
    for n, k in enumerate(need):
        table[n, :k] = order[at:at + k]
        at += k
    return table, count


APPEND = [
    # new, kv, page, H, Hkv, D, rot, interleaved
    ([1, 1, 1], [1, 40, 33], 16, 4, 2, 64, 64, False),
    ([5, 0, 70], [5, 9, 100], 32, 4, 4, 72, 72, False),
    ([300], [300], 64, 2, 2, 72, 40, True),
    ([17, 31, 1, 2], [20, 64, 65, 2], 16, 0, 3, 40, 0, False),
    ([40, 3], [170, 131], 128, 8, 2, 128, 64, True),
    ([3, 100], [3, 108], 16, 2, 1, 8, 8, False),
    ([200], [210], 256, 1, 1, 96, 96, True),
    ([7, 9], [7, 30], 16, 2, 2, 20, 14, False),          # halves inside a chunk
    ([7, 9], [7, 30], 32, 3, 3, 33, 22, True),           # odd widths
    ([6], [1100], 1024, 2, 1, 16, 6, False),
]


@pytest.mark.parametrize("kind", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("layout", ["token", "head", "both"])
@pytest.mark.parametrize("new,kv,page,H,Hkv,D,rot,interleaved", APPEND)
def test_append(torch, kind, layout, new, kv, page, H, Hkv, D, rot, interleaved):
    """What is neither turned nor 8 bits is copied; turned elements are within the roundings
    of the two products and the sum (fp32) and of the cache's type; in 8 bits, what no
    rounding could move to another value is that value.  Everything else stays."""
    import paper_2403_10266_amd as dsp
    r = np.random.default_rng(D + page)
    dtype = "f32" if kind == "f32" else "bf16"
    table, pages = _table(r, kv, page)
    start = _rows_of(new)
    T = start[-1] + 2
    k, v, q = (wu.draw((T, n * D), dtype, r, s) for n, s in ((Hkv, 1.5), (Hkv, 1.0), (max(H, 1), 1.0)))
    k *= np.exp2(r.integers(-6, 7, (T, 1))).astype(np.float32)     # magnitudes that make scales grow
    P = max(kv)
    ang = np.arange(P)[:, None] * 100.0 ** (-np.arange(rot // 2) * 2 / max(rot, 1))
    cos, sin = ((f(ang).astype(np.float32) if rot else None) for f in (np.cos, np.sin))
    held = [r.standard_normal((pages, page, Hkv, D)) for _ in "kv"]
    scales = [None, None]
    if kind == "e4m3":
        held = [ow.e4m3(h * 100) for h in held]
        scales = [2.0 ** r.integers(-9, -4, (pages, Hkv)) for _ in "kv"]
    elif kind == "bf16":
        held = [synth.bf16_round(h.astype(np.float32)) for h in held]
    else:
        held = [h.astype(np.float32) for h in held]
    caches = [_cache(torch, h, kind, layout) for h in held]
    dsc = [None if s is None else torch.from_numpy(s.astype(np.float32)).cuda() for s in scales]
    put = lambda t: None if t is None else torch.from_numpy(t).cuda()  # noqa: E731
    out = torch.full((T, H * D), 7.0, dtype=dev(q[:1], dtype).dtype, device="cuda") if H else None
    got_q = dsp.dsp_kv_append(dev(k, dtype), dev(v, dtype), *caches, _i32(torch, table), _i32(torch, start), _i32(torch, kv),
                              *dsc, cos=put(cos), sin=put(sin), interleaved=interleaved,
                              q=dev(q, dtype) if H else None, out_q=out)
    torch.cuda.synchronize()
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    at = np.concatenate([np.arange(n) + m - n for n, m in zip(new, kv)]).astype(int)
    n_rows = start[-1]

    def near(got, want, x, what, rounded):
        # turned: two products and a sum in fp32, once more in the type.  |a||c| + |b||s| is the
        # first of a pair turned by -|s|, and the second of it turned by |s|
        a = np.abs(x)
        mag = np.maximum(*(ow.turned(a, at, np.abs(cos), t * np.abs(sin), interleaved) for t in (-1, 1))) if rot else a
        tol = 3 * 2.0 ** -24 * mag * (rot > 0) + (rounded * np.abs(want) if rot else 0)
        bad = np.abs(got - want) > tol * (1 + 2.0 ** -6)
        assert not bad.any(), f"{what}: {np.argwhere(bad)[:3]}"

    if H:
        want = ow.turned(q[:n_rows].reshape(n_rows, H, D), at, cos, sin, interleaved)
        near(host(got_q)[:n_rows].reshape(n_rows, H, D), want, q[:n_rows].reshape(n_rows, H, D), "q", u)
        assert (got_q[n_rows:] == 7).all()
    for x, h, s, c, d, turn, name in ((k, held[0], scales[0], caches[0], dsc[0], True, "k"),
                                      (v, held[1], scales[1], caches[1], dsc[1], False, "v")):
        x = x.reshape(T, Hkv, D).astype(np.float64)
        want, ws = h.astype(np.float64).copy(), None if s is None else s.copy()
        ow.append(x, want, table, start, kv, ws, cos if turn else None, sin if turn else None, None, interleaved)
        got = _f64(c)
        if kind != "e4m3":
            mask = np.zeros(want.shape[:2], bool)
            for n in range(len(kv)):
                for i in range(new[n]):
                    p = kv[n] - new[n] + i
                    mask[table[n][p // page], p % page] = True
            assert np.array_equal(got[~mask], h.astype(np.float64)[~mask]), name
            flat = lambda t: np.concatenate([t[[table[n][p // page] for p in range(kv[n] - new[n], kv[n])],  # noqa: E731
                                               [p % page for p in range(kv[n] - new[n], kv[n])]] for n in range(len(kv))
                                             if new[n]])
            if turn:
                near(flat(got), flat(want), x[:n_rows], name, u)
            else:
                assert np.array_equal(flat(got), flat(want)), name
            continue
        assert np.array_equal(_f64(d), ws), name + " scales"
        # a code may differ where the fp32 value lies within its own roundings of a border
        same = got == want
        step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(want), 2.0 ** -6))) - 3)
        assert same.all() or (turn and rot and (np.abs(got - want)[~same] <= step[~same]).all()
                              and (~same).sum() <= 2 + 1e-4 * same.size), f"{name}: {(~same).sum()} of {same.size} codes"


def test_append_is_the_same_in_chunks(torch):
    """A sequence appended token by token, in chunks and at once gives one cache (8 bits: where
    the scales do not shrink along the way, the codes too)."""
    import paper_2403_10266_amd as dsp
    r = np.random.default_rng(3)
    L, page, Hkv, D = 150, 32, 2, 72
    x = wu.draw((L, Hkv * D), "bf16", r)
    x[0::page] *= 64                            # the first token of a page has its largest value
    t = dev(x, "bf16")
    ang = torch.arange(L, device="cuda")[:, None] * 0.1 ** torch.arange(36, device="cuda")
    table = _i32(torch, [[4, 0, 2, 1, 3]])
    for kind in ("bf16", "e4m3"):
        got = []
        for cuts in ([L], [1] * L, [7, 60, 83]):
            c = [_cache(torch, np.zeros((5, page, Hkv, D)), kind, "token") for _ in "kv"]
            s = [torch.zeros(5, Hkv, device="cuda") for _ in "kv"] if kind == "e4m3" else [None, None]
            at = 0
            for n in cuts:
                dsp.dsp_kv_append(t[at:at + n], t[at:at + n], *c, table, _i32(torch, [0, n]), _i32(torch, [at + n]), *s,
                                  cos=ang.cos(), sin=ang.sin())
                at += n
            got.append([a.view(torch.uint8) for a in c] + [a for a in s if a is not None])
        for other in got[1:]:
            assert all(torch.equal(a, b) for a, b in zip(got[0], other)), kind


def test_append_in_place_and_positions(torch):
    """Queries in place in a packed projection; positions of the caller's; one without a row
    gives NaN in what turns, held as NaN in 8 bits without touching the other tokens."""
    import paper_2403_10266_amd as dsp
    r = np.random.default_rng(4)
    T, H, Hkv, D, page = 20, 4, 2, 64, 16
    qkv = dev(wu.draw((T, (H + 2 * Hkv) * D), "bf16", r), "bf16")
    q, k, v = qkv.split((H * D, Hkv * D, Hkv * D), -1)
    ang = torch.arange(50, device="cuda")[:, None] * 0.3 ** torch.arange(16, device="cuda")
    cos, sin = ang.cos(), ang.sin()
    pos = np.arange(T) * 2
    pos[7] = 50
    args = (_i32(torch, [[1, 0]]), _i32(torch, [0, T]), _i32(torch, [T]))
    for kind in ("bf16", "e4m3"):
        c = [_cache(torch, np.zeros((2, page, Hkv, D)), kind, "token") for _ in "kv"]
        s = [torch.zeros(2, Hkv, device="cuda") for _ in "kv"] if kind == "e4m3" else [None, None]
        new = dsp.dsp_kv_append(k, v, *c, *args, *s, cos=cos, sin=sin, pos=_i32(torch, pos), q=q)
        rest = qkv.clone()
        same = dsp.dsp_kv_append(k, v, *c, *args, *s, cos=cos, sin=sin, pos=_i32(torch, pos),
                                 q=rest[:, :H * D], out_q=rest[:, :H * D])
        assert torch.equal(same.nan_to_num(nan=3.0), new.nan_to_num(nan=3.0)) and torch.equal(rest[:, H * D:], qkv[:, H * D:])
        got = c[0].float()[1, 7]
        assert got[:, :32].isnan().all() and not got[:, 32:].isnan().any()
        assert new[7].reshape(H, D)[:, :32].isnan().all() and new.float().isnan().sum() == H * 32
        assert c[0].float().isnan().sum() == Hkv * 32
        if kind == "e4m3":
            assert torch.isfinite(s[0]).all() and (s[0] > 0).all()


def test_append_to_pages_that_are_not_there(torch):
    """Table entries outside the cache, positions past the table and before 0: tokens are
    dropped, everything else is as it was."""
    import paper_2403_10266_amd as dsp
    r = np.random.default_rng(5)
    for kind in ("bf16", "e4m3"):
        table, new, kv = [[1, 9, -1, 2], [-2147483648, 2147483647, 0, 3]], [60, 70], [60, 70]
        x = wu.draw((130, 2 * 40), "bf16", r)
        c = [_cache(torch, np.full((4, 16, 2, 40), 3.0), kind, "token") for _ in "kv"]
        s = [torch.ones(4, 2, device="cuda") for _ in "kv"] if kind == "e4m3" else [None, None]
        dsp.dsp_kv_append(dev(x, "bf16"), dev(x, "bf16"), *c, _i32(torch, table), _i32(torch, _rows_of(new)),
                          _i32(torch, kv), *s)
        want, ws = np.full((4, 16, 2, 40), 3.0), np.ones((4, 2)) if kind == "e4m3" else None
        ow.append(x.reshape(130, 2, 40), want, np.array(table), _rows_of(new), kv, ws)
        assert np.array_equal(_f64(c[0]), want) and (ws is None or np.array_equal(_f64(s[0]), ws))
        before = [a.view(torch.uint8).clone() for a in c]
        for start, lens in (([0, 5, 5], [-3, 0]), ([0, 0, 0], [3, 4]), ([-7, -3, -1], [5, 5]), ([200, 200, 300], [9, 9])):
            dsp.dsp_kv_append(dev(x, "bf16"), dev(x, "bf16"), *c, _i32(torch, table), _i32(torch, start), _i32(torch, lens), *s)
        assert all(torch.equal(a.view(torch.uint8), b) for a, b in zip(c, before))


ATTN = [
    # new, kv, page, H, Hkv, D, left, right, sinks
    ([1, 1, 1], [1, 40, 333], 16, 4, 2, 64, -1, 0, 0),
    ([1, 1], [700, 2500], 64, 8, 2, 72, 100, 0, 4),
    ([3, 0, 2, 1], [50, 20, 2, 0], 32, 4, 4, 40, 12, 0, 1),       # no new tokens; no positions
    ([4, 4], [900, 4], 128, 8, 1, 128, -1, 0, 0),
    ([100, 33, 1], [100, 400, 90], 16, 4, 2, 72, -1, 0, 0),       # chunks and a token
    ([70, 200], [300, 200], 64, 4, 1, 64, 50, 0, 5),
    ([129], [129], 32, 2, 2, 96, -1, -1, 0),                      # new tokens that see one another
    ([40, 9], [60, 300], 256, 6, 3, 80, 20, 3, 17),
    ([65], [70], 1024, 3, 1, 32, -1, 0, 0),
    ([1], [5000], 16, 32, 1, 64, -1, 0, 0),                       # many parts
    ([2, 1], [80, 90], 16, 40, 1, 16, -1, 0, 0),                  # more heads of a group than a block has columns
]


@pytest.mark.parametrize("kind", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("layout", ["token", "head", "both"])
@pytest.mark.parametrize("new,kv,page,H,Hkv,D,left,right,sinks", ATTN)
def test_attention(torch, kind, layout, new, kv, page, H, Hkv, D, left, right, sinks):
    import paper_2403_10266_amd as dsp
    r = np.random.default_rng(D + page + H)
    dtype = "f32" if kind == "f32" else "bf16"
    table, pages = _table(r, kv, page)
    if left >= 0:      # pages that no new token sees were given back
        for n in range(len(kv)):
            for g in range(table.shape[1]):
                if (g + 1) * page <= kv[n] - new[n] - left and g * page >= sinks:
                    table[n, g] = -1
    held = [wu.draw((pages, page, Hkv, D), dtype, r) for _ in "kv"]
    scales = [None, None]
    if kind == "e4m3":
        scales = [2.0 ** r.integers(-9, -5, (pages, Hkv)) for _ in "kv"]
        held = [ow.e4m3(h / s[:, None, :, None]) for h, s in zip(held, scales)]
        held = [np.clip(h, -448, 448) for h in held]
    _attend(torch, dsp, r, kind, dtype, layout, table, held, scales, new, kv, H, Hkv, D, left, right, sinks)


def _attend(torch, dsp, r, kind, dtype, layout, table, held, scales, new, kv, H, Hkv, D, left, right, sinks, max_q=None):
    start = _rows_of(new)
    T = start[-1] + 3
    q = wu.draw((T, H * D), dtype, r)
    caches = [_cache(torch, h, kind, layout) for h in held]
    dsc = [None if s is None else torch.from_numpy(s.astype(np.float32)).cuda() for s in scales]
    out = torch.full((T, H * D), 7.0, device="cuda").to(dev(q[:1], dtype).dtype)
    lse = torch.full((T, H), 7.0, device="cuda")
    dsp.dsp_attn_paged(dev(q, dtype), *caches, _i32(torch, table), _i32(torch, start), _i32(torch, kv), H,
                       max_q=max(new) if max_q is None else max_q, left=left, right=right, sinks=sinks, k_scale=dsc[0],
                       v_scale=dsc[1], out=out, lse=lse)
    torch.cuda.synchronize()
    q64 = q.reshape(T, H, D).astype(np.float64)
    hk, hv = (np.asarray(h, np.float64) for h in held)
    want = ow.attention_paged(q64, hk, hv, table, start, kv, H, left, right, sinks, None, *scales, max_q=max_q)
    got, gl = host(out).reshape(T, H, D), host(lse)
    u, worst = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24, 0.0
    page, scale = held[0].shape[1], D ** -0.5
    for n in range(len(kv)):
        cap = min(max(kv[n], 0), table.shape[1] * page)
        at = [(table[n][j // page], j % page) for j in range(cap)]
        ok = [0 <= g < len(hk) for g, _ in at]
        full = lambda c, s: np.array([c[g, t] * (1 if s is None else s[g][:, None]) if o else np.zeros((Hkv, D))  # noqa: E731
                                      for (g, t), o in zip(at, ok)]).reshape(cap, Hkv, D)
        k, v = full(hk, scales[0]), full(hv, scales[1])
        seen = ow.visible(new[n], cap, kv[n] - new[n], cap, left, right, sinks) & np.array(ok, bool)[None, :]
        used = seen.any(0)[:, None, None]
        k, v = np.where(used, k, 0.0), np.where(used, v, 0.0)
        for i in range(new[n]):
            row = start[n] + i
            if row not in want:
                assert (got[row] == 7).all() and (gl[row] == 7).all()
                continue
            o, l = want[row]
            for h in range(H):
                kk, vv = k[:, h // (H // Hkv)], v[:, h // (H // Hkv)]
                z = np.where(seen[i], kk @ q64[row, h] * scale, -np.inf)
                p = np.zeros(cap) if np.isneginf(l[h]) else np.exp(z - l[h])
                t_o, t_l, _ = wu.row_bounds(q64[row, h][None], kk, vv, p[None], o[h][None], l[h], scale, u)
                assert np.isneginf(l[h]) == np.isneginf(gl[row, h])
                if np.isneginf(l[h]):
                    assert not got[row, h].any()
                    continue
                worst = max(worst, float((np.abs(got[row, h] - o[h]) / (t_o[0] + 1e-30)).max()),
                            float(abs(gl[row, h] - l[h]) / t_l))
    say(f"  {kind} {layout}: {worst:.3f} of its tolerance")
    assert worst <= 1.0
    assert (got[start[-1]:] == 7).all() and (gl[start[-1]:] == 7).all()


@pytest.mark.parametrize("kind", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("new", [[1, 2], [60, 40]])
def test_pages_that_are_not_there(torch, kind, new):
    """Entries outside the cache take their keys out, also where a query sees them, in the
    middle of a tile and at its ends; positions past the table are none."""
    import paper_2403_10266_amd as dsp
    r = np.random.default_rng(6)
    dtype = "f32" if kind == "f32" else "bf16"
    table = np.array([[3, -1, 0, 99, 5, 2, -2147483648], [-1, 7, 6, 4, 1, 2147483647, 8]])
    held = [wu.draw((9, 16, 2, 64), dtype, r) for _ in "kv"]
    scales = [None, None]
    if kind == "e4m3":
        scales = [np.full((9, 2), 0.125) for _ in "kv"]
        held = [ow.e4m3(h * 8) for h in held]
    _attend(torch, dsp, r, kind, dtype, "token", table, held, scales, new, [105, 200], 4, 2, 64, -1, 0, 0)


@pytest.mark.parametrize("max_q", [0, 1, 2])
def test_rows_past_max_q(torch, max_q):
    import paper_2403_10266_amd as dsp
    r = np.random.default_rng(7)
    table, pages = _table(r, [50, 20], 16)
    held = [wu.draw((pages, 16, 2, 64), "bf16", r) for _ in "kv"]
    _attend(torch, dsp, r, "bf16", "bf16", "token", table, held, [None, None], [5, 2], [50, 20], 4, 2, 64, -1, 0, 0, max_q)


def test_nothing_but_seen_slots_is_used(torch):
    """NaN in slots past kv_len, in pages of others and behind the window changes nothing."""
    import paper_2403_10266_amd as dsp
    for new in (2, 60):
        r = np.random.default_rng(8)
        table = _i32(torch, [[2, 5, 1, 7, 0, 4, 6]])
        x = [dev(wu.draw((8, 16, 2, 72), "bf16", r), "bf16") for _ in "kv"]
        q = dev(wu.draw((new, 4 * 72), "bf16", r), "bf16")
        call = lambda k, v: dsp.dsp_attn_paged(q, k, v, table, _i32(torch, [0, new]), _i32(torch, [103]), 4,  # noqa: E731
                                               max_q=new, left=10, sinks=3)
        want = call(*x)
        first = 103 - new - 10
        for t in x:
            t[3] = float("nan")
            for j in range(7 * 16):
                if j >= 103 or 3 <= j < first:
                    t[[2, 5, 1, 7, 0, 4, 6][j // 16], j % 16] = float("inf") if j % 2 else float("nan")
        assert torch.equal(call(*x), want)


def test_tables_of_no_meaning(torch):
    """Row starts that fall, lengths below 0 and past everything: nothing outside is touched,
    rows of no sequence stay."""
    import paper_2403_10266_amd as dsp
    r = np.random.default_rng(9)
    c = [dev(wu.draw((4, 16, 2, 64), "bf16", r), "bf16") for _ in "kv"]
    q = dev(wu.draw((90, 256), "bf16", r), "bf16")
    for start, kv, max_q in (([5, 3, 1], [9, 9], 1), ([-5, 0, 900], [-1, 2147483647], 90),
                             ([0, 90, 20], [2147483647, -2147483648], 90), ([90, 90, 90], [64, 64], 90)):
        out = torch.full((90, 256), 7.0, device="cuda").bfloat16()
        dsp.dsp_attn_paged(q, *c, _i32(torch, [[0, 1, 2, 3], [3, 2, 1, 0]]), _i32(torch, start), _i32(torch, kv), 4,
                           max_q=max_q, out=out)
        torch.cuda.synchronize()
        assert torch.isfinite(out.float()).all()


def test_generation(torch):
    """A run of a program that generates: a prompt in chunks, then tokens, two sequences of
    different lengths, pages given back behind the window.  Every step's output is windowed
    attention over the whole sequence so far; 8 bits: over the values that the pages hold.
    The steps of one token run from a captured graph."""
    import paper_2403_10266_amd as dsp
    r = np.random.default_rng(10)
    H, Hkv, D, page, left, sinks = 4, 2, 72, 16, 37, 3
    steps = [[50, 9], [40, 0], [1, 30]] + [[1, 1]] * 20
    total = [sum(s[n] for s in steps) for n in range(2)]
    L = max(total)
    ang = np.arange(L)[:, None] * 0.2 ** np.arange(36)
    cos, sin = (torch.from_numpy(f(ang).astype(np.float32)).cuda() for f in (np.cos, np.sin))
    data = [{n: wu.draw((total[s], w * D), "bf16", r) for n, w in (("q", H), ("k", Hkv), ("v", Hkv))} for s in range(2)]
    for kind in ("bf16", "e4m3"):
        caches = [_cache(torch, np.zeros((30, page, Hkv, D)), kind, "token") for _ in "kv"]
        scales = [torch.zeros(30, Hkv, device="cuda") for _ in "kv"] if kind == "e4m3" else [None, None]
        full = r.permutation(30)[:2 * 14].reshape(2, 14)
        table, kv, graph = np.full((2, 14), -1), [0, 0], None
        bufs = [torch.zeros(2, w * D, device="cuda").bfloat16() for w in (H, Hkv, Hkv)]
        d_table, d_kv, d_start = _i32(torch, table), _i32(torch, kv), _i32(torch, [0, 1, 2])

        def step(q, k, v, table, start, kv, max_q):
            rq = dsp.dsp_kv_append(k, v, *caches, table, start, kv, *scales, cos=cos, sin=sin, q=q)
            return rq, dsp.dsp_attn_paged(rq, *caches, table, start, kv, H, max_q=max_q, left=left, sinks=sinks,
                                      k_scale=scales[0], v_scale=scales[1])

        for t, new in enumerate(steps):
            at = list(kv)
            kv = [a + n for a, n in zip(at, new)]
            for n in range(2):
                for g in range(14):
                    table[n, g] = full[n, g] if g * page < kv[n] and ((g + 1) * page > at[n] - left or g * page < sinks) else -1
            rows = [torch.cat([dev(data[n][x][at[n]:kv[n]], "bf16") for n in range(2)]) for x in "qkv"]
            if new == [1, 1]:
                for b, x in zip(bufs, rows):
                    b.copy_(x)
                d_table.copy_(_i32(torch, table))
                d_kv.copy_(_i32(torch, kv))
                if graph is None:
                    step(*bufs, d_table, d_start, d_kv, 1)      # the same tokens again: no change
                    graph = torch.cuda.CUDAGraph()
                    with torch.cuda.graph(graph):
                        out = step(*bufs, d_table, d_start, d_kv, 1)
                graph.replay()
            else:
                out = step(*rows, _i32(torch, table), _i32(torch, _rows_of(new)), _i32(torch, kv), max(new))
            torch.cuda.synchronize()
            (turned, got), row = (host(x) for x in out), 0
            for n in range(2):
                if not new[n]:
                    continue
                # the cache's own values where they are still there, at their positions
                k, v = np.zeros((kv[n], Hkv, D)), np.zeros((kv[n], Hkv, D))
                for j in range(kv[n]):
                    g = table[n][j // page]
                    if g >= 0:
                        for x, c, s in ((k, caches[0], scales[0]), (v, caches[1], scales[1])):
                            x[j] = _f64(c[g, j % page]) * (1 if s is None else _f64(s[g])[:, None])
                q = ow.turned(data[n]["q"][at[n]:kv[n]].reshape(-1, H, D), np.arange(at[n], kv[n]),
                              cos.cpu().numpy(), sin.cpu().numpy(), False)
                own = turned[row:row + new[n]].reshape(q.shape)
                assert (np.abs(own - q) <= (2.0 ** -8 + 2.0 ** -20) * np.abs(q) + 2.0 ** -21).all()
                c = dict(q=own.reshape(1, 1, -1, H * D), k=k.reshape(1, 1, -1, Hkv * D),
                         v=v.reshape(1, 1, -1, Hkv * D), H=H, Hkv=Hkv)
                c["do"] = c["q"]
                w = wu.wanted(c, "bf16", left, 0, sinks, [at[n]], grads=False)
                wu.compare(dict(o=got[row:row + new[n]]), dict(o=w["o"]), lambda *a: None)
                row += new[n]
        if kind == "bf16":     # and the tokens themselves, turned by their positions
            want = ow.turned(data[0]["k"].reshape(-1, Hkv, D), np.arange(total[0]), cos.cpu().numpy(), sin.cpu().numpy(), False)
            j = kv[0] - 1
            assert np.abs(_f64(caches[0][table[0][j // page], j % page]) - want[j]).max() <= 2.0 ** -7 * np.abs(want[j]).max()


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("new", [2, 300])
def test_a_held_token_that_is_not_finite_shows(torch, kind, new):
    """A token whose key is NaN, appended in the middle of a sequence, is in every new token that
    sees it, and not in another sequence."""
    import paper_2403_10266_amd as dsp
    r = np.random.default_rng(12)
    H, Hkv, D, page, kv, at = 4, 2, 72, 32, 640, 350
    table = _i32(torch, r.permutation(40).reshape(2, 20))
    c = [_cache(torch, np.zeros((40, page, Hkv, D)), kind, "token") for _ in "kv"]
    s = [torch.zeros(40, Hkv, device="cuda") for _ in "kv"] if kind == "e4m3" else [None, None]
    k, v = (dev(wu.draw((2 * kv, Hkv * D), "bf16", r), "bf16") for _ in "kv")
    q = dev(wu.draw((2 * new, H * D), "bf16", r), "bf16")
    call = lambda: dsp.dsp_attn_paged(q, *c, table, _i32(torch, [0, new, 2 * new]), _i32(torch, [kv, kv]), H,  # noqa: E731
                                      max_q=new, k_scale=s[0], v_scale=s[1], with_lse=True)
    put = lambda: dsp.dsp_kv_append(k, v, *c, table, _i32(torch, [0, kv, 2 * kv]), _i32(torch, [kv, kv]), *s)  # noqa: E731
    put()
    o, lse = call()
    k[kv + at, 5] = float("nan")
    put()
    p, lsp = call()
    first = new + max(at - (kv - new), 0)
    assert p[first:, :144].isnan().all() and lsp[first:, :2].isnan().all()
    assert torch.equal(p[:new], o[:new]) and torch.equal(p[:, 144:], o[:, 144:]) and torch.equal(lsp[:, 2:], lse[:, 2:])


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_long_prompts_and_short_ones(torch, kind):
    """Blocks of many sequences, some with none, some of many: each is taken once."""
    import paper_2403_10266_amd as dsp
    r = np.random.default_rng(13)
    new = [0, 257, 1, 33, 0, 128, 5, 0]
    kv = [10, 257, 90, 300, 0, 130, 5, 0]
    table, pages = _table(r, kv, 16)
    held, scales = [wu.draw((pages, 16, 2, 64), "bf16", r) for _ in "kv"], [None, None]
    if kind == "e4m3":
        scales = [2.0 ** r.integers(-4, 2, (pages, 2)) for _ in "kv"]
        held = [np.clip(ow.e4m3(h / s[:, None, :, None]), -448, 448) for h, s in zip(held, scales)]
    _attend(torch, dsp, r, kind, "bf16", "token", table, held, scales, new, kv, 8, 2, 64, -1, 0, 0)


@pytest.mark.parametrize("kind", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("new,kv,H,Hkv,D,left", [([20, 9, 0, 1], [2100, 1500, 40, 90], 8, 2, 64, -1), ([40], [3000], 4, 1, 72, -1),
                                                 ([17, 33], [1800, 33], 6, 2, 128, 900)])
def test_several_blocks_of_columns_against_a_long_cache(torch, kind, new, kv, H, Hkv, D, left):
    import paper_2403_10266_amd as dsp
    r = np.random.default_rng(14)
    dtype = "f32" if kind == "f32" else "bf16"
    table, pages = _table(r, kv, 32)
    held, scales = [wu.draw((pages, 32, Hkv, D), dtype, r) for _ in "kv"], [None, None]
    if kind == "e4m3":
        scales = [2.0 ** r.integers(-4, 2, (pages, Hkv)) for _ in "kv"]
        held = [np.clip(ow.e4m3(h / s[:, None, :, None]), -448, 448) for h, s in zip(held, scales)]
    _attend(torch, dsp, r, kind, dtype, "token", table, held, scales, new, kv, H, Hkv, D, left, 0, 0)
