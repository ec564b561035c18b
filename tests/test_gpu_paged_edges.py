"""The paged cache on the GPU at the ends of its sizes."""
import numpy as np
import pytest

import synth
from oracle import window as ow
from tests import window_util as wu
from tests.gpu_util import dev, host, say
from tests.test_gpu_paged import _attend, _cache, _f64, _i32, _rows_of, _table, torch  # noqa: F401

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


def _near(got, want, x, at, cos, sin, u, what):
    """Turned rows: two products and a sum in fp32 of the pair's magnitudes, then the type."""
    mag = np.maximum(*(ow.turned(np.abs(x), at, np.abs(cos), t * np.abs(sin), False) for t in (-1, 1)))
    bad = np.abs(got - want) > (3 * 2.0 ** -24 * mag + u * np.abs(want)) * (1 + 2.0 ** -6)
    assert not bad.any(), f"{what}: {np.argwhere(bad)[:3]}"


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("T", [8200, 16500, 33000, 66000])
def test_append_of_many_tokens(torch, kind, T):  # noqa: F811
    """Enough tokens that a work-group takes 2, 4, 8 and 16: it starts inside pages and goes on
    into the next one, the last one of a sequence is not full."""
    import paper_2403_10266_amd as dsp
    r = np.random.default_rng(T)
    page, H, Hkv, D, rot = 16, 1, 1, 8, 8
    new = [T // 3 + 5, 0, 1, T // 2 + 3]
    new.append(T - sum(new))
    kv = [n + p for n, p in zip(new, (0, 9, 30, 7, 21))]
    table, pages = _table(r, kv, page)
    start, P, u = _rows_of(new), max(kv), 2.0 ** -8 if kind == "bf16" else 2.0 ** -24
    q, k, v = (wu.draw((T + 2, n * D), kind, r) for n in (H, Hkv, Hkv))
    ang = np.arange(P)[:, None] * 100.0 ** (-np.arange(rot // 2) / 2)
    cos, sin = (f(ang).astype(np.float32) for f in (np.cos, np.sin))
    caches = [_cache(torch, np.full((pages, page, Hkv, D), 3.0), kind, "token") for _ in "kv"]
    dq = dev(q, kind)
    got_q = dsp.dsp_kv_append(dev(k, kind), dev(v, kind), *caches, _i32(torch, table), _i32(torch, start), _i32(torch, kv),
                              cos=torch.from_numpy(cos).cuda(), sin=torch.from_numpy(sin).cuda(), q=dq,
                              out_q=torch.full_like(dq, 7.0))
    at = np.concatenate([np.arange(m - n, m) for n, m in zip(new, kv)])
    seq = np.repeat(np.arange(len(new)), new)
    g, slot = table[seq, at // page], at % page
    x = q[:T].reshape(T, H, D).astype(np.float64)
    _near(host(got_q)[:T].reshape(x.shape), ow.turned(x, at, cos, sin, False), x, at, cos, sin, u, "q")
    assert (got_q[T:] == 7).all()
    x = k[:T].reshape(T, Hkv, D).astype(np.float64)
    got = [_f64(c) for c in caches]
    _near(got[0][g, slot], ow.turned(x, at, cos, sin, False), x, at, cos, sin, u, "k")
    assert np.array_equal(got[1][g, slot], v[:T].reshape(T, Hkv, D))
    rest = np.ones((pages, page), bool)
    rest[g, slot] = False
    assert rest.any() and all((c[rest] == 3).all() for c in got)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("N,D", [(65, 16), (300, 16), (4200, 8), (3, 256), (2, 250)])
def test_append_of_many_sequences_and_of_wide_heads(torch, kind, N, D):  # noqa: F811
    """As many sequences as take a search of several levels, some without tokens; heads of 256."""
    import paper_2403_10266_amd as dsp
    r = np.random.default_rng(N + D)
    page, Hkv = 16, 2
    new = [int(n) for n in r.choice([0, 1, 2, 3, 20 if N < 1000 else 2], N)]
    kv = [n + int(p) for n, p in zip(new, r.integers(0, 40, N))]
    table, pages = _table(r, kv, page)
    T, start = sum(new), _rows_of(new)
    k, v = (wu.draw((T + 3, Hkv * D), "bf16", r) * np.exp2(r.integers(-3, 4, (T + 3, 1))).astype(np.float32) for _ in "kv")
    held = [r.integers(-8, 9, (pages, page, Hkv, D)) / 4.0 for _ in "kv"]
    scales = [2.0 ** r.integers(-9, -4, (pages, Hkv)) if kind == "e4m3" else None for _ in "kv"]
    caches = [_cache(torch, h, kind, "token") for h in held]
    dsc = [None if s is None else torch.from_numpy(s.astype(np.float32)).cuda() for s in scales]
    dsp.dsp_kv_append(dev(k, "bf16"), dev(v, "bf16"), *caches, _i32(torch, table), _i32(torch, start), _i32(torch, kv), *dsc)
    for x, h, s, c, d in zip((k, v), held, scales, caches, dsc):
        ow.append(x.reshape(-1, Hkv, D).astype(np.float64), h, table, start, kv, s)
        assert np.array_equal(_f64(c), h) and (s is None or np.array_equal(_f64(d), s))


@pytest.mark.parametrize("kind", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("N", [65, 130, 300])
def test_attention_of_many_sequences(torch, kind, N):  # noqa: F811
    """More sequences than are put in order by length, of unequal ones: none, one, a chunk."""
    import paper_2403_10266_amd as dsp
    r = np.random.default_rng(N)
    H, Hkv, D, page = 4, 2, 16, 16
    new = [int(n) for n in r.choice([0, 1, 1, 2, 17, 70], N)]
    new[-1] = 70
    kv = [n + int(p) for n, p in zip(new, r.integers(0, 90, N))]
    table, pages = _table(r, kv, page)
    dtype = "f32" if kind == "f32" else "bf16"
    held, scales = [wu.draw((pages, page, Hkv, D), dtype, r) for _ in "kv"], [None, None]
    if kind == "e4m3":
        scales = [2.0 ** r.integers(-4, 2, (pages, Hkv)) for _ in "kv"]
        held = [np.clip(ow.e4m3(h / s[:, None, :, None]), -448, 448) for h, s in zip(held, scales)]
    _attend(torch, dsp, r, kind, dtype, "token", table, held, scales, new, kv, H, Hkv, D, 50, 0, 2)


@pytest.mark.parametrize("left,sinks", [(-1, 0), (20, 2)])
@pytest.mark.parametrize("start,kv,max_q", [([5, 3, 1], [9, 9], 1), ([-5, 0, 900], [-1, 2147483647], 90),
                                            ([0, 90, 20], [2147483647, -2147483648], 90), ([90, 90, 90], [64, 64], 90),
                                            ([0, 40, 90], [50, 2147483647], 90), ([3, 3, 4], [-7, 64], 2)])
def test_tables_of_no_meaning_write_their_rows_only(torch, start, kv, max_q, left, sinks):  # noqa: F811
    """Row starts that fall or lie outside, lengths below 0 and past everything: rows of no
    sequence and what lies around the outputs stay, the others are those of the clamped starts."""
    import paper_2403_10266_amd as dsp
    r = np.random.default_rng(21)
    T, H, Hkv, D, page = 90, 4, 2, 64, 16
    held = [wu.draw((4, page, Hkv, D), "bf16", r) for _ in "kv"]
    q, table = wu.draw((T, H * D), "bf16", r), np.array([[0, 1, 2, 3], [3, 2, 1, 0]])
    out, lse = torch.full((3 * T, H * D), 7.0, device="cuda").bfloat16(), torch.full((3 * T, H), 7.0, device="cuda")
    dsp.dsp_attn_paged(dev(q, "bf16"), *(dev(h, "bf16") for h in held), _i32(torch, table), _i32(torch, start),
                       _i32(torch, kv), H, max_q=max_q, left=left, sinks=sinks, out=out[T:2 * T], lse=lse[T:2 * T])
    torch.cuda.synchronize()
    got, gl = host(out), host(lse)
    for t in (got, gl):
        assert (t[:T] == 7).all() and (t[2 * T:] == 7).all()
    a = np.clip(start, 0, T)
    b = np.maximum(a[1:], a[:-1])
    hk, hv = (h.astype(np.float64) for h in held)
    done = np.zeros(T, bool)
    for n in range(2):
        new = int(b[n] - a[n])
        if not new:
            continue
        rows, cap = slice(a[n], a[n] + min(new, max_q)), 4 * page
        done[rows] = True
        flat = lambda h: h[table[n]].reshape(1, 1, cap, Hkv * D)  # noqa: E731
        c = dict(q=q[None, None, rows], k=flat(hk), v=flat(hv), H=H, Hkv=Hkv)
        c["do"] = c["q"]
        want = wu.wanted(c, "bf16", left, 0, sinks, [kv[n] - new], [kv[n]], grads=False)
        wu.compare(dict(o=got[T:2 * T][rows], lse=gl[T:2 * T][rows].T), want, say)
    assert (got[T:2 * T][~done] == 7).all() and (gl[T:2 * T][~done] == 7).all()


@pytest.mark.parametrize("kind", ["f32", "bf16", "e4m3"])
@pytest.mark.parametrize("new", [2, 150])
def test_pages_far_apart(torch, kind, new):  # noqa: F811
    """Pages whose offsets pass 2^31 elements, keys and values in one buffer: the bits of a
    compact cache."""
    import paper_2403_10266_amd as dsp
    r = np.random.default_rng(22)
    pages, page, H, Hkv, D, step, kv = 300, 16, 4, 2, 64, 1 << 23, 400
    dtype = "f32" if kind == "f32" else "bf16"
    ct = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}[kind]
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB of free GPU memory")
    base = torch.empty(pages * step, dtype=ct, device="cuda")
    row = Hkv * D
    far = [base[i * row:].as_strided((pages, page, Hkv, D), (step, 2 * row, D, 1), i * row) for i in range(2)]
    near = [torch.zeros(pages, page, Hkv, D, dtype=ct, device="cuda") for _ in "kv"]
    table = _i32(torch, [np.concatenate([[299, 0, 298], r.permutation(np.arange(1, 298))[:22]])])
    k, v, q = (dev(wu.draw((kv, n * D), dtype, r), dtype) for n in (Hkv, Hkv, H))
    got = []
    for c in (far, near):
        s = [torch.zeros(pages, Hkv, device="cuda") for _ in "kv"] if kind == "e4m3" else [None, None]
        for lo, hi in ((0, 250), (250, kv)):
            dsp.dsp_kv_append(k[lo:hi], v[lo:hi], *c, table, _i32(torch, [0, hi - lo]), _i32(torch, [hi]), *s)
        o, lse = dsp.dsp_attn_paged(q[:new], *c, table, _i32(torch, [0, new]), _i32(torch, [kv]), H, max_q=new,
                                    k_scale=s[0], v_scale=s[1], with_lse=True)
        held = [t[table[0].long()].view(torch.uint8) if kind == "e4m3" else t[table[0].long()] for t in c]
        got.append([o, lse] + held + [t for t in s if t is not None])
    assert torch.isfinite(got[0][0].float()).all()
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_the_order_of_sequences_is_cheap(torch):  # noqa: F811
    """64 sequences, put in order by length, take the time of 65, which are not, with as many
    tokens: short passes over a narrow window, whose work-groups spend little else."""
    import paper_2403_10266_amd as dsp
    H, Hkv, D, page, T = 32, 8, 64, 64, 64 * 65 * 15
    times, calls = [[], []], []
    for N in (64, 65):
        n = T // N
        need = -(-n // page)
        cache = [torch.randn(N * need, page, Hkv, D, device="cuda").bfloat16() for _ in "kv"]
        q = torch.randn(T, H * D, device="cuda").bfloat16()
        args = (_i32(torch, np.arange(N * need).reshape(N, need)), _i32(torch, np.arange(N + 1) * n), _i32(torch, [n] * N))
        calls.append(lambda q=q, c=cache, a=args, n=n, o=torch.empty_like(q): dsp.dsp_attn_paged(q, *c, *a, H, max_q=n, left=31,
                                                                                                  out=o))
    ev = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
    for _ in range(12):
        for t, call in zip(times, calls):
            ev[0].record()
            for _ in range(10):
                call()
            ev[1].record()
            torch.cuda.synchronize()
            t.append(ev[0].elapsed_time(ev[1]))
    a, b = (min(t) * 100 for t in times)
    say(f"64 sequences {a:.0f} us, 65 {b:.0f} us")
    assert a < 1.3 * b


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_two_programs_at_once(torch, kind):  # noqa: F811
    """Appending and attending on two streams, and from two graphs replayed in turn and together,
    each with a cache and (its keys cut among work-groups) a workspace of its own."""
    import paper_2403_10266_amd as dsp
    r = np.random.default_rng(23)
    H, Hkv, D, page, kv = 8, 2, 64, 16, [3000, 2000]
    progs = []
    for new in (1, 40):
        table, pages = _table(r, kv, page)
        caches = [_cache(torch, np.clip(ow.e4m3(wu.draw((pages, page, Hkv, D), "bf16", r)), -448, 448), kind, "token")
                  for _ in "kv"]
        s = [torch.full((pages, Hkv), 1.0, device="cuda") for _ in "kv"] if kind == "e4m3" else [None, None]
        rows = [dev(wu.draw((2 * new, n * D), "bf16", r), "bf16") for n in (H, Hkv, Hkv)]
        at = (_i32(torch, table), _i32(torch, [0, new, 2 * new]), _i32(torch, kv))

        def call(stream=None, rows=rows, caches=caches, s=s, at=at, new=new):
            q = dsp.dsp_kv_append(rows[1], rows[2], *caches, *at, *s, q=rows[0], stream=stream)
            return [q, *dsp.dsp_attn_paged(q, *caches, *at, H, max_q=new, k_scale=s[0], v_scale=s[1], with_lse=True,
                                           stream=stream)]
        progs.append(call)
    want = [[x.clone() for x in call()] for call in progs]      # appending the same tokens again changes nothing
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in progs]
    for _ in range(4):
        got = [call(s) for call, s in zip(progs, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))
    graphs, outs = [], []
    for call in progs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(call())
        graphs.append(g)
    for together in (False, True, False, True):
        for o in outs:
            for x in o:
                x.fill_(7)
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s if together else streams[0]):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(outs, want) for a, b in zip(g, w))
