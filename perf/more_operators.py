"""Performance cases of windowed attention and of the paged cache: attention with a
window to either side and first tokens that stay visible (sinks), forward and
backward; the append of new keys and values to a cache of pages, with the position
rotation on the way; and attention of new tokens over such a cache, held in 16 or 32
bits or in 8 bits with a scale for each page and head.

Widths are those of the framework's other cases: 16 heads of 72 (C = 1152) and 32
heads of 64 (C = 2048), grouped key/value heads, and a few widths beside them.

``listed()`` gives the named cases, ``draw(rng)`` one more of the same ranges,
``prepare(case, seed)`` the inputs on the GPU, ``run(state)`` one pass (in plain
torch operations in 32 bits, or with ``own`` by the framework's entry points),
``work(case)`` the bytes and operations it cannot do without, and
``exact(case, seed)`` the results in 64 bits.

Formulas.  A query at position p sees the keys j < kv_len with j <= p + right (right
< 0: no bound) and with j >= p - left (left < 0: no bound) or j < sinks:
    o = sum_j softmax_j(q.k_j / sqrt(D)) v_j  over the keys it sees,
0 with a log-sum-exp of -inf where it sees none.
Pages: position p of sequence n lies in slot p % page of page table[n][p // page].
New tokens are rows q_start[n] .. q_start[n + 1] - 1 of the packed rows and the last
ones of the sequence's kv_len[n] positions.  In 8 bits (e4m3) a page holds x / s, s
the least power of two with |x| <= 448 s for all tokens that the page was given for
that head since its first slot was written; what the page holds is rounded again when
s grows.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

E4M3_MAX = 448.0
LEAST_EXP = -64              # of the scales' powers of two


def _dsp():
    import paper_2403_10266_amd as dsp
    return dsp


def listed():
    return [
        # temporal attention of 128 frames at each of 1024 locations, every frame seeing
        # 16 to either side and the first one: short rows, memory's case
        {"name": "window_temporal_T128", "kind": "window", "B": 1, "X": 1024, "Lq": 128, "Lk": 128, "H": 16, "Hkv": 16,
         "D": 72, "left": 16, "right": 16, "sinks": 1, "lens": "full", "train": False, "dtype": "bf16"},
        # one long causal sequence of the wider model, grouped heads: the matrix units' case
        {"name": "window_causal_8192", "kind": "window", "B": 1, "X": 1, "Lq": 8192, "Lk": 8192, "H": 32, "Hkv": 8,
         "D": 64, "left": 2047, "right": 0, "sinks": 4, "lens": "full", "train": False, "dtype": "bf16"},
        # training on frames of 64 x 64 latents, each token seeing two rows before and after
        {"name": "window_grad_S4096", "kind": "window", "B": 1, "X": 8, "Lq": 4096, "Lk": 4096, "H": 16, "Hkv": 16,
         "D": 72, "left": 128, "right": 128, "sinks": 0, "lens": "full", "train": True, "dtype": "bf16"},
        # training on causal sequences of unequal length, padded, with sinks, whose
        # gradients are sums over all later queries
        {"name": "window_grad_causal_4000", "kind": "window", "B": 4, "X": 1, "Lq": 4000, "Lk": 4000, "H": 32,
         "Hkv": 8, "D": 64, "left": 500, "right": 0, "sinks": 4, "lens": "ragged", "train": True, "dtype": "bf16"},
        # full-precision check run of a training step on odd sizes
        {"name": "window_grad_f32_odd", "kind": "window", "B": 3, "X": 3, "Lq": 77, "Lk": 150, "H": 6, "Hkv": 2,
         "D": 20, "left": 13, "right": 5, "sinks": 3, "lens": "ragged", "train": True, "dtype": "f32"},
        # one new token of each of 64 sequences into an 8-bit cache: the step of a
        # generating program, where the launch is what counts
        {"name": "append_token_8bit", "kind": "append", "N": 64, "new": 1, "kv": 2000, "page": 64, "H": 32, "Hkv": 8,
         "D": 64, "rot": 64, "pairs": "half", "ragged": True, "cache": "e4m3", "layout": "token", "dtype": "bf16"},
        # the first 16000 tokens of one long clip into a 16-bit cache: a pass over memory
        {"name": "append_chunk_16000", "kind": "append", "N": 1, "new": 16000, "kv": 16000, "page": 64, "H": 16,
         "Hkv": 16, "D": 72, "rot": 72, "pairs": "half", "ragged": False, "cache": "same", "layout": "token",
         "dtype": "bf16"},
        # chunks of many sequences, going on inside pages, into an 8-bit cache laid out by heads
        {"name": "append_ragged_8bit", "kind": "append", "N": 32, "new": 700, "kv": 3000, "page": 32, "H": 32,
         "Hkv": 8, "D": 128, "rot": 64, "pairs": "adjacent", "ragged": True, "cache": "e4m3", "layout": "head",
         "dtype": "bf16"},
        # one token of each of 64 sequences over an 8-bit cache of up to 16000 tokens: memory's case
        {"name": "paged_token_8bit", "kind": "paged", "N": 64, "new": 1, "kv": 16000, "page": 64, "H": 32, "Hkv": 8,
         "D": 64, "left": -1, "right": 0, "sinks": 0, "ragged": True, "cache": "e4m3", "layout": "token",
         "dtype": "bf16"},
        # the next frame's token of 200 streams that keep a window and their first frames;
        # pages before it were given back: many short stretches of long tables
        {"name": "paged_token_window", "kind": "paged", "N": 200, "new": 1, "kv": 9000, "page": 16, "H": 16,
         "Hkv": 16, "D": 72, "left": 500, "right": 0, "sinks": 4, "ragged": True, "cache": "same", "layout": "token",
         "dtype": "bf16"},
        # two tokens of one long sequence: few rows, all compute units to be filled
        {"name": "paged_long_2tokens", "kind": "paged", "N": 1, "new": 2, "kv": 100000, "page": 128, "H": 32,
         "Hkv": 8, "D": 128, "left": -1, "right": 0, "sinks": 0, "ragged": False, "cache": "same", "layout": "head",
         "dtype": "bf16"},
        # chunks of prompts of unequal length over their 8-bit caches: products count
        {"name": "paged_chunk_8bit", "kind": "paged", "N": 6, "new": 1000, "kv": 8000, "page": 64, "H": 32, "Hkv": 8,
         "D": 64, "left": -1, "right": 0, "sinks": 0, "ragged": True, "cache": "e4m3", "layout": "token",
         "dtype": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


HEADS = [(16, 16, 72), (16, 4, 72), (32, 8, 64), (32, 32, 64), (8, 2, 128), (4, 4, 40), (6, 3, 96), (12, 4, 80)]


def draw(rng):
    while True:
        dtype = rng.choice(["bf16", "bf16", "bf16", "bf16", "f32"])
        H, Hkv, D = rng.choice(HEADS)
        kind = rng.choice(["window", "window", "append", "paged", "paged"])
        left, sinks = rng.choice([-1, _log_int(rng, 1, 3000)]), rng.choice([0, 0, 1, 4, 7, 40])
        if kind == "window":
            shape = rng.choice(["temporal", "long", "token"])
            train = rng.random() < 0.5 and shape != "token"
            if shape == "temporal":
                B, X, Lq = rng.randint(1, 2), _log_int(rng, 16, 1024), _log_int(rng, 2, 128)
                Lk, left = Lq, _log_int(rng, 1, 64)
            elif shape == "long":
                B, X, Lq = rng.randint(1, 4), rng.randint(1, 4), _log_int(rng, 100, 8000)
                Lk = Lq if rng.random() < 0.7 else _log_int(rng, 100, 8000)
            else:
                B, X, Lq, Lk = rng.randint(1, 8), rng.choice([1, 1, 50]), rng.choice([1, 1, 2, 5]), _log_int(rng, 8, 20000)
            right = 0 if shape == "token" else rng.choice([0, 0, left, rng.randint(0, 100), -1])
            c = {"kind": kind, "B": B, "X": X, "Lq": Lq, "Lk": Lk, "H": H, "Hkv": Hkv, "D": D, "left": left,
                 "right": right, "sinks": sinks, "lens": rng.choice(["full", "ragged"]), "train": train,
                 "dtype": dtype}
            fits = B * X * H * Lq * Lk <= 2.2e9
        else:
            page = rng.choice([16, 32, 64, 64, 128, 256])
            cache = "same" if dtype == "f32" else rng.choice(["same", "e4m3", "e4m3"])
            layout, ragged, N = rng.choice(["token", "head"]), rng.random() < 0.7, _log_int(rng, 1, 200)
            new = rng.choice([1, 1, rng.randint(2, 8), _log_int(rng, 16, 2000)])
            kv = new + _log_int(rng, 1, 30000)
            if kind == "append":
                rot = rng.choice([D, D, 0, D // 16 * 8])
                c = {"kind": kind, "N": N, "new": new, "kv": min(kv, new + 3000), "page": page, "H": H, "Hkv": Hkv,
                     "D": D, "rot": rot, "pairs": rng.choice(["half", "adjacent"]), "ragged": ragged, "cache": cache,
                     "layout": layout, "dtype": dtype}
                fits = N * (c["kv"] + page) * Hkv * D <= 1.0e8
            else:
                c = {"kind": kind, "N": N, "new": new, "kv": kv, "page": page, "H": H, "Hkv": Hkv, "D": D,
                     "left": left, "right": rng.choice([0, 0, 0, -1]), "sinks": sinks, "ragged": ragged,
                     "cache": cache, "layout": layout, "dtype": dtype}
                fits = N * (kv + page) * Hkv * D <= 6.0e8 and N * H * new * kv <= 1.5e9
        if not fits:
            continue
        w = work(c)
        # full-precision steps take a check's sizes
        if w["flops"] <= (2.0e11 if dtype == "bf16" else 2.0e10) and w["bytes"] <= 8.0e8:
            return c


# --------------------------------------------------------------------------- inputs

def _window_lens(c):
    """Keys of each sequence of the batch: all of them, or from all down to none."""
    B, Lk = c["B"], c["Lk"]
    if c["lens"] == "full":
        return [Lk] * B
    return [Lk - (Lk * b) // max(B - 1, 1) if B > 2 else Lk - (Lk * b) // 3 for b in range(B)]


def _q_pos(c):
    """Position of the first query: a sequence's last ones where there are fewer queries
    than keys, its first ones otherwise."""
    return [n - c["Lq"] if c["Lq"] < c["Lk"] else 0 for n in _window_lens(c)]


def _paged_lens(c):
    """(new tokens, positions in all) of each sequence: all alike, or spread down to one
    new token and to a third of the positions; of four or more sequences one has no new
    tokens in a batch of chunks."""
    N, out = c["N"], []
    for n in range(N):
        new, kv = c["new"], c["kv"]
        if c["ragged"] and N > 1:
            new = max(1, new - (new * n) // N)
            if c["new"] > 1 and N > 3 and n == N - 2:
                new = 0
            kv = max(new, kv - (2 * kv * n) // (3 * N) - 5 * (n % 7))
        out.append((new, kv))
    return out


def _page_plan(c):
    """The table's physical pages (-1: none) as a list for each sequence, and their number.
    Pages that no new token sees were given back."""
    page, count, rows = c["page"], 0, []
    for new, kv in _paged_lens(c):
        row = []
        for g in range((kv + page - 1) // page):
            gone = c["kind"] == "paged" and c["left"] >= 0 and (g + 1) * page <= kv - new - c["left"] \
                and g * page >= c["sinks"]
            row.append(-1 if gone else count)
            count += not gone
        rows.append(row)
    return rows, count


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dt)

    s = dict(c)
    H, Hkv, D = c["H"], c["Hkv"], c["D"]
    if c["kind"] == "window":
        B, X, Lq, Lk = c["B"], c["X"], c["Lq"], c["Lk"]
        s["q"] = normal(B, X, Lq, H * D)
        s["k"], s["v"] = normal(B, X, Lk, Hkv * D), normal(B, X, Lk, Hkv * D)
        s["kv_len"] = torch.tensor(_window_lens(c), dtype=torch.int32, device="cuda")
        s["q_pos"] = torch.tensor(_q_pos(c), dtype=torch.int32, device="cuda")
        s["out"] = torch.empty(B, X, Lq, H * D, dtype=dt, device="cuda")
        if c["train"]:
            s["do"] = normal(B, X, Lq, H * D)
            s["grads"] = [torch.empty_like(s[n]) for n in ("q", "k", "v")]
        return s
    N, page, lens = c["N"], c["page"], _paged_lens(c)
    rows, count = _page_plan(c)
    order = torch.randperm(count, generator=g, device="cuda").cpu().numpy()
    table = np.full((N, max(len(r) for r in rows)), -1, np.int32)
    for n, row in enumerate(rows):
        table[n, :len(row)] = [order[i] if i >= 0 else -1 for i in row]
    s["table"] = torch.from_numpy(table).cuda()
    starts = np.concatenate([[0], np.cumsum([new for new, _ in lens])])
    s["q_start"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    s["kv_len"] = torch.tensor([kv for _, kv in lens], dtype=torch.int32, device="cuda")
    s["max_q"] = max(new for new, _ in lens)
    T = int(starts[-1]) + (3 if c["ragged"] else 0)      # a padded batch: rows of no sequence
    s["seq"] = torch.repeat_interleave(torch.arange(N), torch.tensor([new for new, _ in lens])).cuda()
    shape = (count, page, Hkv, D) if c["layout"] == "token" else (count, Hkv, page, D)
    for name in ("k", "v"):
        x = torch.randn(*shape, generator=g, device="cuda") * (1.5 if name == "k" else 1.0)
        x = x if c["layout"] == "token" else x.transpose(1, 2)      # [pages, page, Hkv, D]
        s[name + "_scale"] = None
        if c["cache"] == "e4m3":
            scale = _scale_of(x.abs().amax((1, 3)))
            s[name + "_scale"] = scale
            x = (x / scale[:, None, :, None]).to(torch.float8_e4m3fn)
        else:
            x = x.to(dt)
        s[name + "_cache"] = x
    s["q"] = normal(T, H * D)
    s["out"] = torch.zeros(T, H * D, dtype=dt, device="cuda")
    if c["kind"] == "paged":
        s["lse"] = torch.zeros(T, H, device="cuda")
    else:
        s["k"], s["v"] = normal(T, Hkv * D, scale=1.5), normal(T, Hkv * D)
        P, R = max(kv for _, kv in lens), c["rot"]
        ang = np.arange(P, dtype=np.float64)[:, None] * 10000.0 ** (-np.arange(R // 2, dtype=np.float64) * 2 / max(R, 1))
        s["cos"] = torch.from_numpy(np.cos(ang).astype(np.float32)).cuda() if R else None
        s["sin"] = torch.from_numpy(np.sin(ang).astype(np.float32)).cuda() if R else None
    return s


# --------------------------------------------------------------------------- the pass

def run(state):
    s = state
    if s["kind"] == "window":
        return _run_window(s)
    return _run_append(s) if s["kind"] == "append" else _run_paged(s)


def _run_window(s):
    if own:
        dsp = _dsp()
        kw = dict(left=s["left"], right=s["right"], sinks=s["sinks"], q_pos=s["q_pos"], kv_len=s["kv_len"])
        o, lse = dsp.dsp_attn_window(s["q"], s["k"], s["v"], s["H"], s["Hkv"], out=s["out"], with_lse=True, **kw)
        if not s["train"]:
            return {"o": o, "lse": lse}
        dq, dk, dv = dsp.dsp_attn_window_bwd(s["q"], s["k"], s["v"], o, s["do"], lse, s["H"], s["Hkv"],
                                             dq=s["grads"][0], dk=s["grads"][1], dv=s["grads"][2], **kw)
        return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}
    B, X, Lq, Lk, H, Hkv, D = (s[n] for n in ("B", "X", "Lq", "Lk", "H", "Hkv", "D"))
    G, dt = H // Hkv, s["q"].dtype
    pos = torch.arange(Lq, device="cuda")[None, :] + s["q_pos"].long()[:, None]
    hide = ~_sees(s, pos, s["kv_len"], Lk)[:, None, None, None]                  # [B, 1, 1, 1, Lq, Lk]

    def heads(x, n):  # [B, X, L, n D] -> fp32 [B, X, n, L, D]
        return x.float().reshape(B, X, -1, n, D).transpose(2, 3).contiguous()

    q = heads(s["q"], H).reshape(B, X, Hkv, G * Lq, D)
    k, v = heads(s["k"], Hkv), heads(s["v"], Hkv)
    z = (q @ k.transpose(-1, -2)).reshape(B, X, Hkv, G, Lq, Lk).mul_(1 / math.sqrt(D))
    p, lse = _softmax(z.masked_fill_(hide, -math.inf))
    p = p.reshape(B, X, Hkv, G * Lq, Lk)
    o = p @ v

    def back(x, n):  # [B, X, .., D] by heads -> [B, X, L, n D] of the inputs' type
        return x.reshape(B, X, n, -1, D).transpose(2, 3).reshape(B, X, -1, n * D).to(dt)

    out = {"o": back(o, H), "lse": lse.reshape(B, X, H, Lq)}
    if not s["train"]:
        return out
    do = heads(s["do"], H).reshape(B, X, Hkv, G * Lq, D)
    dv = p.transpose(-1, -2) @ do
    dz = (do @ v.transpose(-1, -2)).sub_((do * o).sum(-1, keepdim=True)).mul_(p).mul_(1 / math.sqrt(D))
    return out | {"dq": back(dz @ k, H), "dk": back(dz.transpose(-1, -2) @ q, Hkv), "dv": back(dv, Hkv)}


def _sees(s, pos, kv_len, Lk):
    """[.., Lq, Lk]: whether the query at pos [.., Lq] sees each key."""
    j, p = torch.arange(Lk, device="cuda"), pos[..., None]
    keep = (j < kv_len.long()[:, None, None]).expand(*pos.shape, Lk)
    if s["right"] >= 0:
        keep = keep & (j <= p + s["right"])
    if s["left"] >= 0:
        keep = keep & ((j >= p - s["left"]) | (j < s["sinks"]))
    return keep


def _softmax(z):
    """Probabilities (in z's memory) and log-sum-exp over the last axis; a row of -inf: 0 and -inf."""
    top = z.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = z.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    return p.div_(torch.where(total > 0, total, 1.0)), (top + total.log())[..., 0]


def _scale_of(top):
    """The least power of two s with top <= 448 s, by the parts of top's own bits."""
    m, e = torch.frexp(top)
    e = torch.where(m <= E4M3_MAX / 512, e - 9, e - 8)
    return torch.ldexp(torch.ones_like(top), torch.where(top > 0, e.clamp(min=LEAST_EXP), LEAST_EXP))


def _turned(s, x, rows):
    """x [T, n, D] in 32 bits with the pairs of its first rot elements turned by the rows' angles."""
    R = s["rot"]
    if not R:
        return x
    cos, sin = s["cos"][rows][:, None], s["sin"][rows][:, None]
    if s["pairs"] == "half":
        a, b = x[..., :R // 2], x[..., R // 2:R]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, x[..., R:]], -1)


def _run_append(s):
    if own:
        _dsp().dsp_kv_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["q_start"], s["kv_len"],
                             k_scale=s["k_scale"], v_scale=s["v_scale"], cos=s["cos"], sin=s["sin"],
                             interleaved=s["pairs"] == "adjacent", q=s["q"], out_q=s["out"])
    else:
        T, Hkv, D, page = s["seq"].shape[0], s["Hkv"], s["D"], s["page"]
        lens = (s["q_start"][1:] - s["q_start"][:-1]).long()
        first = s["kv_len"].long() - lens                            # position of each sequence's first new token
        at = first[s["seq"]] + torch.arange(T, device="cuda") - s["q_start"].long()[s["seq"]]
        pages, slots = s["table"].long()[s["seq"], at // page], at % page
        s["out"][:T] = _turned(s, s["q"][:T].float().reshape(T, -1, D), at).reshape(T, -1).to(s["out"].dtype)
        k = _turned(s, s["k"][:T].float().reshape(T, Hkv, D), at)
        v = s["v"][:T].float().reshape(T, Hkv, D)
        for x, cache, scale in ((k, s["k_cache"], s["k_scale"]), (v, s["v_cache"], s["v_scale"])):
            if scale is not None:
                _grow(s, x, cache, scale, pages, first, lens)
                x = x / scale[pages][..., None]
            cache[pages, slots] = x.to(cache.dtype)
    out = {"k": s["k_cache"], "v": s["v_cache"], "q": s["out"]}
    return out if s["k_scale"] is None else out | {"k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _grow(s, x, cache, scale, pages, first, lens):
    """The scales of the pages that x's tokens go to, with what the pages hold rounded again."""
    page, count = s["page"], scale.shape[0]
    # the slots that stay: those before the first new token, in the page that it goes on with
    stay = torch.zeros(count, dtype=torch.long, device="cuda")
    goes_on = torch.nonzero((first % page > 0) & (lens > 0))[:, 0]
    stay[s["table"].long()[goes_on, first[goes_on] // page]] = first[goes_on] % page
    touched = torch.unique(pages)
    top = torch.zeros_like(scale).index_reduce_(0, pages, x.abs().amax(-1), "amax")
    new = _scale_of(top)
    new = torch.where(stay[:, None] > 0, torch.maximum(new, scale), new)[touched]
    held = cache[touched].float() * (scale[touched] / new)[:, None, :, None]
    keeps = torch.arange(page, device="cuda")[None, :] < stay[touched][:, None]
    cache[touched] = torch.where(keeps[..., None, None], held, cache[touched].float()).to(cache.dtype)
    scale[touched] = new


def _run_paged(s):
    if own:
        dsp = _dsp()
        o, lse = dsp.dsp_attn_paged(s["q"], s["k_cache"], s["v_cache"], s["table"], s["q_start"], s["kv_len"], s["H"],
                                    max_q=s["max_q"], left=s["left"], right=s["right"], sinks=s["sinks"],
                                    k_scale=s["k_scale"], v_scale=s["v_scale"], out=s["out"], lse=s["lse"])
        return {"o": o, "lse": lse}
    N, H, Hkv, D, M = s["N"], s["H"], s["Hkv"], s["D"], s["max_q"]
    G, Lk = H // Hkv, s["table"].shape[1] * s["page"]
    i = torch.arange(M, device="cuda")
    start, lens = s["q_start"].long()[:-1], (s["q_start"][1:] - s["q_start"][:-1]).long()
    rows = (start[:, None] + i).clamp(max=s["q"].shape[0] - 1)                   # [N, M], padded
    pos = (s["kv_len"].long() - lens)[:, None] + i
    held = s["table"].long().clamp(min=0)

    def keys(cache, scale):  # [N, Hkv, Lk, D]
        x = cache[held].float()
        x = x if scale is None else x * scale[held][:, :, None, :, None]
        return x.permute(0, 3, 1, 2, 4).reshape(N, Hkv, Lk, D)

    q = s["q"].float()[rows].reshape(N, M, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(N, Hkv, G * M, D)
    z = (q @ keys(s["k_cache"], s["k_scale"]).transpose(-1, -2)).reshape(N, Hkv, G, M, Lk).mul_(1 / math.sqrt(D))
    p, lse = _softmax(z.masked_fill_(~_sees(s, pos, s["kv_len"], Lk)[:, None, None], -math.inf))
    o = p.reshape(N, Hkv, G * M, Lk) @ keys(s["v_cache"], s["v_scale"])
    o = o.reshape(N, Hkv, G, M, D).permute(0, 3, 1, 2, 4).reshape(N, M, H * D)
    T = s["seq"].shape[0]
    at = torch.arange(T, device="cuda") - start[s["seq"]]
    s["out"][:T] = o[s["seq"], at].to(s["out"].dtype)
    s["lse"][:T] = lse.reshape(N, H, M)[s["seq"], :, at]
    return {"o": s["out"], "lse": s["lse"]}


# --------------------------------------------------------------------------- floors

def _pairs(p0, count, kv, left, right, sinks):
    """(query, key) pairs that see one another, and the keys seen at all, for the queries at
    p0 .. p0 + count - 1."""
    if not count or kv <= 0:
        return 0, 0
    p = np.arange(p0, p0 + count, dtype=np.int64)
    hi = np.full(count, kv) if right < 0 else np.clip(p + right + 1, 0, kv)
    lo = np.zeros(count, np.int64) if left < 0 else np.clip(p - left, 0, hi)
    first = np.minimum(np.minimum(sinks, hi), lo)
    sink = int(first.max())
    return int((hi - lo + first).sum()), int(hi.max()) - max(int(lo.min()), sink) + sink


def work(case):
    c = case
    es = 2 if c["dtype"] == "bf16" else 4
    H, Hkv, D = c["H"], c["Hkv"], c["D"]
    if c["kind"] == "window":
        B, X = c["B"], c["X"]
        got = [_pairs(p0, c["Lq"], n, c["left"], c["right"], c["sinks"]) for n, p0 in zip(_window_lens(c), _q_pos(c))]
        pairs, keys = sum(g[0] for g in got) * X * H, sum(g[1] for g in got) * X * Hkv
        rows = B * X * c["Lq"] * H
        nbytes, flops = (2 * rows + 2 * keys) * D * es + rows * 4, 4 * pairs * D
        if c["train"]:  # q, k, v, o, do and lse read, dq, dk, dv of every row written
            nbytes += (4 * rows + 2 * keys + 2 * B * X * c["Lk"] * Hkv) * D * es + rows * 4
            flops += 10 * pairs * D
        return {"bytes": nbytes, "flops": flops}
    ec = 1 if c["cache"] == "e4m3" else es
    lens = _paged_lens(c)
    new = sum(n for n, _ in lens)
    if c["kind"] == "append":
        nbytes = new * (2 * H * D * es + 2 * Hkv * D * (es + ec)) + new * c["rot"] * 4
        if c["cache"] == "e4m3":  # scales read and written
            nbytes += sum((kv + c["page"] - 1) // c["page"] - (kv - n) // c["page"] for n, kv in lens if n) * Hkv * 16
        return {"bytes": nbytes, "flops": new * ((H + Hkv) * c["rot"] * 3 + 2 * Hkv * D)}
    got = [_pairs(kv - n, n, kv, c["left"], c["right"], c["sinks"]) for n, kv in lens]
    pairs, keys = sum(g[0] for g in got) * H, sum(g[1] for g in got) * Hkv
    return {"bytes": 2 * new * H * D * es + new * H * 4 + 2 * keys * D * ec, "flops": 4 * pairs * D}


# --------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"window": _exact_window, "append": _exact_append, "paged": _exact_paged}[case["kind"]](case, s)


def _exact_heads(q, k, v, p0, kv, c, do=None):
    """One sequence and key/value head: q [X, Lq, G, D], k and v [X, Lk, D] in 64 bits."""
    X, Lq, G, D = q.shape
    n = max(0, min(kv, k.shape[1]))
    i = np.arange(Lq)[:, None] + p0
    j = np.arange(n)[None, :]
    seen = np.ones((Lq, n), bool)
    if c["right"] >= 0:
        seen &= j - i <= c["right"]
    if c["left"] >= 0:
        seen &= (i - j <= c["left"]) | (j < c["sinks"])
    seen = torch.from_numpy(seen).to(q.device)
    o, lse = torch.zeros_like(q), torch.full((X, G, Lq), -math.inf, dtype=q.dtype, device=q.device)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    if n == 0:
        return o, lse, dq, dk, dv
    for g in range(G):
        qg = q[:, :, g].contiguous()
        z = torch.matmul(qg, k[:, :n].transpose(1, 2).contiguous()) / math.sqrt(D)
        z.masked_fill_(~seen, -math.inf)
        row = torch.logsumexp(z, -1)
        p = z.sub_(torch.where(torch.isinf(row), 0.0, row)[..., None]).exp_()
        lse[:, g] = row
        o[:, :, g] = torch.matmul(p, v[:, :n].contiguous())
        if do is None:
            continue
        dg = do[:, :, g].contiguous()
        dv[:, :n] += torch.matmul(p.transpose(1, 2).contiguous(), dg)
        dz = torch.matmul(dg, v[:, :n].transpose(1, 2).contiguous())
        dz = p * (dz - (p * dz).sum(-1, keepdim=True)) / math.sqrt(D)
        dq[:, :, g] = torch.matmul(dz, k[:, :n].contiguous())
        dk[:, :n] += torch.matmul(dz.transpose(1, 2).contiguous(), qg)
    return o, lse, dq, dk, dv


def _exact_window(c, s):
    B, X, H, Hkv, D, Lq = c["B"], c["X"], c["H"], c["Hkv"], c["D"], c["Lq"]
    G = H // Hkv
    split = lambda t, *n: t.double().reshape(B, X, -1, *n, D)  # noqa: E731
    q, k, v = split(s["q"], Hkv, G), split(s["k"], Hkv), split(s["v"], Hkv)
    do = split(s["do"], Hkv, G) if c["train"] else None
    o, dq, dk, dv = (torch.zeros_like(t) for t in (q, q, k, v))
    lse = torch.zeros(B, X, Hkv, G, Lq, dtype=torch.float64, device="cuda")
    for b, (n, p0) in enumerate(zip(_window_lens(c), _q_pos(c))):
        for e in range(Hkv):
            o[b, :, :, e], lse[b, :, e], dq[b, :, :, e], dk[b, :, :, e], dv[b, :, :, e] = _exact_heads(
                q[b, :, :, e], k[b, :, :, e], v[b, :, :, e], p0, n, c, None if do is None else do[b, :, :, e])
    flat = lambda t: t.reshape(B, X, t.shape[2], -1)  # noqa: E731
    out = {"o": flat(o), "lse": lse.reshape(B, X, H, Lq)}
    return out | {"dq": flat(dq), "dk": flat(dk), "dv": flat(dv)} if c["train"] else out


def _exact_paged(c, s):
    H, Hkv, D, page = c["H"], c["Hkv"], c["D"], c["page"]
    G = H // Hkv
    o, lse = s["out"].double(), s["lse"].double()
    table, row = s["table"].cpu().numpy(), 0
    for n, (new, kv) in enumerate(_paged_lens(c)):
        if new == 0:
            continue
        held = torch.from_numpy(np.maximum(table[n, :(kv + page - 1) // page], 0).astype(np.int64)).cuda()
        k, v = (s[m + "_cache"][held].to(torch.float32).double() for m in "kv")
        if c["cache"] == "e4m3":
            k, v = (x * s[m + "_scale"][held].double()[:, None, :, None] for x, m in ((k, "k"), (v, "v")))
        k, v = k.reshape(-1, Hkv, D), v.reshape(-1, Hkv, D)
        q = s["q"][row:row + new].double().reshape(new, Hkv, G, D)
        for e in range(Hkv):
            got = _exact_heads(q[None, :, e], k[None, :, e], v[None, :, e], kv - new, kv, c)
            o[row:row + new].view(new, Hkv, G, D)[:, e] = got[0][0]
            lse[row:row + new].view(new, Hkv, G)[:, e] = got[1][0].t()
        row += new
    return {"o": o, "lse": lse}


def _e4m3(x):
    """x in 64 bits rounded to the values of e4m3 (3 bits after the first, least exponent -6)."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_append(c, s):
    """Token runs page by page; a pair (a, b) turns as the complex number a + ib."""
    H, Hkv, D, R, page = c["H"], c["Hkv"], c["D"], c["rot"], c["page"]
    table, row, q_out = s["table"].cpu().numpy(), 0, s["out"].double()
    caches = {m: s[m + "_cache"].to(torch.float32).double() for m in "kv"}
    scales = {m: None if s[m + "_scale"] is None else s[m + "_scale"].double() for m in "kv"}
    i = torch.arange(R // 2, device="cuda")
    at = (i, i + R // 2) if c["pairs"] == "half" else (2 * i, 2 * i + 1)

    def turned(x, p0):
        if R == 0:
            return x
        by = torch.complex(s["cos"][p0:p0 + x.shape[0]].double(), s["sin"][p0:p0 + x.shape[0]].double())[:, None]
        z = torch.complex(x[..., at[0]], x[..., at[1]]) * by
        x = x.clone()
        x[..., at[0]], x[..., at[1]] = z.real, z.imag
        return x

    for n, (new, kv) in enumerate(_paged_lens(c)):
        if new == 0:
            continue
        p0, rows = kv - new, slice(row, row + new)
        q_out[rows] = turned(s["q"][rows].double().reshape(new, H, D), p0).reshape(new, -1)
        k, v = turned(s["k"][rows].double().reshape(new, Hkv, D), p0), s["v"][rows].double().reshape(new, Hkv, D)
        at0 = p0
        while at0 < kv:
            g, slot = int(table[n, at0 // page]), at0 % page
            stop = min(kv, at0 + page - slot)
            for m, x in (("k", k[at0 - p0:stop - p0]), ("v", v[at0 - p0:stop - p0])):
                if scales[m] is not None:
                    top = x.abs().amax((0, 2))
                    grown = torch.exp2(torch.ceil(torch.log2((top / E4M3_MAX).clamp(min=2.0 ** LEAST_EXP))))
                    if slot:
                        grown = torch.maximum(grown, scales[m][g])
                        caches[m][g, :slot] = _e4m3(caches[m][g, :slot] * (scales[m][g] / grown)[:, None])
                    scales[m][g] = grown
                    x = _e4m3(x / grown[:, None])
                caches[m][g, slot:slot + x.shape[0]] = x
            at0 = stop
        row += new
    out = {"k": caches["k"], "v": caches["v"], "q": q_out}
    return out if scales["k"] is None else out | {"k_scale": scales["k"], "v_scale": scales["v"]}
