"""Performance cases of the position operators of attention: the norm of queries
and keys for each head with the position rotation in the same pass, and attention
with a learned relative position bias by buckets; forward, backward, and the form
for single tokens against a cache.

Widths are those of the framework's other cases: 16 heads of 72 (C = 1152) and 32
heads of 64 (C = 2048), grouped key/value heads, and a few widths beside them.

``listed()`` gives the named cases, ``draw(rng)`` one more of the same ranges,
``prepare(case, seed)`` the inputs on the GPU, ``run(state)`` one pass (in plain
torch operations in 32 bits, or with ``own`` by the framework's entry points),
``work(case)`` the bytes and operations it cannot do without, and
``exact(case, seed)`` the results in 64 bits.

Formulas.  Norm and rotation, for each token and head x of width D:
    n = g * x / sqrt(mean(x^2) + eps),   y = R(p) n,
R(p) turning the pairs of the first R elements by the angles of position p's row of
a table of cosines and sines; pairs (2i, 2i + 1) or (i, i + R/2).
Attention: s_ij = scale q_i.k_j + bias[bucket(j - i - q_pos)], softmax over the keys
j < kv_len (and j <= i + q_pos when causal), o = P v.  A row without keys is 0 with
a log-sum-exp of -inf.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

EPS = 1e-6


def _dsp():
    import paper_2403_10266_amd as dsp
    return dsp


def listed():
    return [
        # one new token of each of 8 sequences: the step of a generating program,
        # where the launch is what counts
        {"name": "qknorm_token_8seq", "kind": "norm", "B": 8, "X": 1, "L": 1, "H": 16, "Hkv": 16, "D": 72, "rot": 72,
         "pairs": "half", "packed": True, "offset": True, "train": False, "dtype": "bf16"},
        # queries and keys of the packed projection of one 32-frame block, frames of
        # 32 x 32: spatial positions along L
        {"name": "qknorm_packed_S1024", "kind": "norm", "B": 1, "X": 32, "L": 1024, "H": 16, "Hkv": 16, "D": 72,
         "rot": 72, "pairs": "half", "packed": True, "offset": False, "train": False, "dtype": "bf16"},
        # the same for a long clip of the wider model, rotated in adjacent pairs: the
        # largest pass over memory
        {"name": "qknorm_wide_T64_S2025", "kind": "norm", "B": 1, "X": 2025, "L": 64, "H": 32, "Hkv": 32, "D": 64,
         "rot": 64, "pairs": "adjacent", "packed": False, "offset": False, "train": False, "dtype": "bf16"},
        # its gradients in a training step on two 17-frame clips of 20 x 20 latents
        {"name": "qknorm_grad_T17_S400", "kind": "norm", "B": 2, "X": 400, "L": 17, "H": 16, "Hkv": 16, "D": 72,
         "rot": 72, "pairs": "half", "packed": True, "offset": False, "train": True, "dtype": "bf16"},
        # full-precision check run: grouped heads of an odd width, half of it rotated
        {"name": "qknorm_grad_f32_odd", "kind": "norm", "B": 3, "X": 5, "L": 333, "H": 6, "Hkv": 2, "D": 44,
         "rot": 22, "pairs": "adjacent", "packed": False, "offset": True, "train": True, "dtype": "f32"},
        # temporal attention of 32 frames at each of 1024 locations: short rows, each
        # with the whole bias table
        {"name": "relpos_temporal_T32", "kind": "attn", "B": 1, "X": 1024, "Lq": 32, "Lk": 32, "H": 16, "Hkv": 16,
         "D": 72, "nb": 32, "M": 128, "causal": False, "lens": "full", "train": False, "dtype": "bf16"},
        # long sequences: nearly every key is further than the table reaches
        {"name": "relpos_long_4096", "kind": "attn", "B": 1, "X": 8, "Lq": 4096, "Lk": 4096, "H": 16, "Hkv": 16,
         "D": 72, "nb": 32, "M": 128, "causal": False, "lens": "full", "train": False, "dtype": "bf16"},
        # the next frame at each of 1024 locations against caches of up to 120 frames
        # in a batch of two, grouped heads: many short caches
        {"name": "relpos_token_many", "kind": "attn", "B": 2, "X": 1024, "Lq": 1, "Lk": 120, "H": 16, "Hkv": 4,
         "D": 72, "nb": 32, "M": 128, "causal": True, "lens": "ragged", "train": False, "dtype": "bf16"},
        # one token of each of four sequences against long caches: few rows, many keys
        {"name": "relpos_token_long", "kind": "attn", "B": 4, "X": 1, "Lq": 1, "Lk": 50000, "H": 32, "Hkv": 8,
         "D": 64, "nb": 32, "M": 128, "causal": True, "lens": "ragged", "train": False, "dtype": "bf16"},
        # training: temporal attention of 49 frames, forward and gradients
        {"name": "relpos_grad_T49", "kind": "attn", "B": 1, "X": 1350, "Lq": 49, "Lk": 49, "H": 16, "Hkv": 16,
         "D": 72, "nb": 32, "M": 64, "causal": False, "lens": "full", "train": True, "dtype": "bf16"},
        # training: causal sequences of unequal length, padded
        {"name": "relpos_grad_causal_2000", "kind": "attn", "B": 4, "X": 1, "Lq": 2000, "Lk": 2000, "H": 32, "Hkv": 8,
         "D": 64, "nb": 32, "M": 128, "causal": True, "lens": "ragged", "train": True, "dtype": "bf16"},
        # full-precision check run of a training step on odd sizes
        {"name": "relpos_grad_f32_odd", "kind": "attn", "B": 3, "X": 3, "Lq": 77, "Lk": 150, "H": 6, "Hkv": 2,
         "D": 20, "nb": 15, "M": 40, "causal": False, "lens": "ragged", "train": True, "dtype": "f32"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        train = rng.random() < 0.45
        if rng.random() < 0.4:
            H, Hkv, D = rng.choice([(16, 16, 72), (32, 32, 64), (8, 2, 128), (12, 4, 80), (6, 6, 40), (4, 1, 96)])
            rot = rng.choice([D, D, D // 4 * 2])
            c = {"kind": "norm", "B": rng.randint(1, 4), "X": _log_int(rng, 1, 1024), "L": _log_int(rng, 1, 4096),
                 "H": H, "Hkv": Hkv, "D": D, "rot": rot, "pairs": rng.choice(["half", "adjacent"]),
                 "packed": H == Hkv and rng.random() < 0.5, "offset": rng.random() < 0.4, "train": train,
                 "dtype": dtype}
        else:
            H, Hkv, D = rng.choice([(16, 16, 72), (16, 4, 72), (32, 8, 64), (32, 32, 64), (8, 2, 128), (4, 4, 40),
                                    (6, 3, 96)])
            shape = rng.choice(["temporal", "long", "token"])
            if shape == "temporal":
                B, X, Lq = rng.randint(1, 2), _log_int(rng, 16, 2048), _log_int(rng, 2, 128)
                Lk = Lq
            elif shape == "long":
                B, X, Lq = rng.randint(1, 4), rng.randint(1, 4), _log_int(rng, 100, 4096)
                Lk = Lq if rng.random() < 0.7 else _log_int(rng, 50, 4096)
            else:
                B, X, Lq = rng.randint(1, 8), rng.choice([1, 1, 50, 700]), rng.choice([1, 1, 2, 5])
                Lk = _log_int(rng, 8, 60000 if X == 1 else 400)
                train = False
            M = rng.choice([16, 64, 128, 200])
            c = {"kind": "attn", "B": B, "X": X, "Lq": Lq, "Lk": Lk, "H": H, "Hkv": Hkv, "D": D,
                 "nb": rng.choice([8, 15, 32, 33]), "M": M, "causal": shape == "token" or (Lq == Lk and rng.random() < 0.5),
                 "lens": rng.choice(["full", "ragged"]), "train": train, "dtype": dtype}
        w = work(c)
        # full-precision steps take a training setup's check sizes
        most = 6.0e11 if dtype == "bf16" else 1.0e10
        if w["flops"] <= most and w["bytes"] <= 1.0e9:
            return c


# --------------------------------------------------------------------------- inputs

def _lens(c):
    """Keys of each sequence of the batch: all of them, or from all down to none."""
    B, Lk = c["B"], c["Lk"]
    if c["lens"] == "full":
        return [Lk] * B
    return [Lk - (Lk * b) // max(B - 1, 1) if B > 2 else Lk - (Lk * b) // 3 for b in range(B)]


def _q_pos(c):
    """Position of the first query: the last ones of the sequence for a cache's new
    tokens, the first ones otherwise."""
    if c["causal"] and c["Lq"] < c["Lk"]:
        return [n - c["Lq"] for n in _lens(c)]
    return [0] * c["B"]


def _buckets(M, nb, causal):
    """Bucket of each distance j - i in -M .. M: exact near 0, then evenly in the
    logarithm; with both directions, half of the buckets for each."""
    out = np.zeros(2 * M + 1, np.int32)
    for d in range(-M, M + 1):
        n, base, half = -d, 0, nb
        if not causal:
            half = max(nb // 2, 1)
            base, n = (half if d > 0 else 0), abs(d)
        n = max(n, 0)
        near = max(half // 2, 1)
        if n >= near:
            far = near + math.floor(math.log(n / near) / math.log(max(M / near, 1.001)) * (half - near) + 1e-9)
            n = min(far, half - 1)
        out[d + M] = min(base + n, nb - 1)
    return out


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32

    def normal(*shape, scale=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dt)

    s = dict(c)
    B, X, H, Hkv, D = c["B"], c["X"], c["H"], c["Hkv"], c["D"]
    if c["kind"] == "norm":
        L, R = c["L"], c["rot"]
        if c["packed"]:  # the projection's [Q | K | V] buffer
            qkv = normal(B, X, L, 3 * H * D, scale=1.5)
            s["q"], s["k"] = qkv[..., :H * D], qkv[..., H * D:2 * H * D]
        else:
            s["q"], s["k"] = normal(B, X, L, H * D, scale=1.5), normal(B, X, L, Hkv * D, scale=0.7)
        s["gq"] = (1 + 0.1 * torch.randn(D, generator=g, device="cuda")).to(dt)
        s["gk"] = (1 + 0.1 * torch.randn(D, generator=g, device="cuda")).to(dt)
        P = L + 1000 if c["offset"] else L
        ang = np.arange(P, dtype=np.float64)[:, None] * 10000.0 ** (-np.arange(R // 2, dtype=np.float64) * 2 / R)
        s["cos"] = torch.from_numpy(np.cos(ang).astype(np.float32)).cuda()
        s["sin"] = torch.from_numpy(np.sin(ang).astype(np.float32)).cuda()
        s["pos"] = None
        if c["offset"]:  # each sequence at a place of its own
            start = torch.randint(0, 1000, (B, 1), generator=g, device="cuda")
            s["pos"] = (start + torch.arange(L, device="cuda")).to(torch.int32)
        s["out"] = [torch.empty(B, X, L, n * D, dtype=dt, device="cuda") for n in (H, Hkv)]
        if c["train"]:
            s["dy"] = [normal(B, X, L, n * D) for n in (H, Hkv)]
        return s
    Lq, Lk = c["Lq"], c["Lk"]
    s["q"] = normal(B, X, Lq, H * D)
    s["k"], s["v"] = normal(B, X, Lk, Hkv * D), normal(B, X, Lk, Hkv * D)
    s["bias"] = normal(c["nb"], H)
    s["buckets"] = torch.from_numpy(_buckets(c["M"], c["nb"], c["causal"])).cuda()
    s["kv_len"] = torch.tensor(_lens(c), dtype=torch.int32, device="cuda")
    s["q_pos"] = torch.tensor(_q_pos(c), dtype=torch.int32, device="cuda")
    s["out"] = torch.empty(B, X, Lq, H * D, dtype=dt, device="cuda")
    if c["train"]:
        s["do"] = normal(B, X, Lq, H * D)
        s["grads"] = [torch.empty_like(s[n]) for n in ("q", "k", "v")]
    return s


# --------------------------------------------------------------------------- the pass

def run(state):
    s = state
    if s["kind"] == "norm":
        return _run_norm(s)
    return _run_attn(s)


def _run_norm(s):
    if own:
        dsp = _dsp()
        kw = dict(pos=s["pos"], interleaved=s["pairs"] == "adjacent", eps=EPS)
        if s["train"]:
            dq, dk, dgq, dgk = dsp.dsp_qk_norm_rope_bwd(s["q"], s["k"], s["dy"][0], s["dy"][1], s["H"], s["Hkv"],
                                                        s["gq"], s["gk"], s["cos"], s["sin"], dq=s["out"][0],
                                                        dk=s["out"][1], **kw)
            return {"dq": dq, "dk": dk, "dgq": dgq, "dgk": dgk}
        yq, yk = dsp.dsp_qk_norm_rope(s["q"], s["k"], s["H"], s["Hkv"], s["gq"], s["gk"], s["cos"], s["sin"],
                                      out_q=s["out"][0], out_k=s["out"][1], **kw)
        return {"yq": yq, "yk": yk}
    if s["train"]:
        dq, dgq = _plain_norm_grad(s, s["q"], s["dy"][0], s["H"], s["gq"])
        dk, dgk = _plain_norm_grad(s, s["k"], s["dy"][1], s["Hkv"], s["gk"])
        return {"dq": dq, "dk": dk, "dgq": dgq, "dgk": dgk}
    return {"yq": _plain_norm(s, s["q"], s["H"], s["gq"]), "yk": _plain_norm(s, s["k"], s["Hkv"], s["gk"])}


def _rows(s):
    """cos and sin of the tokens, to spread over [B, X, L, heads, R / 2]."""
    if s["pos"] is None:
        return s["cos"][None, None, :, None, :], s["sin"][None, None, :, None, :]
    at = s["pos"].long()
    return s["cos"][at][:, None, :, None, :], s["sin"][at][:, None, :, None, :]


def _turn(s, x, cos, sin):
    """x [.., D] with the pairs of its first rot elements turned by the angles."""
    R = s["rot"]
    if s["pairs"] == "half":
        a, b = x[..., :R // 2], x[..., R // 2:R]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, x[..., R:]], -1) if R < x.shape[-1] else turned


def _plain_norm(s, x, heads, gain):
    B, X, L, _ = x.shape
    f = x.float().reshape(B, X, L, heads, s["D"])
    n = f * torch.rsqrt((f * f).mean(-1, keepdim=True) + EPS) * gain.float()
    return _turn(s, n, *_rows(s)).reshape(B, X, L, -1).to(x.dtype)


def _plain_norm_grad(s, x, dy, heads, gain):
    B, X, L, _ = x.shape
    f = x.float().reshape(B, X, L, heads, s["D"])
    r = torch.rsqrt((f * f).mean(-1, keepdim=True) + EPS)
    cos, sin = _rows(s)
    dn = _turn(s, dy.float().reshape(f.shape), cos, -sin)
    dg = (dn * f * r).sum((0, 1, 2, 3), dtype=torch.float64).float()
    w = dn * gain.float()
    dx = r * w - f * (r * r * r * (w * f).mean(-1, keepdim=True))
    return dx.reshape(B, X, L, -1).to(x.dtype), dg


def _run_attn(s):
    if own:
        dsp = _dsp()
        kw = dict(causal=s["causal"], q_pos=s["q_pos"], kv_len=s["kv_len"])
        o, lse = dsp.dsp_attn_relpos(s["q"], s["k"], s["v"], s["H"], s["Hkv"], s["bias"], s["buckets"], out=s["out"],
                                     with_lse=True, **kw)
        if not s["train"]:
            return {"o": o, "lse": lse}
        dq, dk, dv, db = dsp.dsp_attn_relpos_bwd(s["q"], s["k"], s["v"], o, s["do"], lse, s["H"], s["Hkv"], s["bias"],
                                                 s["buckets"], dq=s["grads"][0], dk=s["grads"][1], dv=s["grads"][2],
                                                 **kw)
        return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv, "dbias": db}
    B, X, Lq, Lk, H, Hkv, D = (s[n] for n in ("B", "X", "Lq", "Lk", "H", "Hkv", "D"))
    G, dt = H // Hkv, s["q"].dtype
    j = torch.arange(Lk, device="cuda")
    dist = j[None, None, :] - torch.arange(Lq, device="cuda")[None, :, None] - s["q_pos"].long()[:, None, None]
    keep = (j[None, None, :] < s["kv_len"][:, None, None]).expand(B, Lq, Lk)
    if s["causal"]:
        keep = keep & (dist <= 0)
    keep = keep[:, None, None, None]                              # [B, 1, 1, 1, Lq, Lk]
    bucket = s["buckets"].long()[dist.clamp(-s["M"], s["M"]) + s["M"]]
    bias = s["bias"].float().t().reshape(Hkv, G, -1)[:, :, bucket].permute(2, 0, 1, 3, 4)[:, None]

    def heads(x, n):  # [B, X, L, n D] -> fp32 [B, X, n, L, D]
        return x.float().reshape(B, X, -1, n, D).transpose(2, 3).contiguous()

    q = heads(s["q"], H).reshape(B, X, Hkv, G * Lq, D)
    k, v = heads(s["k"], Hkv), heads(s["v"], Hkv)
    scale = 1 / math.sqrt(D)
    z = (q @ k.transpose(-1, -2)).reshape(B, X, Hkv, G, Lq, Lk).mul_(scale).add_(bias)
    z.masked_fill_(~keep, -math.inf)
    top = z.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = z.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (top + total.log()).reshape(B, X, H, Lq)
    p.div_(torch.where(total > 0, total, 1.0))
    o = (p.reshape(B, X, Hkv, G * Lq, Lk) @ v).reshape(B, X, H, Lq, D)

    def back(x, n):  # [B, X, n, L, D] -> [B, X, L, n D] of the inputs' type
        return x.reshape(B, X, n, -1, D).transpose(2, 3).reshape(B, X, -1, n * D).to(dt)

    if not s["train"]:
        return {"o": back(o, H), "lse": lse}
    do = heads(s["do"], H).reshape(B, X, Hkv, G * Lq, D)
    dv = p.reshape(B, X, Hkv, G * Lq, Lk).transpose(-1, -2) @ do
    dp = (do @ v.transpose(-1, -2)).reshape(B, X, Hkv, G, Lq, Lk)
    delta = (do * o.reshape(do.shape)).sum(-1).reshape(B, X, Hkv, G, Lq, 1)
    dz = dp.sub_(delta).mul_(p)
    flat = dz.reshape(B, X, Hkv, G * Lq, Lk)
    dq = (flat @ k) * scale
    dk = (flat.transpose(-1, -2) @ q) * scale
    # the sum along each distance: rows moved so that a distance is a column
    per = torch.zeros(B, H, Lq, Lk + Lq, dtype=torch.float64, device="cuda")
    per[..., :Lk] = dz.reshape(B, X, H, Lq, Lk).sum(1, dtype=torch.float64).flip(2)
    cols = per.reshape(B, H, -1)[..., :Lq * (Lk + Lq - 1)].reshape(B, H, Lq, Lk + Lq - 1).sum(2)
    at = torch.arange(Lk + Lq - 1, device="cuda") - (Lq - 1) - s["q_pos"].long()[:, None]
    at = s["buckets"].long()[at.clamp(-s["M"], s["M"]) + s["M"]].reshape(-1)
    db = torch.zeros(s["nb"], H, dtype=torch.float64, device="cuda")
    db.index_add_(0, at, cols.transpose(1, 2).reshape(-1, H))
    return {"o": back(o, H), "lse": lse, "dq": back(dq, H), "dk": back(dk, Hkv), "dv": back(dv, Hkv),
            "dbias": db.to(dt)}


# --------------------------------------------------------------------------- floors

def work(case):
    c = case
    es = 2 if c["dtype"] == "bf16" else 4
    B, X, H, Hkv, D = c["B"], c["X"], c["H"], c["Hkv"], c["D"]
    if c["kind"] == "norm":
        tokens, heads = B * X * c["L"], H + Hkv
        table = (B * c["L"] if c["offset"] else c["L"]) * c["rot"] * 4
        n = tokens * heads * D
        if c["train"]:  # x and dy read, dx written; dn, its two sums, dx
            return {"bytes": 3 * n * es + table + 2 * D * (es + 4), "flops": 15 * n}
        return {"bytes": 2 * n * es + table + 2 * D * es, "flops": 7 * n}
    Lq, Lk = c["Lq"], c["Lk"]
    pairs = keys = 0
    for n, first in zip(_lens(c), _q_pos(c)):
        if c["causal"]:  # sum over i < Lq of the keys j <= first + i, j < n
            a, b = min(max(first + 1, 0), n), min(max(first + Lq, 0), n)
            rows = [min(max(first + i + 1, 0), n) for i in range(Lq)]
            pairs, keys = pairs + sum(rows), keys + b
        else:
            pairs, keys = pairs + Lq * n, keys + n
    pairs, rows, keys = pairs * X * H, B * X * Lq * H, keys * X * Hkv
    nbytes = (2 * rows + 2 * keys) * D * es + rows * 4 + c["nb"] * H * es + (2 * c["M"] + 1) * 4
    flops = 4 * pairs * D
    if c["train"]:  # the gradients read q, k, v, o, do and lse, and write dq, dk, dv of every row
        nbytes += (4 * rows + 2 * keys + 2 * B * X * Lk * Hkv) * D * es + rows * 4 + c["nb"] * H * es
        flops += 10 * pairs * D
    return {"bytes": nbytes, "flops": flops}


# --------------------------------------------------------------------------- 64 bits

def exact(case, seed):
    c, s = case, prepare(case, seed)
    B, X, H, Hkv, D = c["B"], c["X"], c["H"], c["Hkv"], c["D"]
    if c["kind"] == "norm":
        out = [_exact_norm(c, s, s["q"], H, s["gq"], 0), _exact_norm(c, s, s["k"], Hkv, s["gk"], 1)]
        if c["train"]:
            return {"dq": out[0][0], "dk": out[1][0], "dgq": out[0][1], "dgk": out[1][1]}
        return {"yq": out[0], "yk": out[1]}
    Lq, Lk, G, M, dev = c["Lq"], c["Lk"], H // Hkv, c["M"], "cuda"
    o = torch.zeros(B, X, Lq, H, D, dtype=torch.float64, device=dev)
    lse = torch.full((B, X, H, Lq), -math.inf, dtype=torch.float64, device=dev)
    dq, dk, dv = torch.zeros_like(o), *(torch.zeros(B, X, Lk, Hkv, D, dtype=torch.float64, device=dev)
                                        for _ in range(2))
    db = torch.zeros(H, c["nb"], dtype=torch.float64, device=dev)
    split = lambda t, n: t.double().reshape(B, X, -1, n, D)  # noqa: E731
    q, k, v = split(s["q"], H), split(s["k"], Hkv), split(s["v"], Hkv)
    do = split(s["do"], H) if c["train"] else None
    for b, (n, first) in enumerate(zip(_lens(c), _q_pos(c))):
        if n == 0:
            continue
        d = np.arange(n)[None, :] - (np.arange(Lq)[:, None] + first)
        which = torch.from_numpy(s["buckets"].cpu().numpy()[np.clip(d, -M, M) + M].astype(np.int64)).to(dev)
        hide = torch.from_numpy(d > 0).to(dev) if c["causal"] else None
        for h in range(H):
            e = h // G
            z = torch.matmul(q[b, :, :, h], k[b, :, :n, e].transpose(1, 2).contiguous()) / math.sqrt(D)
            z = z + s["bias"].double()[:, h][which]
            if hide is not None:
                z = z.masked_fill(hide, -math.inf)
            row = torch.logsumexp(z, -1)
            p = torch.exp(z - torch.where(torch.isinf(row), 0.0, row)[..., None])
            lse[b, :, h] = row
            o[b, :, :, h] = torch.matmul(p, v[b, :, :n, e].contiguous())
            if not c["train"]:
                continue
            dv[b, :, :n, e] += torch.matmul(p.transpose(1, 2), do[b, :, :, h].contiguous())
            dp = torch.matmul(do[b, :, :, h], v[b, :, :n, e].transpose(1, 2).contiguous())
            dz = p * (dp - (p * dp).sum(-1, keepdim=True))
            dq[b, :, :, h] = torch.matmul(dz, k[b, :, :n, e].contiguous()) / math.sqrt(D)
            dk[b, :, :n, e] += torch.matmul(dz.transpose(1, 2), q[b, :, :, h].contiguous()) / math.sqrt(D)
            db[h] += torch.bincount(which.reshape(-1), weights=dz.sum(0).reshape(-1), minlength=c["nb"])
    flat = lambda t: t.reshape(B, X, t.shape[2], -1)  # noqa: E731
    res = {"o": flat(o), "lse": lse}
    if c["train"]:
        res |= {"dq": flat(dq), "dk": flat(dk), "dv": flat(dv), "dbias": db.t().contiguous()}
    return res


def _exact_norm(c, s, x, heads, gain, which):
    """The pass by complex numbers: a pair (a, b) is a + ib, its turn a product."""
    B, X, L, D, R = c["B"], c["X"], c["L"], c["D"], c["rot"]
    f = x.double().reshape(B, X, L, heads, D)
    turn = torch.complex(s["cos"].double(), s["sin"].double())
    turn = turn[:L][None].expand(B, L, R // 2) if s["pos"] is None else turn[s["pos"].long()]
    turn = turn[:, None, :, None]
    i = torch.arange(R // 2, device="cuda")
    at = (i, i + R // 2) if c["pairs"] == "half" else (2 * i, 2 * i + 1)

    def turned(t, by):
        z = torch.complex(t[..., at[0]], t[..., at[1]]) * by
        t = t.clone()
        t[..., at[0]], t[..., at[1]] = z.real, z.imag
        return t

    size = (f.square().sum(-1, keepdim=True) / D + EPS).sqrt()
    unit = f / size
    if not c["train"]:
        return turned(unit * gain.double(), turn).reshape(B, X, L, -1)
    dn = turned(s["dy"][which].double().reshape(f.shape), turn.conj())
    dg = (dn * unit).sum((0, 1, 2, 3))
    du = dn * gain.double()
    dx = (du - unit * (du * unit).sum(-1, keepdim=True) / D) / size
    return dx.reshape(B, X, L, -1), dg
