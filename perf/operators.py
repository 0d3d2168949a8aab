"""Attention with score modifiers and the fused block norm, as measurable cases.

A case is one pass through one operator, on inputs that lie in device memory:

  attn        attention whose scores are capped, biased by distance or masked
              (causal, visible prefix, documents), query heads sharing K/V
              heads; with ``train`` its gradient follows
  norm        the step between two sublayers of a block: the branch (normalised
              first, or not) gated onto the residual stream, the sum normalised
              and modulated for the next sublayer; with ``train`` the gradient
              of that step alone, from the stream that the forward left

``run`` computes the plain form of a case where ``own`` is false, and calls the
package where it is true.
"""

import math

import torch

own = False

D = 128
EPS = 1e-6


def listed():
    return [
        # one new token against a short cache: launch latency
        {"name": "token_small", "op": "attn", "B": 1, "H": 8, "Hkv": 2, "Lq": 1, "Lk": 300, "mask": "cache", "cap": 0.0,
         "bias": False, "train": False},
        # a serving step: sixteen requests, their caches filled to different lengths
        {"name": "token_batch", "op": "attn", "B": 16, "H": 32, "Hkv": 8, "Lq": 1, "Lk": 16384, "mask": "cache",
         "cap": 50.0, "bias": False, "train": False},
        # a chunk of new tokens (a latent frame at 832x480) over the clip before it, biased by distance
        {"name": "chunk_frame", "op": "attn", "B": 1, "H": 12, "Hkv": 12, "Lq": 1560, "Lk": 32760, "mask": "causal",
         "cap": 0.0, "bias": True, "train": False},
        # five clips of different sizes packed into one sequence, its end padded
        {"name": "packed_clips", "op": "attn", "B": 1, "H": 12, "Hkv": 12, "Lq": 16380, "Lk": 16380, "mask": "docs",
         "docs": 5, "cap": 0.0, "bias": False, "train": False},
        # a prefix that sees itself and causal tokens behind it, shared K/V heads, capped scores
        {"name": "prefix_cap", "op": "attn", "B": 2, "H": 16, "Hkv": 4, "Lq": 4001, "Lk": 4001, "mask": "prefix",
         "cap": 30.0, "bias": False, "train": False},
        # post-training on packed clips
        {"name": "train_packed", "op": "attn", "B": 1, "H": 12, "Hkv": 12, "Lq": 8190, "Lk": 8190, "mask": "docs",
         "docs": 4, "cap": 0.0, "bias": False, "train": True},
        # training a causal tower of odd length with everything at once
        {"name": "train_causal", "op": "attn", "B": 2, "H": 16, "Hkv": 4, "Lq": 2049, "Lk": 2049, "mask": "causal",
         "cap": 50.0, "bias": True, "train": True},
        # a block of the 832x480 workload: layer norm, one modulation a sample
        {"name": "block_480p", "op": "norm", "B": 1, "L": 32760, "C": 1536, "stream": "bf16", "norm": "layer",
         "post": "none", "token": False, "train": False},
        # single tokens of sixteen requests, norms before and after the block
        {"name": "block_token", "op": "norm", "B": 16, "L": 1, "C": 5120, "stream": "bf16", "norm": "rms", "post": "rms",
         "token": False, "train": False},
        # the largest model of the package's workloads at 1280x720, its residual stream in 32 bits
        {"name": "block_720p", "op": "norm", "B": 1, "L": 75600, "C": 5120, "stream": "fp32", "norm": "layer",
         "post": "none", "token": False, "train": False},
        # its gradient in training: a norm on the branch, one modulation a sample
        {"name": "train_block", "op": "norm", "B": 2, "L": 16380, "C": 1536, "stream": "bf16", "norm": "rms",
         "post": "rms", "token": False, "train": True},
        # a modulation for every token, the stream in 32 bits
        {"name": "train_block_token", "op": "norm", "B": 1, "L": 7803, "C": 5120, "stream": "fp32", "norm": "layer",
         "post": "none", "token": True, "train": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


# (query heads, K/V heads) of one GPU
HEADS = ((2, 2), (5, 5), (8, 2), (8, 8), (12, 12), (12, 4), (16, 4), (20, 20), (20, 4), (32, 8))
# channels: heads x 128 of whole models and shards, and sizes that fill no power of two
CHANNELS = (256, 640, 768, 1024, 1536, 1544, 2048, 2560, 4096, 4104, 5120)


def draw(rng):
    # scores of the plain form, elements of the norm; and no more bytes or operations than a listed case
    most = {"attn": 12 * 16380 ** 2, "train": 12 * 8190 ** 2, "norm": 75600 * 5120}
    top = {n: max(work(c)[n] for c in listed()) for n in ("bytes", "flops")}
    while True:
        if rng.random() < 0.6:
            H, Hkv = rng.choice(HEADS)
            c = {"op": "attn", "B": rng.choice((1, 1, 2, 3)), "H": H, "Hkv": Hkv,
                 "mask": rng.choice(("cache", "causal", "docs", "cross", "prefix")),
                 "cap": rng.choice((0.0, 0.0, 30.0, 50.0)), "bias": rng.random() < 0.3, "train": False}
            if c["mask"] == "cache":
                c.update(B=rng.choice((1, 4, 16, 24)), Lq=rng.choice((1, 1, 1, 2, 4, 7)), Lk=_log_int(rng, 200, 20000))
            elif c["mask"] == "cross":
                c.update(Lq=_log_int(rng, 500, 20000), Lk=rng.randint(100, 1500), docs=rng.randint(1, 6), bias=False)
            else:
                c["Lk"] = _log_int(rng, 60, 16380)
                c["Lq"] = c["Lk"] if c["mask"] != "causal" or rng.random() < 0.5 else rng.randint(1, c["Lk"])
                if c["mask"] == "docs":
                    c["docs"] = rng.randint(1, 8)
            c["train"] = c["mask"] != "cache" and rng.random() < 0.45
            cost, limit = c["B"] * H * c["Lq"] * c["Lk"], most["train" if c["train"] else "attn"]
            if c["mask"] == "cache":
                cost, limit = c["B"] * Hkv * c["Lk"], 16 * 8 * 16384
        else:
            C = rng.choice(CHANNELS)
            c = {"op": "norm", "B": rng.choice((1, 1, 2, 5)), "L": _log_int(rng, 1, 75600), "C": C,
                 "stream": rng.choice(("bf16", "fp32")), "norm": rng.choice(("layer", "rms")),
                 "post": rng.choice(("none", "none", "rms", "layer")), "token": rng.random() < 0.3,
                 "train": rng.random() < 0.5}
            cost = c["B"] * c["L"] * C * (4 if c["token"] else 1) * (2 if c["train"] else 1)
            limit = most["norm"]
        if cost <= limit and all(work(c)[n] <= top[n] for n in top):
            return c


# ---------------------------------------------------------------- sizes ----


def _doc_lengths(total, n):
    """n lengths, none like its neighbour, that fill all but a 50th of total."""
    left = total - total // 50
    w = [3 + (5 * i) % 7 for i in range(n)]
    lens = [max(1, left * x // sum(w)) for x in w]
    return lens


def _docs(c):
    """Document lengths of queries and of keys."""
    q = _doc_lengths(c["Lq"], c["docs"])
    return q, q if c["mask"] == "docs" else _doc_lengths(c["Lk"], c["docs"])[::-1]


def _filled(c):
    """Tokens in the cache of every batch, the new ones included."""
    least = min(c["Lk"], max(c["Lq"], 1))
    return [max(least, c["Lk"] * (3 + (7 * b) % 10) // 12) for b in range(c["B"])]


def _prefixes(c):
    return [c["Lk"] * (5 + 3 * b) // 12 for b in range(c["B"])]


def _pairs(c):
    """Visible (query, key) pairs of a head, over the batch."""
    B, Lq, Lk = c["B"], c["Lq"], c["Lk"]
    tri = Lq * (Lq + 1) // 2
    if c["mask"] == "causal":
        return B * (Lq * (Lk - Lq) + tri)
    if c["mask"] == "cache":
        return sum(Lq * (n - Lq) + tri for n in _filled(c))
    if c["mask"] == "prefix":
        return sum(tri + p * (p - 1) // 2 for p in _prefixes(c))
    return B * sum(a * b for a, b in zip(*_docs(c)))


def work(c):
    if c["op"] == "attn":
        keys = sum(_filled(c)) if c["mask"] == "cache" else c["B"] * c["Lk"]
        q, kv = c["B"] * c["Lq"] * c["H"] * D * 2, keys * c["Hkv"] * D * 2
        lse = 4 * c["B"] * c["H"] * c["Lq"]
        pairs = c["H"] * _pairs(c)
        if c["train"]:  # q, k, v, dout in; o, lse, dq, dk, dv out
            return {"bytes": 4 * q + 4 * kv + lse, "flops": 14 * D * pairs}
        return {"bytes": 2 * q + 2 * kv, "flops": 4 * D * pairs}
    n, e = c["B"] * c["L"] * c["C"], 2 if c["stream"] == "bf16" else 4
    mods = 4 * c["C"] * c["B"] * (c["L"] if c["token"] else 1)
    if c["train"]:  # dh, dx', x', y, modulations in; dx, dy and the modulations' gradients out
        return {"bytes": n * (2 + 2 * e + 2 + e + 2) + 5 * mods, "flops": 30 * n}
    return {"bytes": n * (2 * e + 4) + 3 * mods, "flops": 15 * n}


# --------------------------------------------------------------- inputs ----


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, mul=1.0, dtype=torch.bfloat16):
    return (torch.randn(shape, generator=g, device="cuda") * mul).to(dtype)


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _ids(lens, total, B):
    row = torch.full((total,), -1, dtype=torch.int32)
    at = 0
    for i, n in enumerate(lens):
        row[at:at + n] = i
        at += n
    return row.cuda().repeat(B, 1).contiguous()


def prepare(c, seed):
    g = _gen(seed)
    s = {"case": c}
    if c["op"] == "attn":
        # queries of trained models are larger than their keys where a cap is of use
        s["q"] = _normal(g, (c["B"], c["Lq"], c["H"], D), 3.0 if c["cap"] else 1.0)
        s["k"] = _normal(g, (c["B"], c["Lk"], c["Hkv"], D))
        s["v"] = _normal(g, (c["B"], c["Lk"], c["Hkv"], D))
        if c["train"]:
            s["dout"] = _normal(g, (c["B"], c["Lq"], c["H"], D))
        s["slopes"] = s["q_doc"] = s["k_doc"] = s["valid"] = s["prefix"] = s["start"] = None
        if c["bias"]:
            s["slopes"] = torch.exp2(-8.0 * torch.arange(1, c["H"] + 1, device="cuda") / c["H"]).float()
        if c["mask"] == "cache":
            s["valid"] = _ints(_filled(c))
            s["start"] = _ints([n - c["Lq"] for n in _filled(c)])
        if c["mask"] == "prefix":
            s["prefix"] = _ints(_prefixes(c))
        if c["mask"] in ("docs", "cross"):
            ql, kl = _docs(c)
            s["q_doc"], s["k_doc"] = _ids(ql, c["Lq"], c["B"]), _ids(kl, c["Lk"], c["B"])
        return s
    stream = torch.bfloat16 if c["stream"] == "bf16" else torch.float32
    B, L, C = c["B"], c["L"], c["C"]
    s["x"] = _normal(g, (B, L, C), 2.0, stream)
    s["y"] = _normal(g, (B, L, C), 0.5)
    mods = _normal(g, (B, L if c["token"] else 1, 3, C), 0.3, torch.float32)
    s["gate"], s["scale"], s["shift"] = mods.unbind(2)  # rows of one modulation table, as a block cuts them
    s["gain"] = 1 + _normal(g, (C,), 0.1, torch.float32) if c["norm"] == "rms" else None
    s["post_gain"] = 1 + _normal(g, (C,), 0.1, torch.float32) if c["post"] != "none" else None
    if c["train"]:
        s["dh"] = _normal(g, (B, L, C))
        s["dx"] = _normal(g, (B, L, C), 1.0, stream)
    return s


def _softmax_scale():
    return float(torch.tensor(1.0 / D ** 0.5, dtype=torch.float32))


# ---------------------------------------------------------- plain forms ----


def _visible(s, c):
    """[B, 1, 1, Lq, Lk]: which key every query sees."""
    dev = s["q"].device
    Lq, Lk = c["Lq"], c["Lk"]
    j = torch.arange(Lk, device=dev)
    start = s["start"][:, None].long() if s["start"] is not None else torch.full((c["B"], 1), Lk - Lq, device=dev)
    pos = start + torch.arange(Lq, device=dev)
    see = torch.ones((c["B"], Lq, Lk), dtype=torch.bool, device=dev)
    if c["mask"] in ("causal", "cache", "prefix"):
        see = j <= pos[:, :, None]
        if s["prefix"] is not None:
            see = see | (j < s["prefix"][:, None, None])
    if s["valid"] is not None:
        see = see & (j < s["valid"][:, None, None])
    if s["q_doc"] is not None:
        see = see & (s["q_doc"][:, :, None] == s["k_doc"][:, None, :]) & (s["q_doc"][:, :, None] >= 0)
    return see[:, None, None], pos


def _plain_attn(s):
    c = s["case"]
    B, H, Hkv, Lq, Lk = c["B"], c["H"], c["Hkv"], c["Lq"], c["Lk"]
    rep = H // Hkv
    # [B, Hkv, rep, Lq, D] and [B, Hkv, 1, Lk, D]
    q = s["q"].float().reshape(B, Lq, Hkv, rep, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, rep * Lq, D)
    k = s["k"].float().permute(0, 2, 1, 3).contiguous()
    v = s["v"].float().permute(0, 2, 1, 3).contiguous()
    scale = _softmax_scale()
    see, pos = _visible(s, c)
    x = (q @ k.transpose(2, 3).contiguous()).mul_(scale).reshape(B, Hkv, rep, Lq, Lk)
    t = None
    if c["cap"]:
        t = torch.tanh(x / c["cap"])
        x = t * c["cap"]
    if c["bias"]:
        dist = (pos[:, :, None] - torch.arange(Lk, device=x.device)).abs().float()
        x = x - s["slopes"].reshape(1, Hkv, rep, 1, 1) * dist[:, None, None]
    x = x.masked_fill_(~see, -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    p = x.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    lse = (m + l.log())[..., 0]
    p = p.div_(torch.where(l > 0, l, torch.ones_like(l)))
    p2 = p.reshape(B, Hkv, rep * Lq, Lk)
    o = p2 @ v

    def rows(y):
        return y.reshape(B, Hkv, rep, Lq, D).permute(0, 3, 1, 2, 4).reshape(B, Lq, H, D).to(s["q"].dtype)

    if not c["train"]:
        return rows(o)
    do = s["dout"].float().reshape(B, Lq, Hkv, rep, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, rep * Lq, D)
    dv = p2.transpose(2, 3) @ do
    ds = (do @ v.transpose(2, 3).contiguous()).sub_((do * o).sum(-1, keepdim=True)).mul_(p2)
    if t is not None:
        ds = ds.mul_((1 - t * t).reshape(B, Hkv, rep * Lq, Lk))
    dq = (ds @ k).mul_(scale)
    dk = (ds.transpose(2, 3) @ q).mul_(scale)
    return {"o": rows(o), "lse": lse.reshape(B, H, Lq), "dq": rows(dq),
            "dk": dk.permute(0, 2, 1, 3).to(s["k"].dtype).contiguous(),
            "dv": dv.permute(0, 2, 1, 3).to(s["v"].dtype).contiguous()}


def _hat(x, kind):
    """x normalised over its channels, and what it was multiplied by."""
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    return x * r, r


def _hat_bwd(g, xh, r, kind):
    out = g - xh * (g * xh).mean(-1, keepdim=True)
    if kind == "layer":
        out = out - g.mean(-1, keepdim=True)
    return out * r


def _plain_norm(s):
    c = s["case"]
    gate, mul, shift = s["gate"], 1 + s["scale"], s["shift"]
    gain = 1.0 if s["gain"] is None else s["gain"]
    pg = 1.0 if s["post_gain"] is None else s["post_gain"]
    y = s["y"].float()
    yh, ry = (y, None) if c["post"] == "none" else _hat(y, c["post"])
    if not c["train"]:
        x = s["x"].float() + gate * (yh * pg)
        xh, _ = _hat(x, c["norm"])
        return {"x": x.to(s["x"].dtype), "h": (xh * gain * mul + shift).to(torch.bfloat16)}
    dh = s["dh"].float()
    xh, rx = _hat(s["x"].float(), c["norm"])
    g = s["dx"].float() + _hat_bwd(dh * (gain * mul), xh, rx, c["norm"])
    du = g * gate
    out = {"dx": g.to(s["x"].dtype)}
    dxh = dh * xh
    if c["post"] == "none":
        out["dy"] = du.to(torch.bfloat16)
    else:
        out["dy"] = _hat_bwd(du * pg, yh, ry, c["post"]).to(torch.bfloat16)
        out["dpost_gain"] = (du * yh).sum((0, 1), dtype=torch.float64).float()
    if s["gain"] is not None:
        out["dgain"] = (dxh * mul).sum((0, 1), dtype=torch.float64).float()
    mods = {"dgate": g * (yh * pg), "dscale": dxh * gain, "dshift": dh}
    if not c["token"]:
        mods = {n: x.sum(1, keepdim=True, dtype=torch.float64).float() for n, x in mods.items()}
    out.update(mods)
    return out


# ------------------------------------------------------------------ run ----


def run(s):
    c = s["case"]
    if not own:
        return _plain_attn(s) if c["op"] == "attn" else _plain_norm(s)
    import paper_2609_18077_amd as vx

    if c["op"] == "attn":
        score = vx.Score(causal=c["mask"] in ("causal", "cache", "prefix"), cap=c["cap"], slopes=s["slopes"],
                         q_doc=s["q_doc"], k_doc=s["k_doc"], kv_valid_len=s["valid"], prefix_len=s["prefix"],
                         q_start=s["start"])
        if not c["train"]:
            return vx.attn_mod_fwd(s["q"], s["k"], s["v"], score)
        o, lse = vx.attn_mod_fwd(s["q"], s["k"], s["v"], score, return_lse=True)
        dq, dk, dv = vx.attn_mod_bwd(s["q"], s["k"], s["v"], o, s["dout"], lse, score)
        return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}
    post = None if c["post"] == "none" else c["post"]
    if not c["train"]:
        x, h = vx.block_norm_fwd(s["x"], s["y"], gate=s["gate"], scale=s["scale"], shift=s["shift"], gain=s["gain"],
                                 post_gain=s["post_gain"], norm=c["norm"], post=post, eps=EPS)
        return {"x": x, "h": h}
    got = vx.block_norm_bwd(s["dh"], s["dx"], s["x"], s["y"], gate=s["gate"], scale=s["scale"], shift=s["shift"],
                            gain=s["gain"], post_gain=s["post_gain"], norm=c["norm"], post=post, eps=EPS)
    names = ["dx", "dy"] + (["dpost_gain"] if post else []) + (["dgain"] if s["gain"] is not None else [])
    return {n: got[n] for n in names + ["dgate", "dscale", "dshift"]}


# ---------------------------------------------------------------- exact ----


def _exact_head(s, c, b, h, rows):
    """o, lse of some query rows of a head in 64 bits, with what the gradient needs."""
    hk = h // (c["H"] // c["Hkv"])
    dev = s["q"].device
    q, k, v = (s[n][b, :, i].double().contiguous() for n, i in (("q", h), ("k", hk), ("v", hk)))
    q = q[rows]
    raw = q @ k.t().contiguous() * _softmax_scale()
    th = torch.tanh(raw / c["cap"]) if c["cap"] else None
    x = raw if th is None else th * c["cap"]
    first = int(s["start"][b]) if s["start"] is not None else c["Lk"] - c["Lq"]
    pos = (rows + first)[:, None]
    key = torch.arange(c["Lk"], device=dev)[None]
    if c["bias"]:
        x = x - float(s["slopes"][h]) * (pos - key).abs().double()
    hide = torch.zeros_like(x, dtype=torch.bool)
    if c["mask"] in ("causal", "cache", "prefix"):
        hide |= key > pos
    if c["mask"] == "prefix":
        hide &= key >= int(s["prefix"][b])
    if c["mask"] == "cache":
        hide |= key >= int(s["valid"][b])
    if c["mask"] in ("docs", "cross"):
        qd, kd = s["q_doc"][b][rows][:, None], s["k_doc"][b][None]
        hide |= (qd != kd) | (qd < 0)
    x = x.masked_fill(hide, -math.inf)
    lse = torch.logsumexp(x, 1)
    p = torch.exp(x - torch.where(lse.isinf(), torch.zeros_like(lse), lse)[:, None])
    return q, k, v, p, th, lse


def exact(c, seed):
    s = prepare(c, seed)
    if c["op"] == "norm":
        return _exact_norm(s, c)
    B, H, Lq = c["B"], c["H"], c["Lq"]
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros((B, H, Lq), dtype=torch.float64, device="cuda")
    grads = {n: torch.zeros(s[n[1:]].shape, dtype=torch.float64, device="cuda") for n in ("dq", "dk", "dv")}
    step = max(1, min(Lq, (1 << 27) // c["Lk"]))
    scale, rep = _softmax_scale(), H // c["Hkv"]
    for b in range(B):
        for h in range(H):
            for i in range(0, Lq, step):
                rows = torch.arange(i, min(i + step, Lq), device="cuda")
                q, k, v, p, th, z = _exact_head(s, c, b, h, rows)
                oh = p @ v
                o[b, rows, h], lse[b, h, rows] = oh, z
                if not c["train"]:
                    continue
                do = s["dout"][b, rows, h].double()
                ds = p * (do @ v.t().contiguous() - (do * oh).sum(1, keepdim=True))
                if th is not None:
                    ds = ds * (1 - th.square())
                grads["dq"][b, rows, h] = ds @ k * scale
                grads["dk"][b, :, h // rep] += ds.t() @ q * scale
                grads["dv"][b, :, h // rep] += p.t() @ do
    return {"o": o, "lse": lse, **grads} if c["train"] else o


def _exact_stats(x, kind):
    mean = x.sum(-1, keepdim=True) / x.shape[-1] if kind == "layer" else torch.zeros_like(x[..., :1])
    var = ((x - mean) ** 2).sum(-1, keepdim=True) / x.shape[-1]
    return mean, 1.0 / torch.sqrt(var + EPS)


def _exact_norm(s, c):
    """A chunk of tokens at a time, so that the 64-bit copies stay small."""
    B, L, C = c["B"], c["L"], c["C"]
    one = torch.ones(C, dtype=torch.float64, device="cuda")
    gain = one if s["gain"] is None else s["gain"].double()
    pg = one if s["post_gain"] is None else s["post_gain"].double()
    names = ("x", "h") if not c["train"] else ("dx", "dy", "dpost_gain", "dgain", "dgate", "dscale", "dshift")
    parts = {n: [] for n in names}
    sums = {}
    step = max(1, (1 << 26) // (B * C))
    for i in range(0, L, step):
        cut = slice(i, min(i + step, L))
        x, y = s["x"][:, cut].double(), s["y"][:, cut].double()
        gate, scale, shift = (s[n][:, cut if c["token"] else slice(0, 1)].double() for n in ("gate", "scale", "shift"))
        u, yh, ry = y, y, None
        if c["post"] != "none":
            my, ry = _exact_stats(y, c["post"])
            yh = (y - my) * ry
            u = yh * pg
        if not c["train"]:
            z = x + gate * u
            mz, rz = _exact_stats(z, c["norm"])
            parts["x"].append(z)
            parts["h"].append((z - mz) * rz * gain * (1 + scale) + shift)
            continue
        dh = s["dh"][:, cut].double()
        mx, rx = _exact_stats(x, c["norm"])
        xh = (x - mx) * rx
        w = dh * gain * (1 + scale)
        back = w - xh * ((w * xh).sum(-1, keepdim=True) / C)
        if c["norm"] == "layer":
            back = back - w.sum(-1, keepdim=True) / C
        g = s["dx"][:, cut].double() + rx * back
        du = g * gate
        dy = du
        if c["post"] != "none":
            a = du * pg
            dy = a - yh * ((a * yh).sum(-1, keepdim=True) / C)
            if c["post"] == "layer":
                dy = dy - a.sum(-1, keepdim=True) / C
            dy = dy * ry
        parts["dx"].append(g)
        parts["dy"].append(dy)
        every = {"dpost_gain": (du * yh).sum((0, 1)), "dgain": (dh * xh * (1 + scale)).sum((0, 1))}
        mods = {"dgate": g * u, "dscale": dh * xh * gain, "dshift": dh}
        if c["token"]:
            for n, z in mods.items():
                parts[n].append(z)
        else:
            every.update({n: z.sum(1, keepdim=True) for n, z in mods.items()})
        for n, z in every.items():
            sums[n] = sums.get(n, 0) + z
    out = {n: torch.cat(z, 1) for n, z in parts.items() if z}
    out.update(sums)
    if s["gain"] is None:
        out.pop("dgain", None)
    if c["post"] == "none":
        out.pop("dpost_gain", None)
    return out
