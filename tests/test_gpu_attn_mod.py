"""Attention with score modifiers (vidax_attn_mod_fwd) against the float64
reference.

Tolerances, per element.  A weight p is rounded to bf16 once, to p (1 + e) with
|e| <= 2^-8, and the output is divided by the sum of the rounded weights: with
sum_j p_j = 1 it is off by sum_j p_j e_j (v_j - o) / (1 + sum_j p_j e_j), at most
2^-8 / (1 - 2^-8) (sum_j p_j |v_j| + |o|).  Its scores are off by at most delta,
which adds 2 delta sum_j p_j |v_j|, and its own rounding 2^-8 of all that.
delta: the fp32 dot product of 128 terms, 128 * 2^-24 of scale * sum |q k|, and
eight roundings (2^-24 each, 2^-22 for the hardware exponential and reciprocal)
of the magnitudes that y passes through: the cap, the bias, the reference.  The
log-sum-exp is off by delta, the fp32 sum of Lk weights and two logarithms'
roundings.  Beside the bound of every element, the relative RMS error of a call
is held to 2^-7.5: two independent roundings of at most 2^-8 each.
"""

import math

import numpy as np
import pytest

import oracle
import paper_2609_18077_amd as vx
from tests.gpu_util import log

pytestmark = pytest.mark.gpu

D = 128
SCALE = float(np.float32(1 / math.sqrt(D)))
HALF = 2.0 ** -8
RMS = 2.0 ** -7.5


def make(B, H, Hkv, Lq, Lk, seed, mul=1.0):
    import torch

    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")
    return ((rnd(B, Lq, H, D) * mul).to(torch.bfloat16), rnd(B, Lk, Hkv, D).to(torch.bfloat16),
            rnd(B, Lk, Hkv, D).to(torch.bfloat16))


def f64(t):
    return t.detach().double().cpu().numpy()


def dev_score(**s):
    """A Score of device tensors and the reference's spec from plain lists."""
    import torch

    kw = {}
    for n, x in s.items():
        if n in ("causal", "cap") or x is None:
            kw[n] = x
        elif n == "slopes":
            kw[n] = torch.tensor(x, dtype=torch.float32, device="cuda")
        else:
            kw[n] = torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")
    spec = dict(s)
    if s.get("slopes") is not None:
        spec["slopes"] = np.asarray(s["slopes"], np.float32).astype(np.float64)
    return vx.Score(**kw), oracle.ScoreSpec(**spec)


def deltas(q, k, scale, spec):
    """delta of every row [B, Lq, H] (a bound on the error of its scores)."""
    B, Lq, H, _ = q.shape
    rep = H // k.shape[2]
    out = np.zeros((B, Lq, H))
    for b in range(B):
        for h in range(H):
            terms = abs(scale) * (np.abs(q[b, :, h]) @ np.abs(k[b, :, h // rep]).T) if k.shape[1] else np.zeros((Lq, 1))
            x, _ = oracle.attn_mod.scores(q[b, :, h], k[b, :, h // rep], b, h, scale, spec)
            seen = np.isfinite(x)
            top = np.where(seen, terms, 0).max(1, initial=0)
            mag = np.where(seen, np.abs(np.where(seen, x, 0)), 0).max(1, initial=0)
            bias = 0.0
            if spec.slopes is not None:
                d = np.abs(oracle.attn_mod.positions(b, Lq, k.shape[1], spec)[:, None] - np.arange(k.shape[1]))
                bias = (abs(spec.slopes[h]) * np.where(seen, d, 0)).max(1, initial=0)
            out[b, :, h] = 128 * 2.0 ** -24 * top + 8 * 2.0 ** -22 * (1 + mag + bias + spec.cap)
    return out


def check(q, k, v, scale=None, what="", workspace=None, **s):
    import torch

    score, spec = dev_score(**s)
    o, lse = vx.attn_mod_fwd(q, k, v, score, scale=scale, return_lse=True, workspace=workspace)
    alone = vx.attn_mod_fwd(q, k, v, score, scale=scale, workspace=workspace)
    torch.cuda.synchronize()
    # without the log-sum-exps: the same but for the weights of parts that are joined, good to a rounding of the sums
    assert (alone.double() - o.double()).norm() <= 2.0 ** -9 * o.double().norm(), what
    return compare(o, lse, q, k, v, SCALE if scale is None else float(np.float32(scale)), spec, what)


def compare(o, lse, q, k, v, sc, spec, what):
    """An output and log-sum-exps against the reference; (o, lse)."""
    qn, kn, vn = f64(q), f64(k), f64(v)
    ro, rl = oracle.attn_mod_ref(qn, kn, vn, sc, spec)
    mag, _ = oracle.attn_mod_ref(qn, kn, np.abs(vn), sc, spec)
    delta = deltas(qn, kn, sc, spec)
    got, gl = f64(o), f64(lse)
    assert np.isfinite(got).all(), what
    off = HALF / (1 - HALF) * (mag + np.abs(ro)) + 2 * delta[..., None] * mag
    tol = off + HALF * (np.abs(ro) + off)
    err = np.abs(got - ro)
    empty = np.isneginf(rl)
    assert np.array_equal(np.isneginf(gl), empty), what
    assert not got[np.moveaxis(empty, 1, 2)].any(), what
    full = ~empty
    lerr = np.abs(gl[full] - rl[full])
    ltol = (np.moveaxis(delta, 2, 1)[full] + k.shape[1] * 2.0 ** -24 + 2.0 ** -22 * (2 + np.abs(rl[full])))
    norm = np.sqrt((ro ** 2).sum())
    rms = np.sqrt((err ** 2).sum()) / norm if norm else 0.0
    worst = float((err / np.maximum(tol, 1e-300)).max(initial=0)) if err.size else 0.0
    log(f"  {what}: worst/bound {worst:.3f}, rel rms {rms:.2e}, lse {float((lerr / ltol).max(initial=0)):.3f} of its bound")
    assert worst <= 1, (what, worst)
    assert rms <= RMS, (what, rms)
    assert (lerr <= ltol).all(), (what, float(lerr.max()))
    return o, lse


def masks(name, B, Lq, Lk, seed=0):
    """Masks by name, from the sizes and a seed."""
    rng = np.random.default_rng([seed, Lq, Lk])
    sorted_ids = lambda L, n: np.sort(rng.integers(0, n, size=(B, L)), 1)
    if name == "all":
        return {}
    if name == "valid":
        return {"kv_valid_len": [[Lk // 2 + 1, 0, Lk + 7, -3][b % 4] for b in range(B)]}
    if name == "causal":
        return {"causal": True}
    if name == "causal_early":  # positions before the keys: the first rows see nothing
        return {"causal": True, "q_start": [-2 - b for b in range(B)]}
    if name == "causal_cache":
        n = [max(Lq, Lk * (2 + b) // (B + 2)) for b in range(B)]
        return {"causal": True, "kv_valid_len": n, "q_start": [x - Lq for x in n]}
    if name == "prefix":
        return {"causal": True, "prefix_len": [Lk // 3 + 5 * b for b in range(B)], "q_start": [0] * B}
    if name == "docs":
        return {"q_doc": sorted_ids(Lq, 4), "k_doc": sorted_ids(Lk, 4)}
    if name == "docs_causal":
        ids = sorted_ids(max(Lq, Lk), 3)
        return {"causal": True, "q_doc": ids[:, -Lq:], "k_doc": ids[:, -Lk:]}
    if name == "docs_any_order":  # also negative ids and ids that the other side lacks
        return {"q_doc": rng.integers(-1, 6, size=(B, Lq)) * 7, "k_doc": rng.integers(-2, 5, size=(B, Lk)) * 7}
    if name == "docs_valid_prefix":
        ids = sorted_ids(max(Lq, Lk), 3)
        ids[:, -max(Lq, Lk) // 9:] = -1
        return {"causal": True, "prefix_len": [Lk // 2] * B, "kv_valid_len": [Lk - 3] * B, "q_doc": ids[:, :Lq],
                "k_doc": ids[:, :Lk]}
    if name == "docs_extreme":  # the largest id there is, and documents that never meet
        return {"q_doc": np.where(np.arange(Lq) % 2, 2 ** 31 - 1, 5)[None].repeat(B, 0),
                "k_doc": np.where(np.arange(Lk) % 3, 2 ** 31 - 1, 6)[None].repeat(B, 0)}
    raise ValueError(name)


MASKS = ("all", "valid", "causal", "causal_early", "causal_cache", "prefix", "docs", "docs_causal", "docs_any_order",
         "docs_valid_prefix", "docs_extreme")


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("cap,bias", [(0.0, False), (20.0, False), (0.0, True), (3.0, True)])
def test_masks_and_modifiers(mask, cap, bias):
    """Several tiles of rows and keys, ragged in both, shared K/V heads."""
    B, H, Hkv, Lq, Lk = 2, 4, 2, 300, 419
    q, k, v = make(B, H, Hkv, Lq, Lk, 11, mul=4.0 if cap else 1.0)
    slopes = [0.5, 0.0, -0.01, 0.02] if bias else None
    check(q, k, v, cap=cap, slopes=slopes, what=f"{mask} cap={cap} bias={bias}", **masks(mask, B, Lq, Lk))


# one token to several tiles, on both sides of every edge of a tile
SIZES = [(1, 1), (1, 2), (2, 1), (5, 3), (33, 32), (64, 64), (65, 63), (256, 64), (257, 65), (255, 128), (129, 129),
         (300, 193), (513, 700), (40, 1300)]


@pytest.mark.parametrize("Lq,Lk", SIZES)
@pytest.mark.parametrize("mask", ["all", "causal", "docs_valid_prefix"])
def test_sizes(Lq, Lk, mask):
    q, k, v = make(1, 3, 3, Lq, Lk, Lq + Lk)
    check(q, k, v, what=f"{Lq}x{Lk} {mask}", **masks(mask, 1, Lq, Lk))


@pytest.mark.parametrize("H,Hkv", [(1, 1), (5, 5), (6, 3), (8, 1), (20, 4), (33, 1)])
def test_heads(H, Hkv):
    q, k, v = make(2, H, Hkv, 70, 150, H)
    check(q, k, v, causal=True, what=f"{H}/{Hkv}")


@pytest.mark.parametrize("scale", [0.0, -0.05, 0.7])
@pytest.mark.parametrize("cap", [0.0, 2.0])
def test_scales(scale, cap):
    q, k, v = make(1, 2, 2, 130, 200, 21)
    check(q, k, v, scale=scale, cap=cap, causal=True, slopes=[0.1, 0.2], what=f"scale {scale} cap {cap}")


@pytest.mark.parametrize("cap", [1e-3, 0.5, 1000.0, 1e20, 3e38])
def test_caps_from_flat_to_none(cap):
    q, k, v = make(1, 2, 2, 70, 100, 22, mul=3.0)
    s = {"causal": True}
    if cap > 1e6:  # tanh is the identity: the bound counts the uncapped score's magnitudes
        import torch

        got = vx.attn_mod_fwd(q, k, v, vx.Score(causal=True, cap=cap))
        ref = vx.attn_mod_fwd(q, k, v, vx.Score(causal=True))
        torch.cuda.synchronize()
        d = (got.float() - ref.float()).abs().max().item()
        assert d <= 2 * HALF * ref.float().abs().max().item()
    else:
        check(q, k, v, cap=cap, what=f"cap {cap}", **s)


def test_growing_scores_reset_the_reference():
    """Keys sorted by score, far apart: every block beats the reference of the ones before."""
    import torch

    q, k, v = make(1, 2, 2, 64, 640, 23)
    ramp = torch.linspace(-30, 30, 640, device="cuda")
    k = (q[:, :1].float().sign().mean(1, keepdim=True) * ramp[None, :, None, None] + 0 * k.float()).to(torch.bfloat16)
    for s in ({}, {"cap": 40.0}, {"slopes": [-1.5, 3.0]}, {"causal": True}):
        check(q, k, v, what=f"ramp {list(s)}", **s)


def test_one_seen_key_gives_its_value_row():
    """Weight 1 exactly: the output is v, bit for bit."""
    import torch

    L = 333
    q, k, v = make(1, 2, 2, L, L, 24)
    ids = torch.arange(L, dtype=torch.int32, device="cuda")[None]
    perm = torch.randperm(L, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    o = vx.attn_mod_fwd(q, k, v, vx.Score(q_doc=ids, k_doc=ids[:, perm].contiguous()))
    want = torch.empty_like(v)
    want[:, perm] = v
    assert torch.equal(o, want)


@pytest.mark.parametrize("Lq", [1, 70, 300])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_no_query_sees_does_not_matter(bad, Lq):
    """NaN and infinities past the valid length, behind the last query and at
    keys of negative documents."""
    import torch

    B, H, Lk = 2, 2, 500
    q, k, v = make(B, H, H, Lq, Lk, 25)
    for s, hidden in [({"kv_valid_len": [201, 64]}, [(0, 201, 500), (1, 64, 500)]),
                      ({"causal": True, "q_start": [130, 0]}, [(0, 130 + Lq, 500), (1, Lq, 500)]),
                      ({"q_doc": np.zeros((B, Lq), int), "k_doc": np.where(np.arange(Lk) % 100 < 37, -1, 0)[None].repeat(B, 0)},
                       [(b, i, i + 37) for b in range(B) for i in range(0, Lk, 100)])]:
        score, _ = dev_score(**s)
        want = vx.attn_mod_fwd(q, k, v, score)
        k2, v2 = k.clone(), v.clone()
        for b, i, j in hidden:
            k2[b, i:j] = bad
            v2[b, i:j] = -bad
        assert torch.equal(vx.attn_mod_fwd(q, k2, v2, score), want), list(s)
        assert torch.isfinite(want.float()).all()


def test_empty_calls():
    import torch

    z = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")
    for shape in ((0, 3, 2), (2, 0, 2), (2, 3, 0)):
        q = z(*shape, D)
        k = z(shape[0], 5, shape[2], D)
        assert vx.attn_mod_fwd(q, k, k).shape == q.shape
    q, k, _ = make(2, 2, 2, 5, 4, 26)
    ids = torch.zeros((2, 5), dtype=torch.int32, device="cuda")
    for score in (None, vx.Score(causal=True), vx.Score(q_doc=ids, k_doc=ids[:, :0].contiguous())):
        o, lse = vx.attn_mod_fwd(q, k[:, :0].contiguous(), k[:, :0].contiguous(), score, return_lse=True)
        assert not o.any() and bool((lse == -math.inf).all())


@pytest.mark.parametrize("Lq,Lk", [(1, 700), (40, 1300), (300, 2000)])
def test_runs_of_keys_are_joined(Lq, Lk):
    """The split the sizes ask for against the smallest workspace."""
    import torch

    q, k, v = make(1, 2, 1, Lq, Lk, 27)
    s = masks("docs_valid_prefix", 1, Lq, Lk)
    need = vx.lib().vidax_attn_mod_fwd_workspace_floats(1, 2, 1, Lq, Lk, D, 1)
    least = 4 * (-(-Lk // 64) + -(-Lq // 64)) + -(-Lk // 256) + -(-Lq // 256)
    assert need > least
    o, lse = check(q, k, v, what="runs", **s)
    o1, lse1 = check(q, k, v, what="one run", workspace=torch.empty(least, device="cuda"), **s)
    # each within its bound of the exact value; rows that see nothing agree exactly
    assert torch.equal(lse == -math.inf, lse1 == -math.inf)
    with pytest.raises(vx.VidaxError):
        check(q, k, v, workspace=torch.empty(least - 1, device="cuda"), **s)


# Sizes whose query tiles are cut into pieces of equal weight on 256 compute units
PIECES = [(3, 16, 4, 296, 3993, "all"), (3, 16, 4, 532, 2375, "valid"), (2, 8, 2, 2814, 2526, "causal"),
          (1, 8, 2, 4001, 4001, "prefix"), (3, 4, 1, 2934, 5374, "lengths"),
          (20, 5, 1, 7, 3100, "lengths"), (2, 3, 1, 4500, 3000, "lengths"), (1, 8, 2, 4001, 4001, "capped")]


def piece_score(B, H, Lq, Lk, mask):
    """What changes the scores, and the slopes as float64 (or None)."""
    s = {}
    if mask in ("lengths", "prefix"):
        s = dict(cap=20.0, slopes=list(0.01 * np.arange(H)))
    if mask == "capped":
        s = dict(cap=20.0)
    if mask not in ("all", "valid"):
        s["causal"] = True
    if mask == "valid":
        s["kv_valid_len"] = [0, Lk, 700][:B]
    if mask == "prefix":
        s["prefix_len"] = [1500]
    if mask == "lengths":
        s |= {n: [x[b % 3] for b in range(B)] for n, x in (("q_start", (-1000, 300, Lk - Lq)), ("kv_valid_len", (1900, 3000, Lk)),
                                                           ("prefix_len", (0, 900, 70)))}
    return s, np.asarray(s["slopes"], np.float32).astype(np.float64) if "slopes" in s else None


@pytest.mark.parametrize("B,H,Hkv,Lq,Lk,mask", PIECES)
def test_pieces_of_tiles_are_joined(B, H, Hkv, Lq, Lk, mask):
    """Checked on two heads of every batch (2814 on 2526: rows and a tile that see nothing)."""
    import torch

    q, k, v = make(B, H, Hkv, Lq, Lk, Lq + Lk)
    s, slopes = piece_score(B, H, Lq, Lk, mask)
    score, _ = dev_score(**s)
    o, lse = vx.attn_mod_fwd(q, k, v, score, return_lse=True)
    again = vx.attn_mod_fwd(q, k, v, score, return_lse=True, workspace=torch.full((1 << 25,), float("nan"), device="cuda"))
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])
    for h in (0, H - 1):
        hs, ks = slice(h, h + 1), slice(h * Hkv // H, h * Hkv // H + 1)
        one = oracle.ScoreSpec(**{**s, "slopes": slopes[hs] if slopes is not None else None})
        compare(o[:, :, hs], lse[:, hs], q[:, :, hs], k[:, :, ks], v[:, :, ks], SCALE, one, f"pieces {Lq}x{Lk} {mask} head {h}")


def test_on_a_stream_beside_the_current_one():
    """Outputs and workspace belong to the stream given: nothing that the current stream still runs or takes next is
    touched, nor the other way round."""
    import torch

    q, k, v = make(1, 8, 2, 4001, 4001, 6)
    score, _ = dev_score(causal=True)
    ref, lse = vx.attn_mod_fwd(q, k, v, score, return_lse=True)
    grads = vx.attn_mod_bwd(q, k, v, ref, q, lse, score)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for n in range(4):
        got = vx.attn_mod_fwd(q, k, v, score, return_lse=True, stream=side)
        dgot = vx.attn_mod_bwd(q, k, v, *got[:1], q, got[1], score, stream=side)
        for size in (1 << 24, 1 << 25):  # the sizes of what the calls have just let go
            torch.empty(size, device="cuda").fill_(float("nan"))
        side.synchronize()
        assert torch.equal(got[0], ref) and torch.equal(got[1], lse), n
        assert all(torch.equal(a, b) for a, b in zip(dgot, grads)), n
    torch.cuda.synchronize()


def test_pieces_in_a_graph():
    import torch

    q, k, v = make(1, 8, 2, 4001, 4001, 5)
    score, _ = dev_score(causal=True)
    ws = torch.empty(1 << 25, device="cuda")
    out = torch.empty_like(q)
    vx.attn_mod_fwd(q, k, v, score, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        vx.attn_mod_fwd(q, k, v, score, out=out, workspace=ws)
    for n in range(3):
        q.copy_(make(1, 8, 2, 4001, 4001, n)[0])
        ws.fill_(float("nan"))
        graph.replay()
        assert torch.equal(out, vx.attn_mod_fwd(q, k, v, score)), n


def test_rows_and_keys_beside_the_call_stay():
    import torch

    B, H, Lq, Lk = 1, 3, 77, 130
    q, k, v = make(B, H, H, Lq, Lk, 28)
    big = torch.full((Lq + 2, H, D), 7.0, dtype=torch.bfloat16, device="cuda")
    out = big[1:Lq + 1].reshape(B, Lq, H, D)
    o = vx.attn_mod_fwd(q, k, v, vx.Score(causal=True), out=out)
    torch.cuda.synchronize()
    assert o.data_ptr() == out.data_ptr() and bool((big[0] == 7).all()) and bool((big[-1] == 7).all())
    assert torch.equal(out, vx.attn_mod_fwd(q, k, v, vx.Score(causal=True)))


def test_same_bits_twice_on_another_stream_and_in_a_graph():
    import torch

    q, k, v = make(2, 4, 2, 300, 900, 29)
    score, _ = dev_score(cap=10.0, **masks("docs_valid_prefix", 2, 300, 900))
    qs, ks, vs = make(2, 4, 2, 3, 900, 30)
    work = lambda: [*vx.attn_mod_fwd(q, k, v, score, return_lse=True),
                    *vx.attn_mod_fwd(qs, ks, vs, vx.Score(causal=True), return_lse=True)]
    want = [t.clone() for t in work()]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = work()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = work()
    for i in range(3):
        for t in held:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want)), i
        assert all(torch.equal(a, b) for a, b in zip(work(), want)), i


@pytest.mark.parametrize("Lq", [1, 40])
def test_offsets_past_32_bits(Lq):
    """A cache of more than 2^31 values a batch: the keys seen are its last ones."""
    import torch

    Hkv, Lk = 8, (1 << 31) // (8 * D) + 1000
    g = torch.Generator(device="cuda").manual_seed(31)
    q = torch.randn((1, Lq, 8, D), generator=g, device="cuda").to(torch.bfloat16)
    k = torch.full((1, Lk, Hkv, D), 1.0, dtype=torch.bfloat16, device="cuda")
    v = torch.full((1, Lk, Hkv, D), 2.0, dtype=torch.bfloat16, device="cuda")
    n = 900
    k[:, -n:] = torch.randn((1, n, Hkv, D), generator=g, device="cuda").to(torch.bfloat16)
    v[:, -n:] = torch.randn((1, n, Hkv, D), generator=g, device="cuda").to(torch.bfloat16)
    kd = torch.zeros((1, Lk), dtype=torch.int32, device="cuda")
    kd[:, -n:] = 1
    qd = torch.ones((1, Lq), dtype=torch.int32, device="cuda")
    o, lse = vx.attn_mod_fwd(q, k, v, vx.Score(causal=True, q_doc=qd, k_doc=kd), return_lse=True)
    kc, vc = k[:, -n:].contiguous(), v[:, -n:].contiguous()
    ro, rl = vx.attn_mod_fwd(q, kc, vc, vx.Score(causal=True), return_lse=True)
    torch.cuda.synchronize()
    # two runs of the same rounding in other groupings
    assert (o.float() - ro.float()).abs().max() <= 4 * HALF * ro.float().abs().max()
    assert (lse - rl).abs().max() <= 2.0 ** -16


@pytest.mark.parametrize("B,H,Hkv,Lq,Lk", [(70, 2, 1, 1, 260), (130, 1, 1, 2, 129), (3, 4, 2, 3, 2100), (5, 32, 1, 1, 1000),
                                           (2, 12, 12, 1, 3000), (9, 8, 2, 7, 640), (1, 8, 4, 16, 4097)])
@pytest.mark.parametrize("fill", ["ragged", "mostly_empty", "full"])
def test_single_tokens_against_caches_of_any_fill(B, H, Hkv, Lq, Lk, fill):
    """Batches cut into units that end one cache and begin the next; empty caches among them."""
    q, k, v = make(B, H, Hkv, Lq, Lk, B + Lk)
    rng = np.random.default_rng([B, Lk])
    n = rng.integers(0, Lk + 1, size=B)
    if fill == "mostly_empty":
        n[rng.random(B) < 0.8] = 0
        n[-1] = Lk // 2
    if fill == "full":
        n[:] = Lk
    check(q, k, v, causal=True, cap=30.0, kv_valid_len=n, q_start=n - Lq, what=f"{B}x{H}/{Hkv} {Lq}x{Lk} {fill}")
