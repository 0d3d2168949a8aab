"""Gradient of attention with score modifiers (vidax_attn_mod_bwd) against the
float64 reference.

Tolerances, per element.  The kernel rounds P and ds to bf16 once each before the
products that consume them (2^-8 of the value at most), forms D from the output
that the forward rounded to bf16 (the reference is given the same output), and
rounds the result once.  With delta the error of a score (as for the forward),
P is off by 2 delta of itself and ds by 4 delta of P (|dP| + |D|) and the fp32
errors of dP and D, 130 * 2^-24 of their terms.  So, with A the same sums taken
over absolute values, an element is off by at most (2^-8 + E) A and 2^-8 of
itself, E = 4 delta + 300 * 2^-24.  A weight below 2^-126 may count as zero, also
in a product with bf16: 2^-126 of the other factors, at most |dP| + |D| <= 256
max|dout| max|v| and |q| or |k| a row or key.  Beside that the relative RMS error of a
tensor is held to 2^-7.5, two independent roundings.
"""

import numpy as np
import pytest

import oracle
import paper_2609_18077_amd as vx
from tests.gpu_util import log
from tests.test_gpu_attn_mod import check as fwd_check
from tests.test_gpu_attn_mod import D, HALF, MASKS, PIECES, RMS, SCALE, deltas, dev_score, f64, make, masks, piece_score

pytestmark = pytest.mark.gpu


def _absolute(q, k, v, o, g, scale, spec):
    """The sums of the gradients over absolute values: (dq, dk, dv)."""
    B, Lq, H, _ = q.shape
    rep = H // k.shape[2]
    out = [np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)]
    for b in range(B):
        for h in range(H):
            qh, kh, vh, gh, oh = q[b, :, h], k[b, :, h // rep], v[b, :, h // rep], g[b, :, h], o[b, :, h]
            x, t = oracle.attn_mod.scores(qh, kh, b, h, scale, spec)
            p, _ = oracle.attn_mod.probabilities(x)
            ds = p * (np.abs(gh) @ np.abs(vh).T + (np.abs(gh) * np.abs(oh)).sum(1)[:, None])
            if t is not None:
                ds = ds * (1 - t * t + 2.0 ** -20)
            out[0][b, :, h] = abs(scale) * ds @ np.abs(kh)
            out[1][b, :, h // rep] += abs(scale) * ds.T @ np.abs(qh)
            out[2][b, :, h // rep] += p.T @ np.abs(gh)
    return out


def check(q, k, v, scale=None, what="", workspace=None, dout=None, **s):
    import torch

    score, spec = dev_score(**s)
    if dout is None:
        gen = torch.Generator(device="cuda").manual_seed(99)
        dout = torch.randn(q.shape, generator=gen, device="cuda").to(torch.bfloat16)
    o, lse = vx.attn_mod_fwd(q, k, v, score, scale=scale, return_lse=True)
    got = vx.attn_mod_bwd(q, k, v, o, dout, lse, score, scale=scale, workspace=workspace)
    torch.cuda.synchronize()
    compare(got, o, dout, q, k, v, SCALE if scale is None else float(np.float32(scale)), spec, what)
    return o, lse, dout, got


def compare(got, o, dout, q, k, v, sc, spec, what):
    args = [f64(t) for t in (q, k, v)]
    ref = oracle.attn_mod_bwd_ref(*args, f64(dout), sc, spec, o_saved=f64(o))
    mags = _absolute(*args, f64(o), f64(dout), sc, spec)
    E = 4 * deltas(*args[:2], sc, spec).max(initial=0) + 300 * 2.0 ** -24
    most = lambda *a: float(np.prod([np.abs(t).max(initial=0) + 1 for t in a]))
    under = 2.0 ** -126 * 256 * (args[0].shape[1] * args[0].shape[2] + args[1].shape[1]) * most(f64(dout), *args)
    for n, x, r, m in zip(("dq", "dk", "dv"), got, ref, mags):
        x = f64(x)
        assert np.isfinite(x).all(), (what, n)
        tol = (HALF + E) * m + HALF * (np.abs(r) + (HALF + E) * m) + under
        err = np.abs(x - r)
        norm = np.sqrt((r ** 2).sum())
        rms = np.sqrt((err ** 2).sum()) / norm if norm else 0.0
        worst = float((err / np.maximum(tol, 1e-300)).max(initial=0)) if err.size else 0.0
        log(f"  {what} {n}: worst/bound {worst:.3f}, rel rms {rms:.2e}")
        assert worst <= 1, (what, n, worst)
        assert norm < 1e-20 or rms <= RMS, (what, n, rms)


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("cap,bias", [(0.0, False), (20.0, False), (0.0, True), (3.0, True)])
def test_masks_and_modifiers(mask, cap, bias):
    B, H, Hkv, Lq, Lk = 2, 4, 2, 300, 419
    q, k, v = make(B, H, Hkv, Lq, Lk, 41, mul=4.0 if cap else 1.0)
    slopes = [0.5, 0.0, -0.01, 0.02] if bias else None
    check(q, k, v, cap=cap, slopes=slopes, what=f"{mask} cap={cap} bias={bias}", **masks(mask, B, Lq, Lk))


@pytest.mark.parametrize("Lq,Lk", [(1, 1), (1, 2), (2, 1), (5, 3), (33, 32), (64, 64), (65, 63), (256, 64), (257, 65),
                                   (255, 128), (129, 257), (300, 193), (513, 700), (40, 1300)])
@pytest.mark.parametrize("mask", ["all", "causal", "docs_valid_prefix"])
def test_sizes(Lq, Lk, mask):
    q, k, v = make(1, 3, 3, Lq, Lk, Lq + Lk)
    check(q, k, v, what=f"{Lq}x{Lk} {mask}", **masks(mask, 1, Lq, Lk))


@pytest.mark.parametrize("H,Hkv", [(1, 1), (5, 5), (6, 3), (8, 1), (20, 4)])
def test_gradients_of_shared_heads(H, Hkv):
    q, k, v = make(2, H, Hkv, 70, 150, H)
    check(q, k, v, causal=True, what=f"{H}/{Hkv}")


@pytest.mark.parametrize("scale", [0.0, -0.05, 0.7])
@pytest.mark.parametrize("cap", [0.0, 2.0])
def test_scales(scale, cap):
    q, k, v = make(1, 2, 2, 130, 200, 21)
    check(q, k, v, scale=scale, cap=cap, causal=True, slopes=[0.1, 0.2], what=f"scale {scale} cap {cap}")


@pytest.mark.parametrize("Lq,Lk,Hkv", [(3000, 100, 1), (4000, 300, 2), (1300, 1300, 1)])
def test_runs_of_queries_are_added_up(Lq, Lk, Hkv):
    import torch

    B, H = 1, 2
    q, k, v = make(B, H, Hkv, Lq, Lk, 27)
    s = masks("docs_valid_prefix", B, Lq, Lk)
    need = vx.lib().vidax_attn_mod_bwd_workspace_floats(B, H, Hkv, Lq, Lk, D, 1)
    most = 2 * B * H * Lq + B * (2 * -(-Lq // 64) + -(-Lk // 256)) + 256 + B * (4 * (-(-Lk // 64) + -(-Lq // 64)) + -(-Lk // 256) + -(-Lq // 256))
    assert need > most  # several runs
    o, lse, dout, got = check(q, k, v, what="runs", **s)
    ws = torch.empty(most, device="cuda")
    *_, one = check(q, k, v, what="one run", workspace=ws, **s)
    assert torch.equal(got[0], one[0])  # the query side does not depend on it
    score, _ = dev_score(**s)
    with pytest.raises(vx.VidaxError):
        vx.attn_mod_bwd(q, k, v, o, dout, lse, score, workspace=ws[:B * H * Lq])


@pytest.mark.parametrize("B,H,Hkv,Lq,Lk,mask", PIECES)
def test_pieces_of_tiles_are_added_up(B, H, Hkv, Lq, Lk, mask):
    """Checked on two groups of heads of every batch."""
    import torch

    q, k, v = make(B, H, Hkv, Lq, Lk, Lq + Lk)
    s, slopes = piece_score(B, H, Lq, Lk, mask)
    score, _ = dev_score(**s)
    dout = make(B, H, Hkv, Lq, 1, 7)[0]
    o, lse = vx.attn_mod_fwd(q, k, v, score, return_lse=True)
    got = vx.attn_mod_bwd(q, k, v, o, dout, lse, score)
    ws = torch.full((vx.lib().vidax_attn_mod_bwd_workspace_floats(B, H, Hkv, Lq, Lk, D, 0),), float("nan"), device="cuda")
    for a, b in zip(got, vx.attn_mod_bwd(q, k, v, o, dout, lse, score, workspace=ws)):
        assert torch.equal(a, b)
    rep = H // Hkv
    for g in {0, Hkv - 1}:
        hs, ks = slice(g * rep, g * rep + rep), slice(g, g + 1)
        one = oracle.ScoreSpec(**{**s, "slopes": slopes[hs] if slopes is not None else None})
        compare([got[0][:, :, hs], got[1][:, :, ks], got[2][:, :, ks]], o[:, :, hs], dout[:, :, hs], q[:, :, hs], k[:, :, ks],
                v[:, :, ks], SCALE, one, f"pieces {Lq}x{Lk} {mask} group {g}")


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_sees_nothing_or_is_not_seen_does_not_matter(bad):
    """NaN and infinities in k, v where no query sees them, in q and dout at rows that see nothing."""
    import torch

    B, H, Lq, Lk = 2, 2, 330, 500
    q, k, v = make(B, H, H, Lq, Lk, 25)
    g = torch.randn(q.shape, device="cuda").to(torch.bfloat16)
    cases = [({"kv_valid_len": [201, 0]}, [(0, 201, 500), (1, 0, 500)], [(1, 0, 330)]),
             ({"causal": True, "q_start": [-37, 30]}, [(0, 293, 500), (1, 360, 500)], [(0, 0, 37)]),
             ({"q_doc": np.where(np.arange(Lq) % 50 < 20, -1, 0)[None].repeat(B, 0),
               "k_doc": np.where(np.arange(Lk) % 100 < 37, -1, 0)[None].repeat(B, 0)},
              [(b, i, i + 37) for b in range(B) for i in range(0, Lk, 100)],
              [(b, i, min(i + 20, Lq)) for b in range(B) for i in range(0, Lq, 50)])]
    for s, keys, rows in cases:
        score, _ = dev_score(**s)
        o, lse = vx.attn_mod_fwd(q, k, v, score, return_lse=True)
        want = vx.attn_mod_bwd(q, k, v, o, g, lse, score)
        q2, k2, v2, g2 = (t.clone() for t in (q, k, v, g))
        for b, i, j in keys:
            k2[b, i:j], v2[b, i:j] = bad, -bad
        for b, i, j in rows:
            q2[b, i:j], g2[b, i:j] = bad, -bad
            assert not want[0][b, i:j].any()
        got = vx.attn_mod_bwd(q2, k2, v2, o, g2, lse, score)
        for n, x, y in zip(("dq", "dk", "dv"), got, want):
            assert torch.isfinite(y.float()).all(), (list(s), n)
            assert torch.equal(x, y), (list(s), n)
        for b, i, j in keys:
            assert not want[1][b, i:j].any() and not want[2][b, i:j].any()


def test_empty_calls():
    import torch

    z = lambda *s, dtype=torch.bfloat16: torch.empty(s, dtype=dtype, device="cuda")
    for B, Lq, Lk, H in ((0, 3, 5, 2), (2, 0, 5, 2), (2, 3, 0, 2), (2, 3, 5, 0)):
        q, k = z(B, Lq, H, D), z(B, Lk, H, D)
        q.fill_(1)
        k.fill_(1)
        lse = torch.full((B, H, Lq), -float("inf"), device="cuda")
        for x in vx.attn_mod_bwd(q, k, k, q, q, lse, vx.Score(causal=True)):
            assert not x.any()


@pytest.mark.parametrize("seed", range(18))
def test_random_calls(seed):
    """Seeded sizes, heads and modifiers of every kind together, lengths and positions past their ends among them."""
    rng = np.random.default_rng(1000 + seed)
    Hkv = int(rng.integers(1, 4))
    B, H = int(rng.integers(1, 4)), Hkv * int(rng.integers(1, 4))
    Lq, Lk = (int(np.exp(rng.uniform(*((0, 6.3) if seed < 12 else (4.5, 7.8))))) for _ in range(2))
    s = dict(causal=bool(rng.integers(2)), cap=float(rng.choice([0.0, 0.0, 3.0, 30.0, 200.0])))
    if rng.integers(2):
        s["slopes"] = list(rng.normal(0, 0.1, H))
    if rng.integers(2):
        s["q_doc"], s["k_doc"] = (np.sort(rng.integers(-1, 4, (B, L)), axis=1) if rng.integers(2) else rng.integers(-1, 3, (B, L))
                                  for L in (Lq, Lk))
    if rng.integers(2):
        s["kv_valid_len"] = rng.integers(-3, Lk + 9, B)
    if s["causal"] and rng.integers(2):
        s["prefix_len"] = rng.integers(-3, Lk + 9, B)
    if rng.integers(2):
        s["q_start"] = rng.integers(-Lq, Lk + 50, B)
    q, k, v = make(B, H, Hkv, Lq, Lk, seed)
    check(q, k, v, what=f"random {seed}: {B}x{H}/{Hkv} {Lq}x{Lk} {sorted(s)}", **s)
    fwd_check(q, k, v, what=f"random {seed}", **s)


def test_differences():
    """The kernel's gradients against central differences of the kernel's forward,
    along random directions.  Forward and gradient are good to about 2^-8 relative
    RMS; a difference over 2 h of sums of n such outputs adds their errors in
    quadrature, sqrt(n) 2^-8 |g o| / (2 h) on the derivative."""
    import torch

    B, H, Hkv, L = 1, 4, 2, 200
    q, k, v = make(B, H, Hkv, L, L, 42, mul=2.0)
    score, _ = dev_score(causal=True, cap=6.0, slopes=[0.1, 0.05, 0.02, 0.01], prefix_len=[50])
    g = torch.randn(q.shape, device="cuda").to(torch.bfloat16)
    o, lse = vx.attn_mod_fwd(q, k, v, score, return_lse=True)
    grads = vx.attn_mod_bwd(q, k, v, o, g, lse, score)
    for i, n in enumerate("qkv"):
        x = (q, k, v)[i]
        # a direction in the gradient's own sign: no cancellation in the sum
        d = grads[i].float().sign() * x.float().abs() * 0.125
        up, down = (x.float() + d).to(torch.bfloat16), (x.float() - d).to(torch.bfloat16)
        step = up.double() - down.double()
        f = [vx.attn_mod_fwd(*[y if j == i else (q, k, v)[j] for j in range(3)], score) for y in (up, down)]
        diff = float((g.double() * (f[0].double() - f[1].double())).sum())
        want = float((grads[i].double() * step).sum())
        noise = float(((g.double() * o.double()) ** 2).sum().sqrt()) * HALF * 2
        # the third derivative: steps of an eighth of the operand change a score by up to an eighth of itself
        assert abs(diff - want) <= 3 * noise + 0.06 * abs(want), (n, diff, want, noise)


def test_same_bits_twice_on_another_stream_and_in_a_graph():
    import torch

    q, k, v = make(2, 4, 2, 300, 900, 29)
    score, _ = dev_score(cap=10.0, **masks("docs_valid_prefix", 2, 300, 900))
    g = torch.randn(q.shape, device="cuda").to(torch.bfloat16)

    def work():
        o, lse = vx.attn_mod_fwd(q, k, v, score, return_lse=True)
        return [o, lse, *vx.attn_mod_bwd(q, k, v, o, g, lse, score)]

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
