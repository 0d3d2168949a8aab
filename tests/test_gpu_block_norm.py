"""The block norm (vidax_block_norm_fwd, _bwd) against the float64 reference.

Tolerances.  A value rounded to bf16 is off by at most 2^-8 of itself.  What
precedes the rounding is fp32: a channel sum takes at most 32 additions in a
lane, 6 between lanes and 8 between waves, a mean and a variance two such sums,
so a normalised value is off by at most about 64 * 2^-24 of the row's scale
rho = max|v| / root (a large mean cancels), and each further product or sum adds
2^-24 of its terms.  U = 128 * 2^-24 covers both, against the magnitudes of the
terms (with absolute values throughout, so that cancellation is not counted
against the kernel).  A sum over tokens adds up to `rows` terms in a lane, up to
8 groups and 512 runs of them: (rows + 600) * 2^-24 of the sum of magnitudes is
a bound for any order.
"""

import numpy as np
import pytest

import oracle
import paper_2609_18077_amd as vx
from tests.gpu_util import log

pytestmark = pytest.mark.gpu

U = 128 * 2.0 ** -24
HALF = 2.0 ** -8


def _np(t):
    return t.detach().double().cpu().numpy()


def _inputs(torch, B, L, C, fp32, norm, post, token, seed, offset=0.0, strided=True):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rnd = lambda *s: torch.randn(s, generator=g, device="cuda")
    stream = torch.float32 if fp32 else torch.bfloat16
    a = {"x": (rnd(B, L, C) * 2 + offset).to(stream), "y": (rnd(B, L, C) * 0.5 + offset / 2).to(torch.bfloat16)}
    rows = L if token else 1
    if strided:
        t = rnd(B, rows, 3, C) * 0.3
        mods = t.unbind(2)
    else:
        mods = [rnd(B, rows, C) * 0.3 if token else rnd(B, C) * 0.3 for _ in range(3)]
    a["gate"], a["scale"], a["shift"] = mods
    a["gain"] = 1 + 0.1 * rnd(C)
    if post:
        a["post_gain"] = 1 + 0.1 * rnd(C)
    return a, dict(norm=norm, post=post, eps=1e-6), rnd


def _within(got, ref, tol, what):
    got = _np(got)
    assert got.shape == ref.shape, what
    assert np.isfinite(got).all(), what
    excess = np.abs(got - ref) - tol
    log(f"  {what}: worst error over its bound {np.max(np.abs(got - ref) / tol):.3f}")
    assert excess.max() <= 0, (what, float(excess.max()))


def _mod(m):
    return _np(m) if m.dim() == 3 else _np(m)[:, None]


def _magnitudes(a, kw, alpha, xo):
    """|terms| of x' and of h, and the scales of the two normalised rows."""
    one = lambda n: np.ones(xo.shape[-1]) if a.get(n) is None else np.abs(_np(a[n]))
    y = _np(a["y"])
    yh, ry = (y, None) if kw["post"] is None else oracle.block_norm.normalise(y, kw["post"], kw["eps"])
    rho_y = np.abs(yh) if ry is None else np.abs(yh) + np.abs(y).max(-1, keepdims=True) * ry
    mx = np.abs(alpha * _np(a["x"])) + np.abs(_mod(a["gate"])) * one("post_gain") * rho_y
    hat, r = oracle.block_norm.normalise(xo, kw["norm"], kw["eps"])
    rho = np.abs(hat) + mx.max(-1, keepdims=True) * r
    return mx, rho, rho_y, hat, r


def check_forward(torch, a, kw, alpha=1.0, out=None, what=""):
    x, h = vx.block_norm_fwd(**a, **kw, alpha=alpha, out=out)
    torch.cuda.synchronize()
    rx, rh = oracle.block_norm_ref(*(_np(a[n]) for n in ("x", "y")), gate=_np(a["gate"]), scale=_np(a["scale"]),
                                   shift=_np(a["shift"]), gain=_np(a["gain"]),
                                   post_gain=_np(a["post_gain"]) if "post_gain" in a else None, **kw, alpha=alpha)
    mx, rho, *_ = _magnitudes(a, kw, alpha, rx)
    half = 0.0 if a["x"].dtype == torch.float32 else HALF
    mul = np.abs(_np(a["gain"]) * (1 + _mod(a["scale"])))
    _within(x, rx, U * mx + half * np.abs(rx), f"{what} x'")
    ph = U * (rho * mul + np.abs(_mod(a["shift"])))
    _within(h, rh, ph + HALF * (np.abs(rh) + ph), f"{what} h")
    return x, h


def check_backward(torch, a, kw, rnd, alpha=1.0, with_dx=True, what=""):
    B, L, C = a["x"].shape
    stream = a["x"].dtype
    dh = rnd(B, L, C).to(torch.bfloat16)
    dx = rnd(B, L, C).to(stream) if with_dx else None
    ops = {n: z for n, z in a.items() if n != "x"}
    got = vx.block_norm_bwd(dh, dx, a["x"], **ops, **kw, alpha=alpha)
    again = vx.block_norm_bwd(dh, dx, a["x"], **ops, **kw, alpha=alpha)
    torch.cuda.synchronize()
    for n in got:
        assert torch.equal(got[n], again[n]), f"{n} differs between two calls"
    ref = oracle.block_norm_bwd_ref(_np(dh), None if dx is None else _np(dx), _np(a["x"]),
                                    **{n: _np(z) for n, z in ops.items()}, **kw, alpha=alpha)
    assert set(got) == set(ref)
    _, rho, rho_y, hat, r = _magnitudes({**a, "gate": a["gate"] * 0}, kw, 1.0, _np(a["x"]))
    one = lambda n: np.ones(C) if n not in a else np.abs(_np(a[n]))
    s1, gate, adh = np.abs(1 + _mod(a["scale"])), np.abs(_mod(a["gate"])), np.abs(_np(dh))
    w = adh * one("gain") * s1
    # |terms| of g; a row sum of products carries the products' own errors
    mg = r * (w * (1 + 0 * rho) + rho * (w * rho).mean(-1, keepdims=True) + w.mean(-1, keepdims=True))
    if dx is not None:
        mg = mg + np.abs(_np(dx))
    half = 0.0 if stream == torch.float32 else HALF
    _within(got["dx"], ref["dx"], abs(alpha) * U * mg + half * (np.abs(ref["dx"]) + U * mg), f"{what} dx")
    da = mg * gate * one("post_gain")
    if kw["post"]:
        _, ry = oracle.block_norm.normalise(_np(a["y"]), kw["post"], kw["eps"])
        da = ry * (da + rho_y * (da * rho_y).mean(-1, keepdims=True) + da.mean(-1, keepdims=True))
    _within(got["dy"], ref["dy"], U * da + HALF * (np.abs(ref["dy"]) + U * da), f"{what} dy")
    rows = vx.lib().vidax_block_norm_bwd_workspace_floats(B, L, C)
    runs = rows // (3 * B * C)
    n_add = -(-L // runs) + 600 + B
    terms = {"dscale": adh * rho * one("gain"), "dshift": adh, "dgain": adh * rho * s1,
             "dgate": mg * rho_y * one("post_gain"), "dpost_gain": mg * gate * rho_y}
    for n in ref:
        if n in ("dx", "dy"):
            continue
        t = terms[n] + np.zeros((B, L, C))
        if n in ("dgain", "dpost_gain"):
            t = t.sum((0, 1))
        elif ref[n].ndim == 2:
            t = t.sum(1)
        elif ref[n].shape[1] != L:
            t = t.sum(1, keepdims=True)
        _within(got[n], ref[n], (U + n_add * 2.0 ** -24) * t + 1e-30, f"{what} {n}")


# one lane's chunk to a row of several waves; a size that fills no wave; the
# widths at which a lane takes another chunk; the largest
CHANNELS = [8, 64, 520, 1536, 1544, 4096, 4104, 5120, 8200, 16384]


@pytest.mark.parametrize("C", CHANNELS)
@pytest.mark.parametrize("norm,post", [("layer", None), ("rms", "rms"), ("layer", "layer"), ("rms", None)])
@pytest.mark.parametrize("fp32", [False, True], ids=["bf16", "fp32"])
def test_forward_and_backward(C, norm, post, fp32):
    import torch

    B, L = 2, 7
    a, kw, rnd = _inputs(torch, B, L, C, fp32, norm, post, False, seed=C + 17 * fp32)
    check_forward(torch, a, kw, what=f"C={C} {norm}/{post}")
    check_backward(torch, a, kw, rnd, what=f"C={C} {norm}/{post}")


@pytest.mark.parametrize("B,L,C", [(1, 1, 1536), (16, 1, 5120), (3, 2, 640), (1, 33, 1544), (2, 1200, 256), (1, 4099, 768),
                                   (5, 257, 1024)])
@pytest.mark.parametrize("token", [False, True], ids=["sample", "token"])
@pytest.mark.parametrize("strided", [False, True], ids=["dense", "strided"])
def test_lengths_and_modulation_rows(B, L, C, token, strided):
    import torch

    a, kw, rnd = _inputs(torch, B, L, C, L % 2 == 0, "rms", "rms", token, seed=L + C, strided=strided)
    check_forward(torch, a, kw, alpha=0.75, what=f"{B}x{L}x{C}")
    check_backward(torch, a, kw, rnd, alpha=0.75, with_dx=L != 33, what=f"{B}x{L}x{C}")


@pytest.mark.parametrize("C", [512, 1536, 5120])
def test_rows_far_from_zero(C):
    """Means of a thousand deviations: the variance is not a difference of squares."""
    import torch

    a, kw, rnd = _inputs(torch, 2, 5, C, True, "layer", "layer", False, seed=C, offset=1000.0)
    check_forward(torch, a, kw, what="offset")
    a["x"] = vx.block_norm_fwd(**a, **kw)[0]
    check_backward(torch, a, kw, rnd, what="offset")


def test_without_branch_gains_or_modulations():
    import torch

    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = torch.randn((2, 9, 776), generator=g, device="cuda").to(torch.bfloat16)
    xo, h = vx.block_norm_fwd(x, norm="layer")
    assert xo is x
    rh = oracle.block_norm_ref(_np(x), norm="layer")[1]
    _within(h, rh, 8 * U + HALF * (np.abs(rh) + 8 * U), "h alone")
    dh = torch.randn((2, 9, 776), generator=g, device="cuda").to(torch.bfloat16)
    got = vx.block_norm_bwd(dh, None, x, norm="layer")
    assert set(got) == {"dx"}
    ref = oracle.block_norm_bwd_ref(_np(dh), None, _np(x), norm="layer")["dx"]
    _within(got["dx"], ref, 64 * U + HALF * (np.abs(ref) + 64 * U), "dx alone")
    x2, h2 = vx.block_norm_fwd(x, alpha=0.5, norm="rms")
    assert torch.equal(x2.float(), x.float() * 0.5)  # exact: a power of two
    y = torch.randn((2, 9, 776), generator=g, device="cuda").to(torch.bfloat16)
    got = vx.block_norm_bwd(dh, x, x, y, norm="rms", post="layer", gain=torch.ones(776, device="cuda"))
    ref = oracle.block_norm_bwd_ref(_np(dh), _np(x), _np(x), _np(y), norm="rms", post="layer", gain=np.ones(776))
    assert set(got) == set(ref) == {"dx", "dy", "dgain"}
    for n in ("dx", "dy"):
        _within(got[n], ref[n], 512 * U + HALF * (np.abs(ref[n]) + 512 * U), n)


def test_in_place_and_given_outputs():
    import torch

    a, kw, _ = _inputs(torch, 2, 37, 1536, False, "rms", "rms", False, seed=4)
    x, h = check_forward(torch, a, kw)
    h2 = torch.empty_like(h)
    a2 = {**a, "x": a["x"].clone()}
    x2, h3 = vx.block_norm_fwd(**a2, **kw, out=(a2["x"], h2))
    assert x2 is a2["x"] and h3 is h2
    assert torch.equal(x2, x) and torch.equal(h2, h)


def test_rows_beside_the_call_stay():
    """The outputs are the middle of larger buffers."""
    import torch

    B, L, C = 1, 13, 1544
    a, kw, _ = _inputs(torch, B, L, C, False, "layer", None, False, seed=5)
    big = torch.full((2, L + 2, C), 7.0, dtype=torch.bfloat16, device="cuda")
    out = tuple(big[i, 1:L + 1].reshape(1, L, C) for i in range(2))
    vx.block_norm_fwd(**a, **kw, out=out)
    torch.cuda.synchronize()
    assert bool((big[:, 0] == 7).all()) and bool((big[:, -1] == 7).all())
    x, h = vx.block_norm_fwd(**a, **kw)
    assert torch.equal(out[0], x) and torch.equal(out[1], h)


def test_empty_calls_and_sums_over_nothing():
    import torch

    z = lambda *s, dtype=torch.bfloat16: torch.empty(s, dtype=dtype, device="cuda")
    for B, L in ((0, 4), (2, 0)):
        x, h = vx.block_norm_fwd(z(B, L, 64), z(B, L, 64), gate=z(B, 64, dtype=torch.float32))
        assert x.shape == h.shape == (B, L, 64)
        got = vx.block_norm_bwd(h, None, x, z(B, L, 64), gate=torch.ones((B, 64), device="cuda"),
                                gain=torch.ones(64, device="cuda"))
        assert not got["dgain"].any() and not got["dgate"].any()


def test_other_stream_and_graph_replays():
    import torch

    a, kw, rnd = _inputs(torch, 2, 300, 1536, False, "rms", "rms", False, seed=6)
    dh, dx = rnd(2, 300, 1536).to(torch.bfloat16), rnd(2, 300, 1536).to(torch.bfloat16)
    ops = {n: z for n, z in a.items() if n != "x"}
    work = lambda: (vx.block_norm_fwd(**a, **kw), vx.block_norm_bwd(dh, dx, a["x"], **ops, **kw))
    flat = lambda r: [*r[0], *(r[1][n] for n in sorted(r[1]))]
    want = [t.clone() for t in flat(work())]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = flat(work())
    s.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = flat(work())
    for i in range(3):
        for t in held:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(held, want)), i
        assert all(torch.equal(p, q) for p, q in zip(flat(work()), want)), i
