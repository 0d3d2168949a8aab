"""A transformer block's attention half as a model runs it, from the operators
together: block norm, projections, rotary embedding, attention with score
modifiers, projection, the gated residual step of the next block norm; forward,
gradients, a step for single tokens on a cache, and a captured graph.

Reference: the same chain in float64 by torch on the CPU, with autograd.
Tolerance: the tensors that are bf16 between the steps are rounded in a second
float64 run of the chain, both ways (activations forward, their gradients
backward); how far that moves a result is what its types cost.  The kernels make
those roundings and inside at most as many again (P and ds to bf16, D from the
rounded output), each of the same size: results are held to three times it,
relative RMS.
"""

import math

import numpy as np
import pytest

import oracle
import paper_2609_18077_amd as vx
from tests.gpu_util import log

pytestmark = pytest.mark.gpu

B, GRID, H, HKV, D = 2, (3, 9, 8), 4, 2, 128
L, C = 216, 512
DOCS = [(0, 100, 180, 200), (0, 37, 38, 216)]  # starts of a sequence's documents; what follows the last belongs to none
CAP, SLOPES = 8.0, (0.02, 0.0, 0.05, 0.01)


def _inputs(torch):
    gen = torch.Generator().manual_seed(17)
    r = lambda *s, mul=1.0: torch.randn(s, generator=gen) * mul
    t = dict(x=r(B, L, C).bfloat16(), scale1=r(B, C, mul=0.3), shift1=r(B, C, mul=0.3), gain1=1 + r(C, mul=0.1),
             gate=r(B, C), scale2=r(B, C, mul=0.3), shift2=r(B, C, mul=0.3), post_gain=1 + r(C, mul=0.1),
             wq=r(H * D, C, mul=C ** -0.5).bfloat16(), wk=r(HKV * D, C, mul=C ** -0.5).bfloat16(),
             wv=r(HKV * D, C, mul=C ** -0.5).bfloat16(), wo=r(C, H * D, mul=(H * D) ** -0.5).bfloat16())
    g = dict(h=r(B, L, C).bfloat16(), x=r(B, L, C).bfloat16())
    ids = torch.full((B, L), -1, dtype=torch.int32)
    for b, starts in enumerate(DOCS):
        for n, (s, e) in enumerate(zip(starts, starts[1:])):
            ids[b, s:e] = n
    return t, g, ids, torch.tensor(SLOPES)


def _chain64(torch, t, g, ids, slopes, causal, rounded):
    """(h, x') and the gradients of every operand, in float64."""

    class Round(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x):
            return x.to(torch.bfloat16).double()

        @staticmethod
        def backward(ctx, g):
            return g.to(torch.bfloat16).double()

    rd = Round.apply if rounded else lambda x: x
    t = {n: x.double().requires_grad_() for n, x in t.items()}

    def ln(x):
        x = x - x.mean(-1, keepdim=True)
        return x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6)

    def rms(x):
        return x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-6)

    f = torch.from_numpy(oracle.rope_angles(oracle.RopeSpec(GRID), np.arange(L)))  # [L, 64]

    def rope(x):
        a, b = x[..., 0::2], x[..., 1::2]
        c, s = f.cos()[None, :, None], f.sin()[None, :, None]
        return torch.stack((a * c - b * s, a * s + b * c), -1).flatten(-2)

    h = rd(rms(t["x"]) * t["gain1"] * (1 + t["scale1"][:, None]) + t["shift1"][:, None])
    q = rd(rope(rd((h @ t["wq"].T)).view(B, L, H, D)))
    k = rd(rope(rd((h @ t["wk"].T)).view(B, L, HKV, D)))
    v = rd(h @ t["wv"].T).view(B, L, HKV, D)
    k2, v2 = (z.repeat_interleave(H // HKV, 2) for z in (k, v))
    s = torch.einsum("bihd,bjhd->bhij", q, k2) / math.sqrt(D)
    i = torch.arange(L, dtype=torch.float64)
    s = CAP * torch.tanh(s / CAP) - slopes.double()[None, :, None, None] * (i[:, None] - i[None]).abs()
    see = (ids[:, :, None] == ids[:, None]) & (ids[:, :, None] >= 0)
    if causal:
        see &= i[None, :, None] >= i[None, None]
    s = s.masked_fill(~see[:, None], -1e300)
    p = torch.softmax(s, -1) * see[:, None]
    o = rd(torch.einsum("bhij,bjhd->bihd", p, v2))
    y = rd(o.flatten(2) @ t["wo"].T)
    x = rd(t["x"] + t["gate"][:, None] * rms(y) * t["post_gain"])
    # (the norm reads x' before it is rounded; the difference is one more rounding)
    out = rd(ln(x) * (1 + t["scale2"][:, None]) + t["shift2"][:, None])
    torch.autograd.backward([out, x], [g["h"].double(), g["x"].double()])
    return dict(h=out.detach(), x=x.detach(), **{"d" + n: z.grad for n, z in t.items()})


def _forward(t, score):
    """(h, x') and what the backward needs."""
    rope = vx.Rope(GRID)
    _, h1 = vx.block_norm_fwd(t["x"], scale=t["scale1"], shift=t["shift1"], gain=t["gain1"], norm="rms")
    h2 = h1.view(-1, C)
    q, k, v = ((h2 @ t[w].T).view(B, L, -1, D) for w in ("wq", "wk", "wv"))
    vx.rope3d(q, rope, out=q)
    vx.rope3d(k, rope, out=k)
    o, lse = vx.attn_mod_fwd(q, k, v, score, return_lse=True)
    y = (o.view(B * L, -1) @ t["wo"].T).view(B, L, C)
    x, h = vx.block_norm_fwd(t["x"], y, gate=t["gate"], scale=t["scale2"], shift=t["shift2"], post="rms",
                             post_gain=t["post_gain"])
    return (h, x), (q, k, v, o, lse, y, x)


def _backward(torch, t, g, score, saved):
    q, k, v, o, lse, y, x = saved
    rope = vx.Rope(GRID)
    r2 = vx.block_norm_bwd(g["h"], g["x"], x, y, gate=t["gate"], scale=t["scale2"], shift=t["shift2"], post="rms",
                           post_gain=t["post_gain"])
    do = (r2["dy"].view(-1, C) @ t["wo"]).view(B, L, H, D)
    dq, dk, dv = vx.attn_mod_bwd(q, k, v, o, do, lse, score)
    vx.rope3d_transpose(dq, rope, out=dq)
    vx.rope3d_transpose(dk, rope, out=dk)
    d3 = torch.cat([z.view(B * L, -1) for z in (dq, dk, dv)], 1)
    dh = (d3 @ torch.cat([t["wq"], t["wk"], t["wv"]])).view(B, L, C)
    r1 = vx.block_norm_bwd(dh, r2["dx"], t["x"], scale=t["scale1"], shift=t["shift1"], gain=t["gain1"], norm="rms")
    return dict(dx=r1["dx"], dscale1=r1["dscale"], dshift1=r1["dshift"], dgain1=r1["dgain"], dgate=r2["dgate"],
                dscale2=r2["dscale"], dshift2=r2["dshift"], dpost_gain=r2["dpost_gain"])


def _score(ids, slopes, causal):
    ids = ids.cuda()
    return vx.Score(causal=causal, cap=CAP, slopes=slopes.cuda(), q_doc=ids, k_doc=ids)


@pytest.mark.parametrize("causal", [False, True])
def test_forward_and_gradients(causal):
    import torch

    t, g, ids, slopes = _inputs(torch)
    ref = _chain64(torch, t, g, ids, slopes, causal, False)
    typed = _chain64(torch, t, g, ids, slopes, causal, True)
    td, gd = ({n: z.cuda() for n, z in m.items()} for m in (t, g))
    score = _score(ids, slopes, causal)
    (h, x), saved = _forward(td, score)
    got = dict(h=h, x=x, **_backward(torch, td, gd, score, saved))
    for n, z in got.items():
        z = z.double().cpu()
        size = ref[n].square().mean().sqrt().item()
        err, cost = ((a - ref[n]).square().mean().sqrt().item() / size for a in (z, typed[n]))
        log(f"block {n}: {err:.2e}, of the types {cost:.2e}")
        assert z.isfinite().all() and err <= 3 * cost + L * 2.0 ** -24, (n, err, cost)  # (and fp32 sums over the tokens)


def test_captured_and_replayed():
    import torch

    t, g, ids, slopes = _inputs(torch)
    td, gd = ({n: z.cuda() for n, z in m.items()} for m in (t, g))
    score = _score(ids, slopes, True)

    def run():
        out, saved = _forward(td, score)
        return [*out, *_backward(torch, td, gd, score, saved).values()]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        static = run()
    for n in range(4):
        td["x"].copy_(torch.randn(td["x"].shape, generator=torch.Generator().manual_seed(n)))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(static, run()):
            assert torch.equal(a, b), n
        torch.cuda.synchronize()


def test_single_tokens_on_a_cache_continue_the_sequence():
    """The rows of one pass over the sequence, and the same tokens one by one on its keys and values."""
    import torch

    t, _, _, slopes = _inputs(torch)
    td = {n: z.cuda() for n, z in t.items()}
    w = torch.cat([td["wq"], td["wk"], td["wk"].flip(0), td["wv"], td["wv"].flip(0)])  # H heads each
    _, h1 = vx.block_norm_fwd(td["x"], scale=td["scale1"], shift=td["shift1"], norm="rms")
    q, k, v = vx.qkv_proj(h1.view(-1, C), w, B, L, H, rope=vx.Rope(GRID))

    def rest(x, q, score):
        o = vx.attn_mod_fwd(q, k, v, score)
        n = o.shape[1]
        y = (o.view(B * n, -1) @ td["wo"].T).view(B, n, C)
        return vx.block_norm_fwd(x, y, gate=td["gate"], scale=td["scale2"], shift=td["shift2"], post="rms")[1]

    s = dict(causal=True, cap=CAP, slopes=slopes.cuda())
    whole = rest(td["x"], q, vx.Score(**s))
    for n in (0, 1, 31, 32, 63, 64, 150, L - 1):
        at = torch.full((B,), n, dtype=torch.int32, device="cuda")
        one = rest(td["x"][:, n:n + 1].contiguous(), q[:, n:n + 1].contiguous(),
                   vx.Score(**s, q_start=at, kv_valid_len=at + 1))
        a, b = one[:, 0].double(), whole[:, n].double()
        # o rounded in each (P too, in the whole pass: 2^-8 at most each), y, h rounded in each
        assert (a - b).square().mean().sqrt() <= 6 * 2.0 ** -8 * b.square().mean().sqrt(), n
