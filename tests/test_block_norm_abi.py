"""Refusals of the block norm: the C ABI rejects what it cannot do before any
launch, the binding what it cannot express.  No GPU is needed."""

import ctypes

import pytest

import paper_2609_18077_amd as vx

INV, UNS = 1, 2
P = 1 << 40  # fake device addresses, far apart, never dereferenced


def _desc(fp32=0, norm=1, post=0, per_token=0, eps=1e-6, alpha=1.0, gain=None, post_gain=None, gate=(None, 0, 0),
          scale=(None, 0, 0), shift=(None, 0, 0)):
    return vx.BlockNormDesc(fp32, norm, post, per_token, eps, alpha, gain, post_gain, vx.BlockMod(*gate),
                            vx.BlockMod(*scale), vx.BlockMod(*shift))


def _p(x):
    return ctypes.c_void_p(x) if x else None


def _fwd(x=P, y=2 * P, xo=3 * P, h=4 * P, B=2, L=8, C=64, desc=None, **d):
    desc = desc or _desc(**d)
    return vx.lib().vidax_block_norm_fwd(_p(x), _p(y), _p(xo), _p(h), B, L, C, ctypes.byref(desc), None)


def _bwd(dh=P, dxo=2 * P, xo=3 * P, y=4 * P, dx=5 * P, dy=6 * P, grads=(), ws=None, wn=0, B=2, L=8, C=64, **d):
    g = vx.BlockNormGrads(**dict(grads))
    return vx.lib().vidax_block_norm_bwd(_p(dh), _p(dxo), _p(xo), _p(y), _p(dx), _p(dy), ctypes.byref(g), _p(ws), wn, B,
                                         L, C, ctypes.byref(_desc(**d)), None)


def test_forward_refusals():
    assert _fwd(B=0, x=0, y=0, xo=0, h=0) == 0
    assert _fwd(C=0) == 0
    for bad in (dict(x=0), dict(h=0), dict(xo=0), dict(x=P + 8), dict(y=2 * P + 2), dict(h=4 * P + 4), dict(B=-1),
                dict(L=-1), dict(C=-8), dict(fp32=2), dict(norm=0), dict(norm=3), dict(post=3), dict(post=-1),
                dict(per_token=2), dict(eps=-1.0), dict(eps=float("nan")), dict(alpha=float("inf")),
                dict(post_gain=8 * P), dict(gain=8 * P + 4), dict(y=0, gate=(8 * P, 64, 0)), dict(y=0, post=1),
                dict(gate=(8 * P, 63, 0)), dict(gate=(8 * P, -64, 0)), dict(scale=(8 * P, 64, 2)),
                dict(shift=(8 * P + 8, 64, 0)), dict(gate=(8 * P, 1 << 60, 0)),
                dict(h=3 * P), dict(h=P + 1024), dict(xo=2 * P), dict(xo=P + 16), dict(h=2 * P + 64),
                dict(gate=(3 * P, 64, 0)), dict(shift=(4 * P, 64, 0)), dict(gain=4 * P), dict(post=1, post_gain=3 * P)):
        assert _fwd(**bad) == INV, bad
    assert _fwd(y=0, xo=0, alpha=0.5) == INV  # x' has to go somewhere
    assert vx.lib().vidax_block_norm_fwd(_p(P), None, None, _p(2 * P), 1, 1, 64, None, None) == INV
    for bad in (dict(C=12), dict(C=16392), dict(B=1 << 16, L=1 << 16)):
        assert _fwd(**bad) == UNS, bad


def test_backward_refusals():
    n = vx.lib().vidax_block_norm_bwd_workspace_floats(2, 8, 64)
    assert n > 0
    assert _bwd(B=0) == 0
    g = dict(grads={"dshift": 9 * P}, ws=10 * P, wn=n)
    for bad in (dict(dh=0), dict(xo=0), dict(dx=0), dict(dy=0), dict(y=0), dict(dh=P + 2), dict(ws=P + 4),
                dict(grads={"dgate": 9 * P}, y=0, dy=0), dict(grads={"dpost_gain": 9 * P}),
                dict(grads={"dshift": 9 * P}),                              # no workspace
                dict(grads={"dshift": 9 * P}, ws=10 * P, wn=n - 1),         # too small
                {**g, "grads": {"dshift": 9 * P + 4}}, {**g, "grads": {"dshift": 5 * P}},
                {**g, "grads": {"dshift": 9 * P, "dgain": 9 * P}}, {**g, "ws": 9 * P}, {**g, "ws": P},
                dict(dx=P), dict(dx=2 * P + 16), dict(dy=5 * P), dict(dy=4 * P), dict(scale=(8 * P, 64, 64)),
                dict(gate=(5 * P, 64, 0)), dict(eps=-1.0)):
        assert _bwd(**bad) == INV, bad
    assert vx.lib().vidax_block_norm_bwd(*[_p(P)] * 6, None, None, 0, 2, 8, 64, ctypes.byref(_desc()), None) == INV
    assert _bwd(C=20) == UNS
    f = vx.lib().vidax_block_norm_bwd_workspace_floats
    assert f(-1, 1, 64) == f(1, 1, 12) == f(1, 1, 32768) == f(1 << 16, 1 << 16, 64) == f(0, 5, 64) == 0


def test_workspace_covers_every_run():
    """Three sums a run of rows: runs times rows cover the tokens."""
    f = vx.lib().vidax_block_norm_bwd_workspace_floats
    for B, L, C in ((1, 1, 8), (1, 75600, 5120), (2, 16380, 1536), (700, 3, 1544), (1, 1 << 20, 16384), (513, 1, 64)):
        runs, rest = divmod(f(B, L, C), 3 * B * C)
        assert rest == 0 and 1 <= runs <= L, (B, L, C)
        assert B * runs <= max(512 + B, B), (B, L, C)


def test_binding_refuses_what_it_cannot_express():
    import torch

    x = torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device tensor"):
        vx.block_norm_fwd(x)
    with pytest.raises(ValueError, match="device tensor"):
        vx.block_norm_bwd(x, None, x)
