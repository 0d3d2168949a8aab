"""Attention with score modifiers, forward and backward, on more batches than a wave
has lanes: prefixes, valid lengths and positions of their own in each.  Checked on
some batches and heads against the float64 reference, within the bounds derived in
tests/test_gpu_attn_mod.py and tests/test_gpu_attn_mod_bwd.py."""

import pytest

import oracle
import paper_2609_18077_amd as vx
from tests.test_gpu_attn_mod import SCALE, compare, dev_score, make
from tests.test_gpu_attn_mod_bwd import compare as compare_grads

pytestmark = pytest.mark.gpu


def _own(B, Lq, Lk, what):
    """A length, prefix or position for every batch."""
    s = {"causal": True}
    if "prefix" in what:
        s["prefix_len"] = [(37 * b) % (Lk + 20) for b in range(B)]
    if "valid" in what:
        s["kv_valid_len"] = [Lk - (29 * b) % Lk for b in range(B)]
    if "start" in what:
        s["q_start"] = [Lk - Lq - (11 * b) % 200 for b in range(B)]
    return s


@pytest.mark.parametrize("B,H,Hkv,Lq,Lk", [(64, 32, 8, 600, 600), (65, 32, 8, 600, 600), (130, 4, 1, 270, 330)])
@pytest.mark.parametrize("what", ["prefix", "valid", "prefix+valid+start"])
def test_batches_with_lengths_of_their_own(B, H, Hkv, Lq, Lk, what):
    import torch

    q, k, v = make(B, H, Hkv, Lq, Lk, 51)
    dout = make(B, H, Hkv, Lq, 1, 52)[0]
    s = _own(B, Lq, Lk, what)
    score, _ = dev_score(**s)
    # (a workspace of NaN: what a launch reads it has written)
    floats = vx.lib().vidax_attn_mod_fwd_workspace_floats(B, H, Hkv, Lq, Lk, 128, 0)
    ws = torch.full((max(floats, 4),), float("nan"), device="cuda")
    out = torch.full_like(q, float("nan"))
    o, lse = vx.attn_mod_fwd(q, k, v, score, return_lse=True, out=out, workspace=ws)
    grads = vx.attn_mod_bwd(q, k, v, o, dout, lse, score)
    rep = H // Hkv
    for b in (0, 31, 63, B - 1):
        g = b % Hkv
        bs, hs, ks = slice(b, b + 1), slice(g * rep, g * rep + rep), slice(g, g + 1)
        spec = oracle.ScoreSpec(**{n: x[b:b + 1] if isinstance(x, list) else x for n, x in s.items()})
        args = q[bs, :, hs], k[bs, :, ks], v[bs, :, ks], SCALE, spec, f"{what} batch {b} of {B}"
        compare(o[bs, :, hs], lse[bs, hs], *args)
        compare_grads([grads[0][bs, :, hs], grads[1][bs, :, ks], grads[2][bs, :, ks]], o[bs, :, hs], dout[bs, :, hs], *args)
    for t in (o, *grads):
        assert torch.isfinite(t).all()


@pytest.mark.parametrize("B,H,Hkv,Lq,Lk", [(32000, 33, 1, 1, 20), (40000, 16, 16, 2, 2), (20000, 33, 1, 1, 33)])
def test_a_million_tiles(B, H, Hkv, Lq, Lk):
    """Short sequences by the thousand: more tiles than a launch that joins pieces of them could hold."""
    import torch

    q, k, v = make(B, H, Hkv, Lq, Lk, 53)
    dout = make(B, H, Hkv, Lq, 1, 54)[0]
    score = vx.Score(causal=True)
    o, lse = vx.attn_mod_fwd(q, k, v, score, return_lse=True)
    grads = vx.attn_mod_bwd(q, k, v, o, dout, lse, score)
    for b in (0, B // 2, B - 2):
        bs = slice(b, b + 2)
        args = q[bs], k[bs], v[bs], SCALE, oracle.ScoreSpec(causal=True), f"batch {b} of {B}"
        compare(o[bs], lse[bs], *args)
        compare_grads([t[bs] for t in grads], o[bs], dout[bs], *args)
    for t in (o, *grads):
        assert torch.isfinite(t).all()
