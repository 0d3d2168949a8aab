"""What the header of attention with score modifiers says of outputs that are cut
differently, with and without log-sum-exps, and of keys that no query may see where
the scores are capped.

Tolerance: two outputs that are each within e = 2^-8 / (1 - 2^-8) (M + |o|) and a
rounding to bf16, 2^-8 (|o| + e), of the exact value, M = sum_j p_j |v_j|, differ by
at most the sum of their distances; M and o are taken from such outputs themselves,
which the factor 1 + 2^-6 covers, as it does fp32 rounding (128 * 2^-24 of the
scores' terms, here below 2^-10 of M).
"""

import pytest

import paper_2609_18077_amd as vx
from tests.test_gpu_attn_mod import D, dev_score, make, masks

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8


def _apart(a, b, q, k, v, score):
    """The largest distance of a and b over its bound."""
    import torch

    m = vx.attn_mod_fwd(q, k, v.abs(), score).double()
    size = torch.maximum(a.double().abs(), b.double().abs())
    e = HALF / (1 - HALF) * (m + size)
    tol = 2 * (1 + 2.0 ** -6) * (e + HALF * (size + e))
    assert torch.isfinite(a).all() and torch.isfinite(b).all()
    return float(((a.double() - b.double()).abs() / tol.clamp_min(1e-30)).max())


@pytest.mark.parametrize("B,H,Hkv,Lq,Lk", [(2, 4, 1, 3, 2100), (1, 4, 2, 300, 2000), (2, 16, 4, 532, 2375)])
@pytest.mark.parametrize("s", [{}, {"causal": True, "cap": 5.0}, {"slopes": 0.001}], ids=["plain", "cap", "bias"])
def test_other_workspaces_and_log_sum_exps(B, H, Hkv, Lq, Lk, s):
    import torch

    s = dict(s, slopes=[s["slopes"] * (h + 1) for h in range(H)]) if "slopes" in s else s
    score, _ = dev_score(**s)
    q, k, v = make(B, H, Hkv, Lq, Lk, 61)
    full = vx.lib().vidax_attn_mod_fwd_workspace_floats(B, H, Hkv, Lq, Lk, D, 0)
    outs = []
    for floats in (0, full // 3, full):
        ws = torch.empty(max(floats, 4), device="cuda")[:floats] if floats else torch.empty(0, device="cuda")
        outs.append(vx.attn_mod_fwd(q, k, v, score, workspace=ws))
        o, _ = vx.attn_mod_fwd(q, k, v, score, workspace=ws, return_lse=True)
        outs.append(o)
        assert torch.equal(outs[-2], vx.attn_mod_fwd(q, k, v, score, workspace=ws))
    for o in outs[1:]:
        assert _apart(outs[0], o, q, k, v, score) <= 1


@pytest.mark.parametrize("Lq", [1, 70, 300])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), 3e38])
def test_unseen_keys_with_a_cap(bad, Lq):
    import torch

    B, H, Lk = 2, 4, 500
    q, k, v = make(B, H, 2, Lq, Lk, 62, mul=4.0)
    for s, hidden in (({"kv_valid_len": [201, 64]}, [(0, 201, 500), (1, 64, 500)]),
                      ({"causal": True, "q_start": [130, 0], "prefix_len": [7, 400]},
                       [(0, 130 + Lq, 500), (1, max(Lq, 400), 500)]),
                      ({"q_doc": torch.zeros(B, Lq), "k_doc": masks("docs_any_order", B, Lq, Lk)["k_doc"].clip(-1, 0)}, None)):
        score, _ = dev_score(cap=6.0, **s)
        k2, v2 = k.clone(), v.clone()
        if hidden is None:
            k2[score.k_doc < 0], v2[score.k_doc < 0] = bad, -bad
        else:
            for b, i, j in hidden:
                k2[b, i:j], v2[b, i:j] = bad, -bad
        got, want = vx.attn_mod_fwd(q, k2, v2, score), vx.attn_mod_fwd(q, k, v, score)
        assert _apart(got, want, q, k, v, score) <= 1, list(s)
