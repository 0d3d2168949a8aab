"""The float64 references of the block norm and of attention with score
modifiers: gradients against central differences, and identities that do not
repeat the references' own formulas."""

import math

import numpy as np
import pytest

import oracle
from oracle import attn_mod


def _central(f, x, h=1e-5):
    g = np.zeros_like(x)
    it = np.nditer(x, flags=["multi_index"])
    for _ in it:
        i = it.multi_index
        y = x.copy()
        y[i] += h
        up = f(y)
        y[i] -= 2 * h
        g[i] = (up - f(y)) / (2 * h)
    return g


@pytest.mark.parametrize("norm,post,token", [("layer", None, False), ("rms", "rms", False), ("layer", "layer", True),
                                             ("rms", None, True)])
def test_block_norm_gradients_are_the_differences(norm, post, token):
    rng = np.random.default_rng(5)
    B, L, C = 2, 3, 8
    m = (B, L, C) if token else (B, C)
    a = {"x": rng.normal(size=(B, L, C)), "y": rng.normal(size=(B, L, C)), "gate": rng.normal(size=m),
         "scale": rng.normal(size=m), "shift": rng.normal(size=m), "gain": rng.normal(size=C)}
    if post:
        a["post_gain"] = rng.normal(size=C)
    dh, dxo = rng.normal(size=(B, L, C)), rng.normal(size=(B, L, C))
    kw = dict(norm=norm, post=post, eps=1e-3, alpha=0.7)

    def loss(**over):
        xo, h = oracle.block_norm_ref(**{**a, **over}, **kw)
        return float((xo * dxo).sum() + (h * dh).sum())

    xo, _ = oracle.block_norm_ref(**a, **kw)
    got = oracle.block_norm_bwd_ref(dh, dxo, xo, **{n: z for n, z in a.items() if n != "x"}, **kw)
    assert set(got) == {"d" + n for n in a}
    for n, z in a.items():
        # central differences: truncation h^2 f''' / 6 and cancellation 2^-53 |f| / h, both below 1e-8
        np.testing.assert_allclose(got["d" + n], _central(lambda v: loss(**{n: v}), z), atol=1e-6, err_msg=n)


def test_block_norm_by_hand():
    xo, h = oracle.block_norm_ref([[[1.0, 3.0]]], [[[2.0, -2.0]]], gate=[[0.5, 1.0]], scale=[[1.0, 0.0]],
                                  shift=[[0.25, -1.0]], norm="layer", eps=0.0)
    assert xo.tolist() == [[[2.0, 1.0]]]  # hat = (1, -1)
    assert h.tolist() == [[[2.25, -2.0]]]


def _case(rng, Lq=5, Lk=7, H=4, Hkv=2, d=6, B=2):
    return tuple(rng.normal(size=s) for s in ((B, Lq, H, d), (B, Lk, Hkv, d), (B, Lk, Hkv, d), (B, Lq, H, d)))


SPECS = [
    oracle.ScoreSpec(),
    oracle.ScoreSpec(causal=True, cap=1.5),
    oracle.ScoreSpec(causal=True, prefix_len=[3, 0], slopes=[0.3, -0.1, 0.0, 1.0], q_start=[0, -2]),
    oracle.ScoreSpec(q_doc=[[0, 0, 1, 5, -1], [2, 0, 2, 0, 2]], k_doc=[[0, 1, 0, -1, 1, 4, 0], [0, 2, 1, 2, 0, 0, -1]],
                     cap=0.7, kv_valid_len=[6, 99]),
]


@pytest.mark.parametrize("spec", SPECS, ids=["plain", "causal_cap", "prefix_bias", "docs_cap"])
def test_attention_gradients_are_the_differences(spec):
    q, k, v, g = _case(np.random.default_rng(6))
    loss = lambda q, k, v: float((oracle.attn_mod_ref(q, k, v, 0.4, spec)[0] * g).sum())
    got = oracle.attn_mod_bwd_ref(q, k, v, g, 0.4, spec)
    for n, d in zip("qkv", got):
        a = {"q": q, "k": k, "v": v}
        np.testing.assert_allclose(d, _central(lambda z: loss(**{**a, n: z}), a[n]), atol=1e-6, err_msg=n)


@pytest.mark.parametrize("spec", SPECS, ids=["plain", "causal_cap", "prefix_bias", "docs_cap"])
def test_attention_is_the_sum_over_the_seen_keys(spec):
    """Key by key in plain Python, visibility spelled out."""
    q, k, v, _ = _case(np.random.default_rng(7))
    o, lse = oracle.attn_mod_ref(q, k, v, 0.4, spec)
    B, Lq, H, d = q.shape
    Lk, rep = k.shape[1], H // k.shape[2]
    for b in range(B):
        for h in range(H):
            for i in range(Lq):
                p = i + (Lk - Lq if spec.q_start is None else spec.q_start[b])
                seen = []
                for j in range(Lk):
                    if spec.kv_valid_len is not None and j >= spec.kv_valid_len[b]:
                        continue
                    if spec.q_doc is not None and (spec.q_doc[b][i] != spec.k_doc[b][j] or spec.q_doc[b][i] < 0):
                        continue
                    if spec.causal and j > p and not (spec.prefix_len is not None and j < spec.prefix_len[b]):
                        continue
                    s = 0.4 * math.fsum(q[b, i, h] * k[b, j, h // rep])
                    if spec.cap:
                        s = spec.cap * math.tanh(s / spec.cap)
                    if spec.slopes is not None:
                        s -= spec.slopes[h] * abs(p - j)
                    seen.append((s, v[b, j, h // rep]))
                if not seen:
                    assert not o[b, i, h].any() and lse[b, h, i] == -math.inf
                    continue
                z = math.fsum(math.exp(s) for s, _ in seen)
                want = sum(math.exp(s) / z * x for s, x in seen)
                np.testing.assert_allclose(o[b, i, h], want, rtol=1e-12, atol=1e-13)
                assert abs(lse[b, h, i] - math.log(z)) < 1e-12


def test_attention_without_modifiers_is_the_plain_one():
    rng = np.random.default_rng(8)
    q, k, v = (rng.normal(size=s) for s in ((2, 5, 3, 128), (2, 9, 3, 128), (2, 9, 3, 128)))
    spec = oracle.ScoreSpec(kv_valid_len=[9, 4])
    o, lse = oracle.attn_mod_ref(q, k, v, 0.1, spec)
    ro, rl = oracle.attn_ref(q, k, v, 0.1, kv_valid_len=np.array([9, 4]))
    np.testing.assert_allclose(o, ro, atol=1e-13)
    np.testing.assert_allclose(lse, rl, atol=1e-13)


def test_a_large_cap_is_none_and_documents_cut_into_calls():
    rng = np.random.default_rng(9)
    q, k, v, g = _case(rng, Lq=7, Lk=7, B=1)
    a = oracle.attn_mod_ref(q, k, v, 0.4, oracle.ScoreSpec(cap=1e9))[0]
    np.testing.assert_allclose(a, oracle.attn_mod_ref(q, k, v, 0.4)[0], atol=1e-12)
    doc = [[0, 0, 0, 1, 1, 1, 1]]
    whole = oracle.attn_mod_bwd_ref(q, k, v, g, 0.4, oracle.ScoreSpec(q_doc=doc, k_doc=doc, causal=True))
    for cut in (slice(0, 3), slice(3, 7)):
        part = oracle.attn_mod_bwd_ref(*(x[:, cut] for x in (q, k, v, g)), 0.4, oracle.ScoreSpec(causal=True))
        for x, y in zip(whole, part):
            np.testing.assert_allclose(x[:, cut], y, atol=1e-12)
    assert attn_mod.visible(0, 2, 2, oracle.ScoreSpec(causal=True, q_start=[-1])).tolist() == [[False, False],
                                                                                              [True, False]]
