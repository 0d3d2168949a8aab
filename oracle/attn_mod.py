"""Reference of attention with score modifiers and of its gradient (float64,
definition).

For batch b, query head h, query i at position p_i = q_start[b] + i (by default
Lk - Lq + i) and key j of K/V head h // (H / Hkv):

    s_ij = scale * <q_i, k_j>
    s_ij = cap * tanh(s_ij / cap)                    where a cap is given
    s_ij = s_ij - slopes[h] * |p_i - j|              where slopes are given
    o_i  = sum_j softmax_j(s_ij) v_j   over the keys that i sees:
           j < kv_valid_len[b] (clamped to [0, Lk]; all without it),
           q_doc[b, i] == k_doc[b, j] >= 0           where documents are given,
           j <= p_i or j < prefix_len[b]             where causal.

A query that sees no key has o = 0, lse = -inf and passes no gradient.  The
paper masks attention by segment ids (porting-bug table, "Sharding, Parallelism
& Custom Kernels") and runs causal and full pathways side by side (Section 3);
it prints no formula.
"""

from __future__ import annotations

from dataclasses import dataclass

import numpy as np


@dataclass(frozen=True)
class ScoreSpec:
    causal: bool = False
    cap: float = 0.0
    slopes: object = None
    q_doc: object = None
    k_doc: object = None
    kv_valid_len: object = None
    prefix_len: object = None
    q_start: object = None


def positions(b, Lq, Lk, s: ScoreSpec):
    first = Lk - Lq if s.q_start is None else int(s.q_start[b])
    return first + np.arange(Lq)


def visible(b, Lq, Lk, s: ScoreSpec):
    """bool [Lq, Lk]: which keys every query of batch b sees."""
    j = np.arange(Lk)[None, :]
    see = np.ones((Lq, Lk), bool)
    if s.kv_valid_len is not None:
        see &= j < min(max(int(s.kv_valid_len[b]), 0), Lk)
    if s.q_doc is not None:
        qd, kd = np.asarray(s.q_doc[b])[:, None], np.asarray(s.k_doc[b])[None, :]
        see &= (qd == kd) & (kd >= 0)
    if s.causal:
        back = j <= positions(b, Lq, Lk, s)[:, None]
        if s.prefix_len is not None:
            back = back | (j < int(s.prefix_len[b]))
        see &= back
    return see


def scores(q, k, b, h, scale, s: ScoreSpec):
    """(modified scores with -inf where nothing is seen, tanh or None) of one head's q [Lq, d], k [Lk, d]."""
    x = scale * (q @ k.T)
    t = None
    if s.cap:
        t = np.tanh(x / s.cap)
        x = s.cap * t
    if s.slopes is not None:
        dist = np.abs(positions(b, len(q), len(k), s)[:, None] - np.arange(len(k))[None, :])
        x = x - float(s.slopes[h]) * dist
    return np.where(visible(b, len(q), len(k), s), x, -np.inf), t


def probabilities(x):
    """(softmax rows, lse); a row of -inf gives zeros and -inf."""
    m = x.max(1, initial=-np.inf)
    m0 = np.where(np.isneginf(m), 0.0, m)
    p = np.exp(x - m0[:, None])
    l = p.sum(1)
    with np.errstate(divide="ignore"):
        lse = m0 + np.log(l)
    return p / np.where(l > 0, l, 1.0)[:, None], lse


def attn_mod_ref(q, k, v, scale, s: ScoreSpec = ScoreSpec()):
    """(o [B, Lq, H, d], lse [B, H, Lq]) of q [B, Lq, H, d] and k, v [B, Lk, Hkv, d]."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    B, Lq, H, d = q.shape
    rep = H // k.shape[2]
    o, lse = np.zeros(q.shape), np.zeros((B, H, Lq))
    for b in range(B):
        for h in range(H):
            x, _ = scores(q[b, :, h], k[b, :, h // rep], b, h, scale, s)
            p, lse[b, h] = probabilities(x)
            o[b, :, h] = p @ v[b, :, h // rep]
    return o, lse


def attn_mod_bwd_ref(q, k, v, dout, scale, s: ScoreSpec = ScoreSpec(), o_saved=None):
    """(dq, dk, dv); o_saved: the output D is formed from (as a forward left it)."""
    q, k, v, dout = (np.asarray(x, np.float64) for x in (q, k, v, dout))
    B, Lq, H, d = q.shape
    rep = H // k.shape[2]
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for b in range(B):
        for h in range(H):
            qh, kh, vh, gh = q[b, :, h], k[b, :, h // rep], v[b, :, h // rep], dout[b, :, h]
            x, t = scores(qh, kh, b, h, scale, s)
            p, _ = probabilities(x)
            oh = p @ vh if o_saved is None else np.asarray(o_saved, np.float64)[b, :, h]
            ds = p * (gh @ vh.T - (gh * oh).sum(1)[:, None])
            if t is not None:
                ds = ds * (1.0 - t * t)
            dq[b, :, h] = scale * (ds @ kh)
            dk[b, :, h // rep] += scale * (ds.T @ qh)
            dv[b, :, h // rep] += p.T @ gh
    return dq, dk, dv
