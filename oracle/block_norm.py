"""Reference of the step between two sublayers (float64, definition).

Per token, over the C channels of a residual stream x and a branch y:

    u  = post(y) * post_gain
    x' = alpha * x + gate * u
    h  = norm(x') * gain * (1 + scale) + shift

with layer norm (v - mean) / sqrt(mean((v - mean)^2) + eps) or RMS norm
v / sqrt(mean(v^2) + eps).  The paper names adaptive layer norm per sample and
per token (Section 3) without formulas; these are the standard ones.
"""

from __future__ import annotations

import numpy as np


def _rows(m, like):
    """A modulation [B, C], [B, 1, C] or [B, L, C] (or None) against [B, L, C]."""
    if m is None:
        return None
    m = np.asarray(m, np.float64)
    return m[:, None, :] if m.ndim == 2 else m


def normalise(v, kind, eps):
    """(normalised rows, 1 / root) of v [..., C]; kind "layer" or "rms"."""
    v = np.asarray(v, np.float64)
    if kind == "layer":
        v = v - v.mean(-1, keepdims=True)
    elif kind != "rms":
        raise ValueError(kind)
    r = 1.0 / np.sqrt((v * v).mean(-1, keepdims=True) + eps)
    return v * r, r


def block_norm_ref(x, y=None, gate=None, scale=None, shift=None, gain=None, post_gain=None, norm="layer", post=None,
                   eps=1e-6, alpha=1.0):
    """(x', h) in float64."""
    xo = alpha * np.asarray(x, np.float64)
    if y is not None:
        u = np.asarray(y, np.float64) if post is None else normalise(y, post, eps)[0]
        if post_gain is not None:
            u = u * post_gain
        g = _rows(gate, x)
        xo = xo + (u if g is None else g * u)
    h = normalise(xo, norm, eps)[0]
    if gain is not None:
        h = h * gain
    if scale is not None:
        h = h * (1.0 + _rows(scale, x))
    if shift is not None:
        h = h + _rows(shift, x)
    return xo, h


def _normalise_grad(d, hat, r, kind):
    """Gradient through normalise(): d is the gradient of hat."""
    out = d - hat * (d * hat).mean(-1, keepdims=True)
    if kind == "layer":
        out = out - d.mean(-1, keepdims=True)
    return out * r


def _like(m, g):
    """g [B, L, C] summed to the shape of the modulation m."""
    m = np.asarray(m)
    if m.ndim == 3 and m.shape[1] == g.shape[1]:
        return g
    g = g.sum(1)
    return g if m.ndim == 2 else g[:, None, :]


def block_norm_bwd_ref(dh, dxo, xo, y=None, gate=None, scale=None, shift=None, gain=None, post_gain=None,
                       norm="layer", post=None, eps=1e-6, alpha=1.0):
    """Gradients at the stream x' = xo, for gradients dh of h and dxo (or None)
    of x', as a dict with the entries of the operands given."""
    dh = np.asarray(dh, np.float64)
    hat, r = normalise(xo, norm, eps)
    mul = np.ones(dh.shape[-1]) if gain is None else np.asarray(gain, np.float64)
    s1 = 1.0 if scale is None else 1.0 + _rows(scale, dh)
    g = _normalise_grad(dh * mul * s1, hat, r, norm)
    if dxo is not None:
        g = g + np.asarray(dxo, np.float64)
    out = {"dx": alpha * g}
    if scale is not None:
        out["dscale"] = _like(scale, dh * hat * mul)
    if shift is not None:
        out["dshift"] = _like(shift, dh)
    if gain is not None:
        out["dgain"] = (dh * hat * s1).sum((0, 1))
    if y is not None:
        yh, ry = (np.asarray(y, np.float64), None) if post is None else normalise(y, post, eps)
        pg = np.ones(dh.shape[-1]) if post_gain is None else np.asarray(post_gain, np.float64)
        if gate is not None:
            out["dgate"] = _like(gate, g * yh * pg)
        du = g if gate is None else g * _rows(gate, dh)
        if post_gain is not None:
            out["dpost_gain"] = (du * yh).sum((0, 1))
        out["dy"] = du * pg if post is None else _normalise_grad(du * pg, yh, ry, post)
    return out
