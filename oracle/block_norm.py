"""The norms around a block with its gate, residual scale and residual sum, and their gradients, in float64.

    out = x_scale * x + y_scale * gate * N_post(y);   h = N_pre(out)
    N(v) = (v - mu) / sqrt(mean((v - mu)^2) + eps) * (w + offset) + b,   mu = 0 ("rms") or mean(v) ("layer")

Beside every result goes its scale: the sum of the magnitudes of the terms it is made of, which is what an error of
float32 arithmetic is relative to (a difference of large terms has the error of the terms, not of the difference).
"""
from __future__ import annotations

import numpy as np


def _moments(v, kind, eps):
    mu = v.mean(axis=1, keepdims=True) if kind == "layer" else np.zeros((v.shape[0], 1))
    r = 1.0 / np.sqrt(((v - mu) ** 2).mean(axis=1, keepdims=True) + eps)
    return mu, r


def _weight(w, offset, d):
    return np.ones(d) if w is None else w + offset


def norm(v, kind, eps, w=None, b=None, offset=0.0):
    """-> N(v) and its scale."""
    if kind is None:
        return v, np.abs(v)
    d = v.shape[1]
    mu, r = _moments(v, kind, eps)
    weight, bias = _weight(w, offset, d), np.zeros(d) if b is None else b
    return (v - mu) * r * weight + bias, (np.abs(v) + np.abs(mu)) * r * np.abs(weight) + np.abs(bias)


def norm_gradient(v, dv, kind, eps, w=None, offset=0.0):
    """dv = gradient of N(v) -> gradient of v, of w and of b (the last two per token), each with its scale."""
    if kind is None:
        return (dv, np.abs(dv)), None, None
    mu, r = _moments(v, kind, eps)
    weight = _weight(w, offset, v.shape[1])
    hat, hat_s = (v - mu) * r, (np.abs(v) + np.abs(mu)) * r
    q, q_s = dv * weight, np.abs(dv * weight)
    g = q - hat * (q * hat).mean(axis=1, keepdims=True)
    g_s = q_s + hat_s * (q_s * hat_s).mean(axis=1, keepdims=True)
    if kind == "layer":
        g = g - q.mean(axis=1, keepdims=True)
        g_s = g_s + q_s.mean(axis=1, keepdims=True)
    return (r * g, r * g_s), (dv * hat, np.abs(dv) * hat_s), (dv, np.abs(dv))


def _gate(gate, kind):
    if kind is None:
        return 1.0
    return gate.reshape(-1, 1) if kind == "token" else gate


def stream(x, y, cfg, p):
    """out and its scale.  cfg: post, pre, gate, x_scale, y_scale, post_eps, pre_eps, offset; p: parameters by name."""
    z, z_s = norm(y, cfg["post"], cfg["post_eps"], p.get("post_weight"), p.get("post_bias"), cfg["offset"])
    g = cfg["y_scale"] * _gate(p.get("gate"), cfg["gate"])
    return cfg["x_scale"] * x + g * z, np.abs(cfg["x_scale"] * x) + np.abs(g) * z_s


def pre_norm(out, cfg, p):
    """h and its scale."""
    return norm(out, cfg["pre"], cfg["pre_eps"], p.get("pre_weight"), p.get("pre_bias"), cfg["offset"])


def gradients(out, y, dout, dh, cfg, p):
    """dict name -> (gradient, scale): dx, dy, dgate, dpost_weight, dpost_bias, dpre_weight, dpre_bias.  y = None: the pre norm alone,
    h = N_pre(x) and out = x, in which x_scale has no part."""
    res = {}
    D = np.zeros_like(out) if dout is None else dout
    D_s = np.abs(D)
    if cfg["pre"]:
        (g, g_s), dw, db = norm_gradient(out, dh, cfg["pre"], cfg["pre_eps"], p.get("pre_weight"), cfg["offset"])
        D, D_s = D + g, D_s + g_s
        if "pre_weight" in p:
            res["dpre_weight"] = tuple(a.sum(axis=0) for a in dw)
        if "pre_bias" in p:
            res["dpre_bias"] = tuple(a.sum(axis=0) for a in db)
    if y is None:
        res["dx"] = (D, D_s)
        return res
    res["dx"] = (cfg["x_scale"] * D, np.abs(cfg["x_scale"]) * D_s)
    z, z_s = norm(y, cfg["post"], cfg["post_eps"], p.get("post_weight"), p.get("post_bias"), cfg["offset"])
    ys = cfg["y_scale"]
    if cfg["gate"]:
        full = (ys * z * D, np.abs(ys) * z_s * D_s)
        res["dgate"] = full if cfg["gate"] == "element" else tuple(a.sum(axis=0 if cfg["gate"] == "channel" else 1) for a in full)
    g = _gate(p.get("gate"), cfg["gate"])
    dz, dz_s = ys * g * D, np.abs(ys * g) * D_s
    if not cfg["post"]:
        res["dy"] = (dz, dz_s)
        return res
    (dy, _), dw, db = norm_gradient(y, dz, cfg["post"], cfg["post_eps"], p.get("post_weight"), cfg["offset"])
    # the same sums of magnitudes, from the scale of dz
    (_, dy_s), (_, dw_s), (_, db_s) = norm_gradient(y, dz_s, cfg["post"], cfg["post_eps"], p.get("post_weight"), cfg["offset"])
    res["dy"] = (dy, dy_s)
    if "post_weight" in p:
        res["dpost_weight"] = (dw[0].sum(axis=0), dw_s.sum(axis=0))
    if "post_bias" in p:
        res["dpost_bias"] = (db[0].sum(axis=0), db_s.sum(axis=0))
    return res
