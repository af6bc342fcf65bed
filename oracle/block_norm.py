"""fp64 oracle for the norms before and after a block with gate and residual scale.

    Xn = a X + beta * gate * Npost(F),  H = Npre(Xn)

kind "none", "rms" or "layer"; gate None, [N] (a parameter) or [b, N].
"""
from __future__ import annotations

import numpy as np


def normalise(v, kind: str, eps: float):
    """(normalised rows, reciprocal roots [b, 1])."""
    if kind == "none":
        return v, np.ones((v.shape[0], 1))
    if kind == "layer":
        v = v - v.mean(axis=1, keepdims=True)
    r = 1.0 / np.sqrt(np.mean(v * v, axis=1, keepdims=True) + eps)
    return v * r, r


def norm(v, kind: str, w, b, eps: float):
    y, _ = normalise(v, kind, eps)
    y = y if w is None else y * w
    return y if b is None else y + b


def norm_vjp(v, kind: str, w, dn, eps: float):
    """Gradient with respect to v at the cotangent dn of the norm."""
    u = dn if w is None else dn * w
    if kind == "none":
        return u
    y, r = normalise(v, kind, eps)
    out = u - y * np.mean(u * y, axis=1, keepdims=True)
    if kind == "layer":
        out = out - np.mean(u, axis=1, keepdims=True)
    return r * out


def forward(X, F, post, post_w, post_b, gate, pre, pre_w, pre_b, eps, a, beta):
    """(Xn, H); H is None without a pre-norm, Xn is X where F is None."""
    Xn = X
    if F is not None:
        z = norm(F, post, post_w, post_b, eps)
        Xn = a * X + beta * (z if gate is None else gate * z)
    return Xn, None if pre == "none" else norm(Xn, pre, pre_w, pre_b, eps)


def backward(Xn, F, post, post_w, post_b, gate, pre, pre_w, dXn, dH, eps, a, beta):
    """Gradients by name: dX, dF, dgate, dpost_w, dpost_b, dpre_w, dpre_b (those that exist)."""
    T = np.zeros(Xn.shape) if dXn is None else np.array(dXn, np.float64)
    out = {}
    if pre != "none":
        dh = np.zeros(Xn.shape) if dH is None else dH
        T = T + norm_vjp(Xn, pre, pre_w, dh, eps)
        out["dpre_w"] = np.sum(dh * normalise(Xn, pre, eps)[0], axis=0)
        out["dpre_b"] = np.sum(dh, axis=0)
    if F is None:
        out["dX"] = T
        return out
    out["dX"] = a * T
    z = norm(F, post, post_w, post_b, eps)
    dz = beta * (T if gate is None else gate * T)
    if gate is not None:
        dg = beta * T * z
        out["dgate"] = dg.sum(axis=0) if gate.ndim == 1 else dg
    out["dF"] = norm_vjp(F, post, post_w, dz, eps)
    if post != "none":
        out["dpost_w"] = np.sum(dz * normalise(F, post, eps)[0], axis=0)
        out["dpost_b"] = np.sum(dz, axis=0)
    return out
