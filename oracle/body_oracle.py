"""fp64 CPU oracle for the operators of a student's body.

TEST INFRASTRUCTURE ONLY (same rules as kdkl_oracle.py: never imported by the product path, no code shared with the
CUDA path). Written from the definitions:

    record      for every 32 consecutive values of a row, e = the smallest integer with max|x| <= Q 2^e (Q = 127 for
                int8, 448 for e4m3), at least -126; x~ = 2^e round(x 2^-e), rounding to nearest even among the integers
                or among the e4m3 values; NaN throughout a group that holds something that is not finite
    gated       h = act(g) u, act(g) = g sigmoid(k(g)), k = g (silu) or 2 sqrt(2/pi) (g + 0.044715 g^3) (gelu)
    dweight     dW = dY^T x~
    block norm  n = b rho(b) (w1 + o), x = beta r + alpha gate n, y = x rho(x) (w2 + o), rho(v) = 1/sqrt(mean v^2 + eps);
                the gradient of <dy, y> + <dx, x>, evaluated at what was kept of b and x with the forward pass's rho.

All inputs are widened to float64. The forward functions return unrounded values; where a kernel rounds before it keeps
a tensor, the caller passes the rounded one.
"""
from __future__ import annotations

import numpy as np

Q = {"int8": 127.0, "e4m3": 448.0}
GROUP = 32


def record_exponents(x, fmt):
    """e [T, ceil(H / 32)] as integers."""
    x = np.asarray(x, dtype=np.float64)
    T, H = x.shape
    p = np.zeros((T, -(-H // GROUP) * GROUP))
    p[:, :H] = x
    top = np.abs(p.reshape(T, -1, GROUP)).max(axis=2)
    fine = np.isfinite(top)
    e = np.full(top.shape, -126, dtype=np.int64)
    need = fine & (top > Q[fmt] * 2.0 ** -126)
    guess = np.ceil(np.log2(top[need] / Q[fmt])).astype(np.int64)
    guess = np.where(top[need] > Q[fmt] * 2.0 ** guess, guess + 1, guess)           # log2 is not exact
    guess = np.where(top[need] <= Q[fmt] * 2.0 ** (guess - 1), guess - 1, guess)
    e[need] = np.maximum(guess, -126)
    return e, fine


def round_e4m3(q):
    """Nearest e4m3 value (ties to even) of |q| <= 448: 3 fraction bits above 2^-6, multiples of 2^-9 below."""
    a = np.maximum(np.abs(q), 2.0 ** -6)
    step = 2.0 ** (np.floor(np.log2(a)) - 3)
    return np.rint(q / step) * step


def record_values(x, fmt):
    """x~ [T, H]."""
    x = np.asarray(x, dtype=np.float64)
    T, H = x.shape
    e, fine = record_exponents(x, fmt)
    unit = np.repeat(2.0 ** e.astype(np.float64), GROUP, axis=1)[:, :H]
    fine = np.repeat(fine, GROUP, axis=1)[:, :H]
    q = np.where(fine, x, 0.0) / unit
    q = np.rint(q) if fmt == "int8" else round_e4m3(q)
    return np.where(fine, q * unit, np.nan)


def _sigmoid(k):
    return np.where(k >= 0, 1 / (1 + np.exp(-np.abs(k))), np.exp(-np.abs(k)) / (1 + np.exp(-np.abs(k))))


def _gate(g, act):
    if act == "silu":
        return _sigmoid(g), np.ones_like(g)
    c = 2 * np.sqrt(2 / np.pi)
    return _sigmoid(c * (g + 0.044715 * g ** 3)), c * (1 + 3 * 0.044715 * g ** 2)


def gated_forward(g, u, act):
    g, u = (np.asarray(v, dtype=np.float64) for v in (g, u))
    return g * _gate(g, act)[0] * u


def gated_backward(g, u, dh, act):
    g, u, dh = (np.asarray(v, dtype=np.float64) for v in (g, u, dh))
    s, slope = _gate(g, act)
    return dh * u * (s + g * s * (1 - s) * slope), dh * g * s


def dweight(dy, x):
    return np.asarray(dy, dtype=np.float64).T @ np.asarray(x, dtype=np.float64)


def _wide(gate, kind):
    if kind == "none":
        return 1.0
    gate = np.asarray(gate, dtype=np.float64)
    return gate[:, None] if kind == "token" else gate[None, :]


def norm_forward(r, b, w1=None, w2=None, gate=None, kind="none", eps=1e-6, offset=0.0, alpha=1.0, beta=1.0):
    """dict(x, y, rho1, rho2)."""
    r, b = (np.asarray(v, dtype=np.float64) for v in (r, b))
    T = b.shape[0]
    rho1, n = np.ones((T, 1)), b
    if w1 is not None:
        rho1 = 1 / np.sqrt((b * b).mean(axis=1, keepdims=True) + eps)
        n = b * rho1 * (np.asarray(w1, dtype=np.float64) + offset)
    x = beta * r + alpha * _wide(gate, kind) * n
    rho2, y = np.ones((T, 1)), None
    if w2 is not None:
        rho2 = 1 / np.sqrt((x * x).mean(axis=1, keepdims=True) + eps)
        y = x * rho2 * (np.asarray(w2, dtype=np.float64) + offset)
    return {"x": x, "y": y, "rho1": rho1, "rho2": rho2}


def norm_backward(dy, dx, b, x, rho1, rho2, w1=None, w2=None, gate=None, kind="none", offset=0.0, alpha=1.0, beta=1.0):
    """dict(dr, db, dw1, dw2, dgate) at the kept b and x."""
    b, x = (np.asarray(v, dtype=np.float64) for v in (b, x))
    T, H = b.shape
    d = np.zeros((T, H)) if dx is None else np.asarray(dx, dtype=np.float64).copy()
    out = {"dw1": None, "dw2": None, "dgate": None}
    if w2 is not None:
        dy = np.asarray(dy, dtype=np.float64)
        xh = x * rho2
        gy = dy * (np.asarray(w2, dtype=np.float64) + offset)
        out["dw2"] = (dy * xh).sum(axis=0)
        d = d + rho2 * (gy - xh * (gy * xh).mean(axis=1, keepdims=True))
    out["dr"] = beta * d
    bh = b * rho1
    w = 1.0 if w1 is None else np.asarray(w1, dtype=np.float64) + offset
    if kind != "none":
        out["dgate"] = (alpha * d * bh * w).sum(axis=1 if kind == "token" else 0)
    dn = alpha * _wide(gate, kind) * d
    if w1 is None:
        out["db"] = dn * np.ones((T, H))
    else:
        out["dw1"] = (dn * bh).sum(axis=0)
        gb = dn * w
        out["db"] = rho1 * (gb - bh * (gb * bh).mean(axis=1, keepdims=True))
    return out
