"""fp64 CPU oracle of the operators around the memory layer (test infrastructure only): the norms
before and after a block with its gate and residual scale, their backward, the global gradient norm
with clipping, and low-rank adapters.

Written from the definitions, one function per step, in numpy float64.  Shares nothing with the HIP
path.
"""
from __future__ import annotations

import numpy as np


def standardise(x, kind, eps):
    """(x^, 1 / spread) per row: LayerNorm's centred rows, or RMS."""
    x = np.asarray(x, dtype=np.float64)
    mean = x.mean(axis=1, keepdims=True) if kind == "layer" else 0.0
    with np.errstate(divide="ignore", invalid="ignore"):
        r = 1.0 / np.sqrt(np.square(x - mean).mean(axis=1, keepdims=True) + eps)
        return (x - mean) * r, r


def affine(xh, gamma, beta):
    out = xh * np.asarray(gamma, dtype=np.float64)
    return out if beta is None else out + np.asarray(beta, dtype=np.float64)


def block_in(h, kind, gamma, beta, eps):
    return affine(standardise(h, kind, eps)[0], gamma, beta)


def gate_value(gate, kind, act, T, d):
    """(value, slope) of the gate, each spread over [T, d]."""
    if kind == "none":
        return np.ones((T, d)), np.zeros((T, d))
    z = np.asarray(gate, dtype=np.float64)
    z = np.broadcast_to({"channel": z.reshape(1, -1), "token": z.reshape(-1, 1), "full": z}[kind], (T, d))
    if act == "linear":
        return z, np.ones((T, d))
    v = 1.0 / (1.0 + np.exp(-z))
    return v, v * (1.0 - v)


def exit_norm(y, kind, gamma, beta, eps):
    if kind == "none":
        return np.asarray(y, dtype=np.float64)
    return affine(standardise(y, kind, eps)[0], gamma, beta)


def block_out(h, y, gate, gate_kind, act, kind, gamma, beta, eps, res_scale, out_scale):
    T, d = np.shape(y)
    value, _ = gate_value(gate, gate_kind, act, T, d)
    return res_scale * np.asarray(h, dtype=np.float64) + out_scale * value * exit_norm(y, kind, gamma, beta, eps)


def norm_backward(x, kind, gamma, eps, dn):
    """(dx, dgamma, dbeta) of Norm(x) from the gradient dn of its output."""
    dn = np.asarray(dn, dtype=np.float64)
    xh, r = standardise(x, kind, eps)
    v = dn * np.asarray(gamma, dtype=np.float64)
    dx = v - xh * (v * xh).mean(axis=1, keepdims=True)
    if kind == "layer":
        dx = dx - v.mean(axis=1, keepdims=True)
    return r * dx, (dn * xh).sum(axis=0), dn.sum(axis=0)


def block_in_backward(h, kind, gamma, eps, dn, dres):
    dx, dg, db = norm_backward(h, kind, gamma, eps, dn)
    return (dx if dres is None else dx + np.asarray(dres, dtype=np.float64)), dg, db


def block_out_backward(y, gate, gate_kind, act, kind, gamma, beta, eps, res_scale, out_scale, dh_out):
    """dict of dh, dy, dgate (None without a gate), dgamma, dbeta (None without a norm)."""
    T, d = np.shape(y)
    up = np.asarray(dh_out, dtype=np.float64)
    value, slope = gate_value(gate, gate_kind, act, T, d)
    dgate = out_scale * up * exit_norm(y, kind, gamma, beta, eps) * slope
    dm = out_scale * up * value
    out = {"dh": res_scale * up, "dy": dm, "dgamma": None, "dbeta": None,
           "dgate": {"none": None, "channel": dgate.sum(axis=0), "token": dgate.sum(axis=1), "full": dgate}[gate_kind]}
    if kind != "none":
        out["dy"], out["dgamma"], out["dbeta"] = norm_backward(y, kind, gamma, eps, dm)
    return out


def global_norm(grads):
    with np.errstate(over="ignore", invalid="ignore"):
        return float(np.sqrt(sum(float(np.square(np.asarray(g, dtype=np.float64)).sum()) for g in grads)))


def clip_factor(norm, max_norm):
    return 1.0 if norm <= max_norm else max_norm / norm


def adapter_add(x, ids, a, b, scale, base):
    """base[t] + scale[i] B_i (A_i x[t]); a [n, r, d_in], b [n, d_out, r], ids outside [0, n): base[t]."""
    x, a, b = (np.asarray(v, dtype=np.float64) for v in (x, a, b))
    out = np.zeros((len(x), b.shape[1])) if base is None else np.array(base, dtype=np.float64)
    for t, i in enumerate(ids):
        if 0 <= i < len(a):
            out[t] += (1.0 if scale is None else float(scale[i])) * (b[i] @ (a[i] @ x[t]))
    return out
