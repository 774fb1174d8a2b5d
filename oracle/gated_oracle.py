"""Gated linear recurrence (include/ssm_gated.h) in float64, step by step: the definition the kernels are checked against.

Inputs are numpy arrays: x, gate, in_gate (batch, L, D), A (D,), reset (batch, L) of truth values, h0 (batch, D)."""
from __future__ import annotations

import numpy as np


def _sigma(z):
    """sigma(z) and 1 - sigma(z), each without cancellation."""
    e = np.exp(-np.abs(z))
    small, large = e / (1.0 + e), 1.0 / (1.0 + e)
    return np.where(z >= 0, large, small), np.where(z >= 0, small, large)


def _gates(x, gate, in_gate, A):
    g, og = _sigma(gate)
    if A is None:
        return og, g * x, (g, og)
    iota, oi = _sigma(in_gate)
    la = g * A
    beta = np.sqrt(-np.expm1(2.0 * la))
    return np.exp(la), beta * iota * x, (g, og, iota, oi, beta)


def _double(*arrays):
    return [None if v is None else np.asarray(v, dtype=np.float64) for v in arrays]


def gated_fwd(x, gate, in_gate=None, A=None, reset=None, h0=None):
    """(y, h_last): y (batch, L, D), h_last (batch, D)."""
    x, gate, in_gate, A, h0 = _double(x, gate, in_gate, A, h0)
    batch, L, D = x.shape
    a, u, _ = _gates(x, gate, in_gate, A)
    h = np.zeros((batch, D)) if h0 is None else h0
    y = np.empty_like(x)
    for t in range(L):
        kept = a[:, t] * h
        if reset is not None:
            kept = np.where(np.asarray(reset)[:, t, None] != 0, 0.0, kept)
        h = kept + u[:, t]
        y[:, t] = h
    return y, h


def gated_bwd(x, gate, in_gate, A, dy, reset=None, h0=None, dh_last=None):
    """dict of dx, dgate, din_gate, dA, dh0 (din_gate and dA None without A), and dA_terms = sum of |terms| of dA."""
    x, gate, in_gate, A, h0, dy, dh_last = _double(x, gate, in_gate, A, h0, dy, dh_last)
    batch, L, D = x.shape
    y, _ = gated_fwd(x, gate, in_gate, A, reset, h0)
    a, _, parts = _gates(x, gate, in_gate, A)
    out = {"dx": np.empty_like(x), "dgate": np.empty_like(x), "din_gate": None, "dA": None, "dA_terms": None}
    if A is not None:
        out["din_gate"], out["dA"], out["dA_terms"] = np.empty_like(x), np.zeros(D), np.zeros(D)
    carry = np.zeros((batch, D)) if dh_last is None else dh_last
    first = np.zeros((batch, D)) if h0 is None else h0
    for t in reversed(range(L)):
        cut = np.zeros((batch, 1), bool) if reset is None else np.asarray(reset)[:, t, None] != 0
        prev = np.where(cut, 0.0, y[:, t - 1] if t else first)
        mu = dy[:, t] + carry
        if A is None:
            g, og = (v[:, t] for v in parts)
            out["dx"][:, t] = mu * g
            out["dgate"][:, t] = mu * (x[:, t] - prev) * g * og
        else:
            g, og, iota, oi, beta = (v[:, t] for v in parts)
            out["dx"][:, t] = mu * beta * iota
            out["din_gate"][:, t] = mu * beta * x[:, t] * iota * oi
            # d u / d a = -a / beta iota x; where beta is 0, rho is too, and its gradient goes to 0 with it
            slope = np.divide(a[:, t], beta, out=np.zeros_like(beta), where=beta > 0)
            m = mu * a[:, t] * (prev - slope * iota * x[:, t])
            out["dgate"][:, t] = m * A * g * og
            out["dA"] += (m * g).sum(0)
            out["dA_terms"] += np.abs(m * g).sum(0)
        carry = np.where(cut, 0.0, a[:, t] * mu)
    out["dh0"] = carry
    return out
