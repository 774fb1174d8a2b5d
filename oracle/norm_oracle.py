"""Norm of rows (include/ssm_norm.h) in float64: the definition the kernels are checked against.  s: (rows, D), the sum that
the norm is of."""
from __future__ import annotations

import numpy as np


def _stats(s, rms, eps):
    m = np.zeros(s.shape[0]) if rms else s.mean(1)
    return m, 1.0 / np.sqrt(((s - m[:, None]) ** 2).mean(1) + eps)


def norm_fwd(s, weight, bias=None, rms=False, eps=1e-5):
    """(y, stats): stats (rows, 2) of mean (0 with rms) and reciprocal deviation."""
    s, weight = np.asarray(s, np.float64), np.asarray(weight, np.float64)
    m, r = _stats(s, rms, eps)
    y = (s - m[:, None]) * r[:, None] * weight
    return (y if bias is None else y + np.asarray(bias, np.float64)), np.stack([m, r], 1)


def norm_bwd(s, weight, dy, dresidual_out=None, rms=False, eps=1e-5):
    """dict of ds, dweight, dbias, and ds_terms, dweight_terms, dbias_terms = sums of |terms|."""
    s, weight, dy = (np.asarray(v, np.float64) for v in (s, weight, dy))
    m, r = _stats(s, rms, eps)
    xh = (s - m[:, None]) * r[:, None]
    q = dy * weight
    ds, terms = q - xh * (q * xh).mean(1, keepdims=True), np.abs(q) + np.abs(xh * (q * xh).mean(1, keepdims=True))
    if not rms:
        ds, terms = ds - q.mean(1, keepdims=True), terms + np.abs(q.mean(1, keepdims=True))
    ds, terms = ds * r[:, None], terms * r[:, None]
    if dresidual_out is not None:
        ds, terms = ds + np.asarray(dresidual_out, np.float64), terms + np.abs(np.asarray(dresidual_out, np.float64))
    return {"ds": ds, "ds_terms": terms, "dweight": (dy * xh).sum(0), "dbias": dy.sum(0), "dweight_terms": np.abs(dy * xh).sum(0),
            "dbias_terms": np.abs(dy).sum(0)}
