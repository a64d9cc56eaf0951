"""Distillation from a teacher's top entries, in double precision with numpy: the definition, a row at a time."""
from __future__ import annotations

import numpy as np


def _lse(x: np.ndarray) -> float:
    m = x.max() if x.size else -np.inf
    return float(m) if not np.isfinite(m) else float(m + np.log(np.exp(x - m).sum()))


def distill(logits, temperature, t_idx, t_prob, t_count, weight=None, tail=False):
    """logits [B,R,V]; temperature [B]; t_idx, t_prob [B,R,K]; t_count [B,R]; weight [B,R] or None.
    Returns (loss [B,R], grad [B,R,V], outside [B,R]): float64; outside = the student's mass outside the entries.
    Bad data: NaN in the row's loss and gradient."""
    B, R, V = logits.shape
    loss, grad, out = np.zeros((B, R)), np.zeros((B, R, V)), np.ones((B, R))
    for b in range(B):
        T = float(temperature[b])
        for i in range(R):
            n = int(t_count[b, i])
            if n == 0:
                continue
            l = logits[b, i].astype(np.float64)
            ok = np.isfinite(T) and T > 0 and 0 < n <= t_idx.shape[2]
            at, t = t_idx[b, i, :max(n, 0)].astype(np.int64), t_prob[b, i, :max(n, 0)].astype(np.float64)
            ok = ok and len(set(at.tolist())) == len(at) and np.all((at >= 0) & (at < V))
            ok = ok and np.all(np.isfinite(t)) and np.all(t >= 0)
            ok = ok and not np.any(np.isnan(l) | (l == np.inf)) and np.any(l > -np.inf)
            if not ok:
                loss[b, i], grad[b, i] = np.nan, np.nan
                continue
            x = l / T
            log_s = x - _lse(x)
            rest = log_s.copy()
            rest[at] = -np.inf
            log_r = _lse(rest)
            A = t.sum()
            r = max(0.0, 1.0 - A) if tail else 0.0
            pos = t > 0
            with np.errstate(divide="ignore"):
                v = float((t[pos] * (np.log(t[pos]) - log_s[at][pos])).sum())
            if r > 0:
                v += r * (np.log(r) - log_r)
            g = (A + r) * np.exp(log_s)
            g[at] -= t
            if r > 0 and log_r > -np.inf:
                g -= r * np.exp(rest - log_r)
            w = 1.0 if weight is None else float(weight[b, i])
            loss[b, i], grad[b, i], out[b, i] = v, w / T * g, np.exp(log_r)
    return loss, grad, out
