"""Distillation from a teacher's top entries and sampling from dense rows, in double precision with numpy: the definitions, a
row at a time."""
from __future__ import annotations

import numpy as np


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
            log_s = x - x.max()                     # (first: ln of the sum is lost in a maximum of 1e38)
            log_z = np.log(np.exp(log_s).sum())
            log_s -= log_z
            rest = x.copy()                         # (relative to its own maximum: beside an entry of 1e16 its differences are lost)
            rest[at] = -np.inf
            top = rest.max()
            q = np.exp(rest - top) if top > -np.inf else np.zeros_like(rest)
            log_r = (top - x.max()) + np.log(q.sum()) - log_z if top > -np.inf else -np.inf
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
                g -= r * q / q.sum()
            w = 1.0 if weight is None else float(weight[b, i])
            loss[b, i], grad[b, i], out[b, i] = v, w / T * g, np.exp(log_r)
    return loss, grad, out


CHUNK = 1024


def sample(logits, temperature, u, top_k=None, top_p=None, min_p=None, chunk=CHUNK):
    """logits [B,R,V]; temperature [B]; u [B,R,2]; top_k, top_p, min_p [B] or None.  Returns (token, prob, logprob,
    count) [B,R]; -1, -1, NaN, -1 for bad data."""
    B, R, V = logits.shape
    token, count = np.full((B, R), -1, np.int32), np.full((B, R), -1, np.int32)
    prob, logprob = np.full((B, R), -1.0), np.full((B, R), np.nan)
    for b in range(B):
        T = float(temperature[b])
        k = 0 if top_k is None else int(top_k[b])
        p = 1.0 if top_p is None else float(top_p[b])
        m = 0.0 if min_p is None else float(min_p[b])
        if not (np.isfinite(T) and T > 0) or k < 0 or not p > 0 or not 0 <= m <= 1:
            continue
        for i in range(R):
            l = logits[b, i].astype(np.float64)
            if np.any(np.isnan(l) | (l == np.inf)) or not np.any(l > -np.inf):
                continue
            order = np.lexsort((np.arange(V), -l))
            order = order[l[order] > -np.inf]
            w = np.exp((l - l.max()) / T)
            Z = w.sum()
            s = w[order]
            keep = np.ones(order.size, bool)
            if k:
                keep &= np.arange(order.size) < k
            if p < 1:
                keep &= np.concatenate([[0.0], np.cumsum(s)[:-1]]) < p * Z
            if m > 0:                               # (w >= m: exp rounds weights next to 1 to 1)
                keep &= (l[order] - l.max()) / T >= np.log(m)
            keep[0] = True
            kept = np.zeros(V)
            kept[order[keep]] = s[keep]
            mass = np.add.reduceat(kept, np.arange(0, V, chunk))
            upto = np.cumsum(mass)
            c = min(int((upto <= float(u[b, i, 0]) * upto[-1]).sum()), int(np.nonzero(mass)[0][-1]))
            inside = kept[c * chunk:(c + 1) * chunk]
            upto_e = np.cumsum(inside)
            e = min(int((upto_e <= float(u[b, i, 1]) * upto_e[-1]).sum()), int(np.nonzero(inside)[0][-1]))
            t = c * chunk + e
            token[b, i], count[b, i] = t, int(keep.sum())
            prob[b, i], logprob[b, i] = kept[t] / upto[-1], np.log(w[t] / Z)
    return token, prob, logprob, count
