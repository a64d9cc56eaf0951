"""Penalties, biases and masks on rows of logits, the tokens appended to a history, and the clipping of gradients, in double
precision with numpy: the definitions, a row at a time."""
from __future__ import annotations

import numpy as np


def _bad_sequence(b, V, history, length, prompt_length, scalars, bias):
    rho, presence, frequency = scalars
    if rho is not None and not (np.isfinite(rho) and rho > 0):
        return True
    if any(x is not None and not np.isfinite(x) for x in (presence, frequency)):
        return True
    if history is not None and any(x is not None for x in scalars):
        n, p = int(length[b]), 0 if prompt_length is None else int(prompt_length[b])
        if not 0 <= p <= n <= history.shape[1] or np.any((history[b, :n] < 0) | (history[b, :n] >= V)):
            return True
    if bias is not None:
        idx, value, count = bias
        k = int(count[b])
        if not 0 <= k <= idx.shape[1] or np.any((idx[b, :k] < 0) | (idx[b, :k] >= V)):
            return True
        if np.any(np.isnan(value[b, :k]) | (value[b, :k] == np.inf)):
            return True
    return False


def penalize(logits, history=None, length=None, prompt_length=None, draft_tok=None, repetition=None, presence=None, frequency=None,
             bias=None, mask=None, mask_row=None, grad=None):
    """logits [B,R,V]; history [B,L], length, prompt_length [B]; draft_tok [B,R-1]; repetition, presence, frequency [B]; bias = (idx [B,K],
    value [B,K], count [B]); mask [M,W] words with mask_row [B,R], or [B,R,W].  With `grad` [B,R,V]: the gradient with respect to the
    logits instead (logits may be None without repetition).  Returns float64 [B,R,V], NaN where the data is bad."""
    B, R, V = (grad if logits is None else logits).shape
    out = np.full((B, R, V), np.nan)
    if grad is not None:
        presence = frequency = bias = None
        if repetition is None:
            history = draft_tok = None
    counted = any(x is not None for x in (repetition, presence, frequency))
    for b in range(B):
        rho, pres, freq = (None if x is None else float(x[b]) for x in (repetition, presence, frequency))
        if _bad_sequence(b, V, history, length, prompt_length, (rho, pres, freq), bias):
            continue
        prompt, made = np.zeros(V, bool), np.zeros(V, np.int64)
        if counted and history is not None:
            n, p = int(length[b]), 0 if prompt_length is None else int(prompt_length[b])
            prompt[history[b, :p]] = True
            np.add.at(made, history[b, p:n], 1)
        extra = np.zeros(V)
        if bias is not None:
            for j in range(int(bias[2][b])):
                extra[bias[0][b, j]] = float(bias[1][b, j])
        for i in range(R):
            if i and counted and draft_tok is not None:
                t = int(draft_tok[b, i - 1])
                if not 0 <= t < V:
                    break
                made[t] += 1
            allowed = np.ones(V, bool)
            if mask is not None:
                m = 0 if mask_row is None else int(mask_row[b, i])
                if not -1 <= m < (1 if mask_row is None else mask.shape[0]):
                    continue
                if m >= 0:
                    words = mask[b, i] if mask_row is None else mask[m]
                    allowed = (words[np.arange(V) // 32].astype(np.int64) >> (np.arange(V) % 32)) & 1 != 0
            l = None if logits is None else logits[b, i].astype(np.float64)
            y = (l if grad is None else grad[b, i].astype(np.float64)).copy()
            seen = prompt | (made > 0)
            with np.errstate(invalid="ignore"):
                if rho is not None:
                    y[seen] *= np.where(l[seen] > 0, 1 / rho, rho)
                if grad is None:
                    at = made > 0
                    y[at] = y[at] - (freq or 0.0) * made[at] - (pres or 0.0)
                    y = y + extra
            y[~allowed] = -np.inf if grad is None else 0.0
            out[b, i] = y
    return out


def append(history, length, token=None, draft_tok=None, accept_len=None):
    """Returns (history, length) after the call, and whether any sequence had bad data."""
    history, length, bad = history.copy(), length.copy(), False
    for b in range(history.shape[0]):
        n = 0 if accept_len is None else int(accept_len[b])
        if n < 0:
            continue
        if n > (0 if draft_tok is None else draft_tok.shape[1]):
            bad = True
            continue
        new = ([] if draft_tok is None else draft_tok[b, :n].tolist()) + ([] if token is None else [int(token[b])])
        at = int(length[b])
        if not 0 <= at <= history.shape[1] or at + len(new) > history.shape[1] or any(t < 0 for t in new):
            bad = True
            continue
        history[b, at:at + len(new)] = new
        length[b] = at + len(new)
    return history, length, bad


def clip(grads, max_norm, norm=None):
    """(norm, scale, scaled gradients) of a list of arrays."""
    if norm is None:
        norm = float(np.sqrt(sum(float((g.astype(np.float64) ** 2).sum()) for g in grads)))
    scale = max_norm / norm if np.isfinite(norm) and norm > max_norm else 1.0
    return norm, scale, [g.astype(np.float64) * scale for g in grads]
