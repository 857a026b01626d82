"""Operators on an LM head's logits, in 64 bits on whole rows (test infrastructure; see package header).

Rows are the V columns of the vocabulary without pads, as float64 arrays; how a layout cuts them is the caller's
business (a Split or Merge changes it without changing the model, section 6.2, preserving training semantics).
Loops per row and entry, written from the definitions:

* :func:`constrain` -- repetition, frequency and presence penalties, biases, an allowed set;
* :func:`topk`      -- the k largest with their log-probabilities, equal values in column order;
* :func:`distill`   -- KL divergence from a teacher's listed probabilities to the softmax, with its gradient.
"""
from __future__ import annotations

import numpy as np


def constrain(x, history=None, prompt_len=None, theta=None, frequency=None, presence=None, biases=None, allowed=None):
    """x [rows, V]. history[r]: the row's tokens (those outside [0, V) are skipped), of which the first
    prompt_len[r] are the prompt. biases[r]: (token, value) pairs. allowed[r]: boolean [V] or None."""
    out = np.array(x, dtype=np.float64)
    rows, V = out.shape
    for r in range(rows):
        seen, count = set(), {}
        for i, v in enumerate(history[r] if history is not None else ()):
            if 0 <= v < V:
                seen.add(v)
                if i >= (prompt_len[r] if prompt_len is not None else 0):
                    count[v] = count.get(v, 0) + 1
        if theta is not None:
            for v in seen:
                out[r, v] = out[r, v] / theta[r] if out[r, v] > 0 else out[r, v] * theta[r]
        for v, n in count.items():
            out[r, v] -= (frequency[r] * n if frequency is not None else 0) + (presence[r] if presence is not None else 0)
        total = {}
        for v, b in (biases[r] if biases is not None else ()):
            if 0 <= v < V:
                total[v] = total.get(v, 0.0) + b
        for v, b in total.items():
            out[r, v] += b
        if allowed is not None and allowed[r] is not None:
            out[r, ~allowed[r]] = -np.inf
    return out


def log_softmax(x, tau=1.0):
    """(log softmax(x / tau), log sum exp(x / tau)) of every row, relative to its largest value: at the ends of a
    type's range log V would be lost beside it. A NaN or +infinity anywhere gives NaN, -infinity alone -infinity."""
    m = np.max(np.where(np.isnan(x), -np.inf, x), axis=1)
    safe = np.where(np.isinf(m) & (m < 0), 0.0, m)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        d = (x - safe[:, None]) / tau
        log_s = np.log(np.exp(d).sum(1))
        return np.where(d == -np.inf, np.where(np.isnan(log_s), np.nan, -np.inf)[:, None], d - log_s[:, None]), safe / tau + log_s


def log_sum_exp(x):
    return log_softmax(x)[1]


def topk(x, k, tau=1.0):
    """(index, log-probability, lse) of the k largest of every row."""
    rows, V = x.shape
    log_q, lse = log_softmax(x, tau)
    index, logp = np.full((rows, k), -1, np.int64), np.full((rows, k), -np.inf)
    for r in range(rows):
        order = [int(v) for v in np.argsort(-x[r], kind="stable") if x[r, v] > -np.inf][:k]
        index[r, :len(order)] = order
        logp[r, :len(order)] = log_q[r, order]
        if np.isnan(lse[r]):
            logp[r] = np.nan
    return index, logp, lse


def distill(z, index, value, weight=None, tau=1.0, tail=False):
    """dict(loss, grad, lse, factor, p, q) for student logits z [rows, V] and a teacher's entries [rows, k]."""
    z = np.asarray(z, dtype=np.float64)
    rows, V = z.shape
    every, lse = log_softmax(z, tau)
    loss, grad, factor, P, Q = np.zeros(rows), np.zeros((rows, V)), np.ones(rows), np.zeros((rows, V)), np.zeros((rows, V))
    for r in range(rows):
        w = 1.0 if weight is None else float(weight[r])
        if w == 0:
            continue
        p, listed = np.zeros(V), np.zeros(V, bool)
        entries = [(int(v), float(t)) for v, t in zip(index[r], value[r]) if 0 <= v < V]
        if not tail:
            top = max([t for _, t in entries], default=-np.inf)
            if top == -np.inf:
                continue
            entries = [(v, np.exp(t - top)) for v, t in entries]
            total = sum(e for _, e in entries)
            entries = [(v, e / total) for v, e in entries]
        else:
            entries = [(v, np.exp(t)) for v, t in entries]
        for v, e in entries:
            p[v] += e
            listed[v] = True
        with np.errstate(invalid="ignore", divide="ignore"):
            log_q = every[r]
            q = np.exp(log_q)
            L = sum(p[v] * (np.log(p[v]) - log_q[v]) for v in np.flatnonzero(p != 0))
            f = 1.0
            if tail:
                rest = max(0.0, 1.0 - sum(e for _, e in entries))
                q_rest = q[~listed].sum()
                if rest > (0 if q_rest > 0 else 2.0 ** -20):
                    L += rest * (np.log(rest) - np.log(q_rest))
                if not q_rest < 2.0 ** -100:
                    f = 1.0 - rest / q_rest
        loss[r], factor[r] = w * L, f
        grad[r] = w / tau * np.where(listed, q - p, q * f)
        P[r], Q[r] = p, q
    return dict(loss=loss, grad=grad, lse=lse, factor=factor, p=P, q=Q)
