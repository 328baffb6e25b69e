"""64-bit definition of softmax attention over spans of keys, with capped and distance-biased scores, and its gradients, in numpy.

Row i of batch entry b sees the keys begin[b, i] <= j < end[b, i] (cut to those there are).  With s = scale q_i . k_j a score is cap tanh(s / cap)
where cap > 0, less slopes[h] |i + L_k - L_q - j| where slopes are given.  A row that sees nothing has a zero output, the statistic -inf
and zero gradients."""
from __future__ import annotations

import numpy as np


def spans_of(mask, B, L_q, L_k, window=0):
    """(begin, end) [B, L_q] of the masks "none", "causal" and "sliding_window" (bottom-right aligned)."""
    i = np.arange(L_q) + L_k - L_q
    end = np.full(L_q, L_k) if mask == "none" else np.clip(i + 1, 0, L_k)
    begin = np.maximum(i + 1 - window, 0) if mask == "sliding_window" else np.zeros(L_q, dtype=int)
    return np.tile(begin, (B, 1)), np.tile(end, (B, 1))


def document_spans(offsets, L, mask="causal", window=0, prefix=None):
    """(begin, end) [B, L] of documents offsets[b][d] <= i < offsets[b][d + 1], token by token."""
    offsets = np.atleast_2d(offsets)
    begin, end = np.zeros((len(offsets), L), dtype=int), np.zeros((len(offsets), L), dtype=int)
    for b, at in enumerate(offsets):
        for d in range(len(at) - 1):
            first, behind = max(at[d], 0), min(at[d + 1], L)
            for i in range(first, behind):
                begin[b, i], end[b, i] = first, behind
                if mask != "none":
                    end[b, i] = i + 1
                    if prefix is not None:
                        end[b, i] = max(i + 1, first + min(max(np.atleast_2d(prefix)[b][d], 0), behind - first))
                if mask == "sliding_window":
                    begin[b, i] = max(first, i + 1 - window)
    return begin, end


def _scores(q, k, b, h, begin, end, scale, cap, slopes):
    """Modified scores [L_q, L_k] with -inf where hidden, and the derivative of the cap."""
    L_q, L_k = len(q), len(k)
    s = scale * (q @ k.T)
    bend = np.ones_like(s)
    if cap:
        t = np.tanh(s / cap)
        s, bend = cap * t, 1 - t * t
    j = np.arange(L_k)
    if slopes is not None:
        s = s - slopes[h] * np.abs(np.arange(L_q)[:, None] + L_k - L_q - j)
    seen = (j >= begin[b][:, None]) & (j < end[b][:, None])
    return np.where(seen, s, -np.inf), bend


def _softmax(s):
    top = s.max(1, keepdims=True)
    with np.errstate(invalid="ignore", divide="ignore"):
        w = np.exp(s - np.where(np.isfinite(top), top, 0.0))
        total = w.sum(1, keepdims=True)
        return w / np.where(total > 0, total, 1.0), np.where(total > 0, top + np.log(np.where(total > 0, total, 1.0)), -np.inf)[:, 0]


def span_attention(Q, K, V, begin, end, *, scale, cap=0.0, slopes=None):
    """O [B, H_q, L_q, D_v], stats [B, H_q, L_q], and sum_j p_j |v_j| of O's shape (what a relative error of the weights amounts to)."""
    Q, K, V = (np.asarray(x, dtype=np.float64) for x in (Q, K, V))
    g = Q.shape[1] // K.shape[1]
    O, mag, stats = np.zeros(Q.shape[:3] + V.shape[3:]), np.zeros(Q.shape[:3] + V.shape[3:]), np.zeros(Q.shape[:3])
    for b in range(Q.shape[0]):
        for h in range(Q.shape[1]):
            s, _ = _scores(Q[b, h], K[b, h // g], b, h, begin, end, scale, cap, slopes)
            p, stats[b, h] = _softmax(s)
            O[b, h], mag[b, h] = p @ V[b, h // g], p @ np.abs(V[b, h // g])
    return O, stats, mag


def span_attention_backward(Q, K, V, dO, begin, end, *, scale, cap=0.0, slopes=None, e_p=0.0, e_dp=0.0):
    """(dQ, dK, dV) and, for each, what it changes by at most where weights are off by e_p of them, dP - delta by e_dp (times scale, an absolute
    error of the row), and weights and score gradients are rounded to bf16 (2^-8 of each) for the products."""
    Q, K, V, dO = (np.asarray(x, dtype=np.float64) for x in (Q, K, V, dO))
    g, half = Q.shape[1] // K.shape[1], 2.0 ** -8
    grads, bounds = [np.zeros(x.shape) for x in (Q, K, V)], [np.zeros(x.shape) for x in (Q, K, V)]
    for b in range(Q.shape[0]):
        for h in range(Q.shape[1]):
            q, k, v, do = Q[b, h], K[b, h // g], V[b, h // g], dO[b, h]
            s, bend = _scores(q, k, b, h, begin, end, scale, cap, slopes)
            p, _ = _softmax(s)
            dp = do @ v.T
            ds = p * (dp - (p * dp).sum(1, keepdims=True)) * bend * scale
            off = np.abs(ds) * (half + 2 * e_p) + p * abs(scale) * e_dp + (p * np.abs(dp - (p * dp).sum(1, keepdims=True)) * abs(scale) * 4e-7 if cap else 0.0)
            grads[0][b, h], bounds[0][b, h] = ds @ k, off @ np.abs(k)
            grads[1][b, h // g] += ds.T @ q
            bounds[1][b, h // g] += off.T @ np.abs(q)
            grads[2][b, h // g] += p.T @ do
            bounds[2][b, h // g] += (p * (half + 2 * e_p)).T @ np.abs(do)
    return grads, bounds
