"""The layers of networks over tokens from their formulas, in 64 bits on the host: what their tests compare with."""
from __future__ import annotations

import math

import torch

INF = math.inf


def log_softmax(x):
    """By distances to the largest: next to logits of 10^38 64 bits do not hold log(classes)."""
    d = x - x.amax(dim=-1, keepdim=True)
    return d - torch.logsumexp(d, dim=-1, keepdim=True)


def embedding(tokens, table, scale):
    """tokens (points, positions), table (vocabulary, channels) in 64 bits."""
    V, C = table.shape
    y = torch.zeros(*tokens.shape, C, dtype=torch.float64)
    known = (tokens >= 0) & (tokens < V)
    y[known] = table[tokens[known]] * scale
    y[tokens >= V] = math.nan
    return y


def embedding_gradient(dy, tokens, vocabulary, scale, bounds):
    """Returns the gradient per run, and the sums of the absolute values of its terms, and the number of terms."""
    runs, C = len(bounds) - 1, dy.shape[-1]
    out, size, count = (torch.zeros(runs, vocabulary, n, dtype=torch.float64) for n in (C, C, 1))
    for r in range(runs):
        t, d = tokens[bounds[r]:bounds[r + 1]].reshape(-1), dy[bounds[r]:bounds[r + 1]].reshape(-1, C)
        known = (t >= 0) & (t < vocabulary)
        out[r].index_add_(0, t[known], d[known])
        size[r].index_add_(0, t[known], d[known].abs())
        count[r].index_add_(0, t[known], torch.ones(int(known.sum()), 1, dtype=torch.float64))
    return out * scale, size * abs(scale), count


def log_probs(x, tokens, top):
    """x (rows, classes) in 64 bits; returns logp, entropy, top_index, top_logp, row by row as the definition says."""
    N, V = x.shape
    logp, entropy = torch.zeros(N, dtype=torch.float64), torch.zeros(N, dtype=torch.float64)
    index, values = torch.full((N, top), -1, dtype=torch.int64), torch.full((N, top), -INF, dtype=torch.float64)
    for i in range(N):
        row, t = x[i], -1 if tokens is None else int(tokens[i])
        if bool(row.isnan().any()) or bool((row == INF).any()):
            logp[i], entropy[i], values[i] = 0.0 if t < 0 else math.nan, math.nan, math.nan
            continue
        can = row > -INF
        if not bool(can.any()):
            logp[i] = 0.0 if t < 0 else math.nan if t >= V else -INF
            continue
        c = row[can].max()
        l = row - c - torch.log(torch.exp(row[can] - c).sum())
        p = torch.exp(l)
        entropy[i] = -(p[p > 0] * l[p > 0]).sum()
        logp[i] = 0.0 if t < 0 else math.nan if t >= V else l[t]
        if top:
            ranked = torch.sort(row + 0.0, descending=True, stable=True).indices[:top]
            ranked = ranked[can[ranked]]
            index[i, :len(ranked)], values[i, :len(ranked)] = ranked, l[ranked]
    return logp, entropy, index, values


def log_probs_gradient(x, tokens, dlogp, dentropy):
    N, V = x.shape
    out = torch.zeros(N, V, dtype=torch.float64)
    for i in range(N):
        row, t = x[i], -1 if tokens is None else int(tokens[i])
        a = 0.0 if t < 0 else float(dlogp[i])
        b = 0.0 if dentropy is None else float(dentropy[i])
        if t >= V or bool(row.isnan().any()) or bool((row == INF).any()):
            out[i] = math.nan
            continue
        can = row > -INF
        if not bool(can.any()):
            continue
        l = log_softmax(row)
        p = torch.exp(l)
        safe = torch.where(p > 0, l, torch.zeros(()).double())
        out[i] = -a * p - b * p * (safe - (p * safe).sum())
        if t >= 0:
            out[i, t] += a
    return out


def distill(x, index, z, T, weights):
    """x (rows, classes), z (rows, top) in 64 bits; returns loss, gradient, and the sum of the absolute values of the loss's terms."""
    N, V = x.shape
    loss, grad, size = torch.zeros(N, dtype=torch.float64), torch.zeros(N, V, dtype=torch.float64), torch.zeros(N, dtype=torch.float64)
    for i in range(N):
        row, w = x[i] / T, 1.0 if weights is None else float(weights[i])
        there = (index[i] >= 0) & (z[i] != -INF)
        if not bool(there.any()):
            continue
        j, zi = index[i][there], z[i][there] / T
        if bool((j >= V).any()) or bool(zi.isnan().any()) or bool((zi == INF).any()) or bool(row.isnan().any()) or bool((row == INF).any()):
            loss[i], grad[i], size[i] = math.nan, math.nan, 1.0
            continue
        log_q = log_softmax(zi)
        q = torch.exp(log_q)
        if bool((row == -INF).all()):
            loss[i] = w * INF
            continue
        log_p = log_softmax(row)
        counts = q > 0
        loss[i] = w * T * T * (q[counts] * (log_q[counts] - log_p[j[counts]])).sum()
        size[i] = abs(w) * T * T * (q[counts] * (1 + log_q[counts].abs() + log_p[j[counts]].abs())).sum()
        grad[i] = w * T * torch.exp(log_p)
        grad[i].index_add_(0, j, -w * T * q)
    return loss, grad, size
