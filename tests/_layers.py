"""The network layers from their formulas, in 64 bits on the host: what the tests of the layers compare with."""
from __future__ import annotations

import numpy as np
import torch

U = 2.0 ** -24                                           # half a unit in the last place of fp32, relative
HALF_ULP = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16)}      # of a rounding to nearest, relative
GOLDEN = 0x9E3779B97F4A7C15
ACTS = ("none", "relu", "silu")                          # in the order of enum cr_activation


def wide(t):
    return t.detach().double().cpu()


def act(kind, z):
    return {"none": z, "relu": torch.where(z < 0, torch.zeros_like(z), z), "silu": z / (1 + torch.exp(-z))}[kind]


def act_slope(kind, z):
    if kind == "none":
        return torch.ones_like(z)
    if kind == "relu":
        return (z > 0).double()
    s = 1 / (1 + torch.exp(-z))
    return s + z * s * (1 - s)


def norm_forward(x, gamma, beta, groups, eps, kind):
    """x (points, positions, channels) in 64 bits; returns y, mean, rstd."""
    N, P, C = x.shape
    v = x.reshape(N, P, groups, C // groups)
    mean = v.mean(dim=(1, 3))
    var = (v - mean[:, None, :, None]).square().mean(dim=(1, 3))
    rstd = (var + eps) ** -0.5
    h = ((v - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(N, P, C)
    return act(kind, h * gamma + beta), mean, rstd


def norm_backward(dy, x, mean, rstd, gamma, beta, groups, kind, bounds):
    """Returns dx, dgamma, dbeta, and the sums of the absolute values of the terms of the last two."""
    N, P, C = x.shape

    def spread(s):
        return s.repeat_interleave(C // groups, dim=1)[:, None, :]

    def group_mean(v):
        return spread(v.reshape(N, P, groups, C // groups).mean(dim=(1, 3)))

    h = (x - spread(mean)) * spread(rstd)
    dz = dy * act_slope(kind, gamma * h + beta)
    dx = spread(rstd) * (gamma * dz - group_mean(gamma * dz) - h * group_mean(gamma * dz * h))

    def per_run(v):
        v = v.sum(dim=1)
        return torch.stack([v[bounds[r]:bounds[r + 1]].sum(dim=0) for r in range(len(bounds) - 1)])

    return dx, per_run(dz * h), per_run(dz), per_run((dz * h).abs()), per_run(dz.abs())


def mix(z):
    with np.errstate(over="ignore"):
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        return z ^ (z >> np.uint64(31))


def least_kept(rate):
    return int(np.floor(rate * 65536 + 0.5))


def kept(points, positions, channels, rate, seed, draw):
    """The mask for the points with these indices: (len(points), positions, channels) truth values, and the scale."""
    words = (channels + 3) // 4
    with np.errstate(over="ignore"):
        key = mix(np.array([(seed + (draw + 1) * GOLDEN) % (1 << 64)], dtype=np.uint64))
        point = np.array([int(p) % (1 << 64) for p in points], dtype=np.uint64)[:, None, None]
        row = point * np.uint64(positions) + np.arange(positions, dtype=np.uint64)[None, :, None]
        number = row * np.uint64(words) + np.arange(words, dtype=np.uint64)
        z = mix(key + (number + np.uint64(1)) * np.uint64(GOLDEN))
    fields = np.stack([(z >> np.uint64(16 * f)) & np.uint64(0xFFFF) for f in range(4)], axis=-1).reshape(len(points), positions, 4 * words)
    least = least_kept(rate)
    return torch.from_numpy(fields[:, :, :channels].astype(np.int64) >= least), 65536.0 / (65536 - least)


def softmax_loss(x, targets, weights):
    """Returns loss, lse, gradient in 64 bits, row by row as the definition says (an infinite sum is not a number)."""
    N, V = x.shape
    loss, lse, grad = torch.zeros(N, dtype=torch.float64), torch.zeros(N, dtype=torch.float64), torch.zeros(N, V, dtype=torch.float64)
    for i in range(N):
        row, t, w = x[i], int(targets[i]), 1.0 if weights is None else float(weights[i])
        lse[i] = np.nan if bool((row == np.inf).any()) else torch.logsumexp(row, dim=0)
        none = bool((row == -np.inf).all())
        if t < 0:
            continue
        if t >= V:
            loss[i], grad[i] = np.nan, np.nan
            continue
        loss[i] = w * np.inf if none else w * (lse[i] - row[t])
        if not none:
            grad[i] = w * torch.exp(row - lse[i])
            grad[i, t] -= w
    return loss, lse, grad
