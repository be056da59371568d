"""A small network over tokens distilled from a teacher under coded aggregation, with stragglers.

    python examples/coded_tokens.py [--points 240] [--steps 30]

A data point is a sequence of tokens, some shorter than others (their ends have no token).  Network: the tokens' rows of a table, residual blocks of group norm
with SiLU, a dense layer and bias, dropout and residual in one call, and at every position a dense layer to logits over the vocabulary.  The teacher, a network of the same
form with weights of its own, writes down its most probable tokens for every position once; the student's loss is the distillation loss on them, a sum over
positions, so that a point's gradient depends on that point alone.  What the dense layers multiply is torch's; the rest are the framework's layers.  Each step
  - the forward and backward pass over all data points, with the gradients of every run of points between two borders of the plan's segments,
  - the slab gradients that the workers would have formed: sums of runs,
  - the encode under a random straggler mask, the decode, the step.
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1902_01981_amd as cr  # noqa: E402
from examples.coded_network import Tree  # noqa: E402


class Network:
    """Parameters are views of one vector `w`; gradients of runs are rows of one matrix of the same layout."""

    def __init__(self, vocabulary: int, channels: int, blocks: int, groups: int, rate: float, seed: int, device="cuda"):
        self.vocabulary, self.channels, self.blocks, self.groups, self.rate, self.seed = vocabulary, channels, blocks, groups, rate, seed
        self.scale = channels ** 0.5                     # of the table's rows
        self.layout = [("table", (vocabulary, channels))]
        for b in range(blocks):
            self.layout += [(f"gamma{b}", (channels,)), (f"beta{b}", (channels,)), (f"dense{b}", (channels, channels)), (f"bias{b}", (channels,))]
        self.layout.append(("out", (channels, vocabulary)))
        self.size = sum(int(np.prod(shape)) for _, shape in self.layout)
        gen = torch.Generator(device=device).manual_seed(seed)
        self.w = torch.empty(self.size, device=device)
        for name, p in self.parameters(self.w).items():
            if p.dim() == 2:
                p.normal_(0.0, channels ** -0.5, generator=gen)
            else:
                p.fill_(1.0 if name.startswith("gamma") else 0.0)

    def parameters(self, vector) -> dict:
        """The parameters, or their gradients for several runs, as views of a vector, or of rows."""
        out, at = {}, 0
        for name, shape in self.layout:
            n = int(np.prod(shape))
            out[name] = vector[..., at:at + n].view(*vector.shape[:-1], *shape)
            at += n
        return out

    def logits(self, tokens, step: int, first_point: int = 0, train: bool = True):
        """Logits of every position, a row each, the points' indices being first_point, first_point + 1, ...; keeps what the gradient needs."""
        p, rate = self.parameters(self.w), self.rate if train else 0.0
        N, P = tokens.shape
        u = self.w.new_empty(N, P, self.channels)
        cr.cr_embedding_forward(tokens, p["table"], u, scale=self.scale)
        kept = {"tokens": tokens, "step": step, "first": first_point, "rate": rate, "u": [], "v": [], "mean": [], "rstd": []}
        for b in range(self.blocks):
            v, mean, rstd = torch.empty_like(u), u.new_empty(N, self.groups), u.new_empty(N, self.groups)
            cr.cr_group_norm_forward(u, p[f"gamma{b}"], p[f"beta{b}"], self.groups, v, mean, rstd, activation=cr.CR_ACT_SILU)
            z, y = v @ p[f"dense{b}"], torch.empty_like(u)
            cr.cr_dropout_forward(z, y, rate, self.seed, step * self.blocks + b, bias=p[f"bias{b}"], residual=u, first_point=first_point)
            for name, value in zip(("u", "v", "mean", "rstd"), (u, v, mean, rstd)):
                kept[name].append(value)
            u = y
        kept["last"] = u
        return u.view(N * P, self.channels) @ p["out"], kept

    def answers(self, tokens, top: int):
        """The `top` most probable tokens of every position, and their log probabilities; none where there is no token."""
        logits, _ = self.logits(tokens, 0, train=False)
        index, values = torch.empty(logits.shape[0], top, dtype=torch.int64, device=logits.device), logits.new_empty(logits.shape[0], top)
        cr.cr_log_probs(logits, top_index=index, top_logp=values)
        index[tokens.reshape(-1) < 0] = -1
        return index, values

    def forward(self, tokens, answers, temperature: float, step: int, first_point: int = 0):
        """The loss of every position; the logits' gradient takes their place."""
        logits, kept = self.logits(tokens, step, first_point)
        loss = logits.new_empty(logits.shape[0])
        cr.cr_distill_loss(logits, *answers, loss, temperature=temperature, dlogits=logits)
        kept["dlogits"] = logits
        return loss.view(tokens.shape), kept

    def gradients(self, kept, bounds):
        """Gradients of the summed loss over each run of points: a row per run."""
        p, runs = self.parameters(self.w), len(bounds) - 1
        out = self.w.new_empty(runs, self.size)
        g = self.parameters(out)
        tokens, step = kept["tokens"], kept["step"]
        N, P = tokens.shape

        def products(name, left, right):                 # left^T right, run by run
            left, right = left.reshape(N, P, left.shape[-1]), right.reshape(N, P, right.shape[-1])
            for r in range(runs):
                a, b = (t[bounds[r]:bounds[r + 1]].reshape(-1, t.shape[-1]) for t in (left, right))
                g[name][r] = a.t() @ b

        def vectors():                                   # where a layer leaves a vector per run
            return out.new_empty(runs, self.channels)

        products("out", kept["last"], kept["dlogits"])
        du = (kept["dlogits"] @ p["out"].t()).view(N, P, self.channels)
        for b in reversed(range(self.blocks)):
            dz, dbias, dgamma, dbeta = torch.empty_like(du), vectors(), vectors(), vectors()
            cr.cr_dropout_backward(du, dz, kept["rate"], self.seed, step * self.blocks + b, dbias=dbias, bounds=bounds, first_point=kept["first"])
            products(f"dense{b}", kept["v"][b], dz)
            dv, dx = dz @ p[f"dense{b}"].t(), torch.empty_like(dz)
            cr.cr_group_norm_backward(dv, kept["u"][b], kept["mean"][b], kept["rstd"][b], p[f"gamma{b}"], p[f"beta{b}"], self.groups, dx, dgamma, dbeta,
                                      activation=cr.CR_ACT_SILU, bounds=bounds)
            g[f"bias{b}"].copy_(dbias)
            g[f"gamma{b}"].copy_(dgamma)
            g[f"beta{b}"].copy_(dbeta)
            du = du + dx                                 # the residual's gradient is that of the sum
        dtable = out.new_empty(runs, self.vocabulary, self.channels)
        cr.cr_embedding_backward(du, tokens, dtable, scale=self.scale, bounds=bounds)
        g["table"].copy_(dtable)
        return out


def data(points: int, positions: int, vocabulary: int, seed: int):
    """Sequences of tokens, frequent ones and rare ones; a third of them end early."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    tokens = (torch.rand(points, positions, generator=gen, device="cuda") ** 3 * vocabulary).long().clamp_(max=vocabulary - 1)
    lengths = torch.randint(1, positions + 1, (points,), generator=gen, device="cuda")
    lengths[torch.rand(points, generator=gen, device="cuda") < 2 / 3] = positions
    tokens[torch.arange(positions, device="cuda") >= lengths[:, None]] = -1
    return tokens


def train(points=240, positions=12, vocabulary=300, channels=48, blocks=2, groups=8, rate=0.1, top=8, temperature=2.0, steps=30, lr=0.3, tree=(2, 3, 1), seed=7, say=print):
    """Returns the mean loss per step, and the largest relative distance of a decoded gradient from the uncoded one."""
    tokens = data(points, positions, vocabulary, seed)
    answers = Network(vocabulary, channels, blocks, groups, rate, seed + 1).answers(tokens, top)
    net = Network(vocabulary, channels, blocks, groups, rate, seed)
    workers = Tree(*tree, points, net.size)
    rng = np.random.default_rng(seed)
    n, s = tree[1], tree[2]
    count = int((tokens >= 0).sum())
    losses, worst = [], 0.0
    for step in range(steps):
        mask = np.zeros(workers.info.num_workers, dtype=np.uint8)
        for group in range(workers.info.num_groups):
            mask[group * n + rng.choice(n, size=s, replace=False)] = 1
        loss, kept = net.forward(tokens, answers, temperature, step)
        runs = net.gradients(kept, workers.bounds)
        g, whole = workers.aggregate(runs, mask), runs.double().sum(dim=0)
        worst = max(worst, float((g.double() - whole).norm() / whole.norm()))
        net.w -= lr / count * g
        losses.append(float(loss.sum()) / count)
        if say and step % 5 == 0:
            say(f"step {step:3d}  loss {losses[-1]:.4f}  stragglers {int(mask.sum())} of {len(mask)}  decoded against uncoded gradient {worst:.1e}")
    workers.close()
    return losses, worst


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--points", type=int, default=240)
    parser.add_argument("--steps", type=int, default=30)
    args = parser.parse_args()
    train(points=args.points, steps=args.steps)
