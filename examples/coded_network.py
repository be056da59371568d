"""A small residual network trained under coded aggregation, with stragglers: its layers, their gradients per run of data points, and the tree.

    python examples/coded_network.py [--points 600] [--steps 30]

The network takes `positions` tokens per data point: an embedding, residual blocks of group norm with SiLU, a dense layer and bias, dropout and residual
in one call, the mean over positions and a dense layer to the classes; softmax loss.  What its dense layers multiply is torch's; the rest are the
framework's layers.  Each step
  - the forward and backward pass over all data points, with the gradients of every run of points between two borders of the plan's segments,
  - the slab gradients that the workers would have formed: sums of runs,
  - the encode under a random straggler mask, the decode, the step.
The decoded gradient is the uncoded one whatever the mask, since every point's gradient depends on that point alone.
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_1902_01981_amd as cr  # noqa: E402


class Network:
    """Parameters are views of one vector `w`; gradients of runs are rows of one matrix of the same layout."""

    def __init__(self, inputs: int, channels: int, classes: int, blocks: int, groups: int, rate: float, seed: int, device="cuda"):
        self.channels, self.classes, self.blocks, self.groups, self.rate, self.seed = channels, classes, blocks, groups, rate, seed
        self.layout = [("embed", (inputs, channels))]
        for b in range(blocks):
            self.layout += [(f"gamma{b}", (channels,)), (f"beta{b}", (channels,)), (f"dense{b}", (channels, channels)), (f"bias{b}", (channels,))]
        self.layout.append(("out", (channels, classes)))
        self.size = sum(int(np.prod(shape)) for _, shape in self.layout)
        gen = torch.Generator(device=device).manual_seed(seed)
        self.w = torch.empty(self.size, device=device)
        for name, p in self.parameters(self.w).items():
            if p.dim() == 2:
                p.normal_(0.0, p.shape[0] ** -0.5, generator=gen)
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

    def forward(self, x, targets, step: int, first_point: int = 0, train: bool = True):
        """Loss of every point, the points' indices being first_point, first_point + 1, ...; keeps what the gradient needs."""
        p, rate = self.parameters(self.w), self.rate if train else 0.0
        N, P, _ = x.shape
        u = x @ p["embed"]
        kept = {"x": x, "step": step, "first": first_point, "rate": rate, "u": [], "v": [], "mean": [], "rstd": []}
        for b in range(self.blocks):
            v, mean, rstd = torch.empty_like(u), u.new_empty(N, self.groups), u.new_empty(N, self.groups)
            cr.cr_group_norm_forward(u, p[f"gamma{b}"], p[f"beta{b}"], self.groups, v, mean, rstd, activation=cr.CR_ACT_SILU)
            z, y = v @ p[f"dense{b}"], torch.empty_like(u)
            cr.cr_dropout_forward(z, y, rate, self.seed, step * self.blocks + b, bias=p[f"bias{b}"], residual=u, first_point=first_point)
            for name, value in zip(("u", "v", "mean", "rstd"), (u, v, mean, rstd)):
                kept[name].append(value)
            u = y
        kept["pooled"] = u.mean(dim=1)
        logits = kept["pooled"] @ p["out"]
        loss, kept["dlogits"] = u.new_empty(N), torch.empty_like(logits)
        cr.cr_softmax_loss(logits, targets, loss, dlogits=kept["dlogits"])
        return loss, kept

    def gradients(self, kept, bounds):
        """Gradients of the summed loss over each run of points: a row per run."""
        p, runs = self.parameters(self.w), len(bounds) - 1
        out = self.w.new_empty(runs, self.size)
        g = self.parameters(out)
        x, step = kept["x"], kept["step"]
        N, P, _ = x.shape

        def products(name, left, right):                 # left^T right, run by run
            left, right = left.reshape(N, -1, left.shape[-1]), right.reshape(N, -1, right.shape[-1])
            for r in range(runs):
                a, b = (t[bounds[r]:bounds[r + 1]].reshape(-1, t.shape[-1]) for t in (left, right))
                g[name][r] = a.t() @ b

        def vectors(name):                               # where a layer leaves a vector per run
            return out.new_empty(runs, self.channels)

        products("out", kept["pooled"], kept["dlogits"])
        # the mean's gradient is the same at every position: a broadcast view for the layers, which take strides
        du = (kept["dlogits"] @ p["out"].t() / P)[:, None, :].expand(N, P, self.channels)
        for b in reversed(range(self.blocks)):
            dz, dbias, dgamma, dbeta = out.new_empty(N, P, self.channels), vectors("bias"), vectors("gamma"), vectors("beta")
            cr.cr_dropout_backward(du, dz, kept["rate"], self.seed, step * self.blocks + b, dbias=dbias, bounds=bounds, first_point=kept["first"])
            products(f"dense{b}", kept["v"][b], dz)
            dv, dx = dz @ p[f"dense{b}"].t(), torch.empty_like(dz)
            cr.cr_group_norm_backward(dv, kept["u"][b], kept["mean"][b], kept["rstd"][b], p[f"gamma{b}"], p[f"beta{b}"], self.groups, dx, dgamma, dbeta,
                                      activation=cr.CR_ACT_SILU, bounds=bounds)
            g[f"bias{b}"].copy_(dbias)
            g[f"gamma{b}"].copy_(dgamma)
            g[f"beta{b}"].copy_(dbeta)
            du = du + dx                                 # the residual's gradient is that of the sum
        products("embed", x, du)
        return out


class Tree:
    """The workers of a tree, their slab gradients as sums of runs, and the coded sum of them."""

    def __init__(self, L: int, n: int, s: int, points: int, size: int):
        self.plan = cr.cr_plan_ex(L, n, s, points, size, model=cr.CR_AGGREGATE_ONLY)
        self.workspace = cr.Workspace(self.plan)
        self.info = self.workspace.info
        begin, end, _, _ = cr.cr_plan_get_segments(self.plan)
        self.bounds = np.unique(np.concatenate([[0, points], begin, end])).astype(np.int64)
        inside = (self.bounds[None, :-1] >= begin[:, None]) & (self.bounds[None, 1:] <= end[:, None])
        self.member = torch.from_numpy(inside.astype(np.float32)).cuda()                 # is run r part of slab p?
        self.slabs = torch.empty(self.info.num_slabs, size, device="cuda")
        self.g = torch.empty(size, device="cuda")

    def aggregate(self, run_gradients, mask):
        torch.matmul(self.member, run_gradients, out=self.slabs)
        cr.cr_load_partial_grads(self.plan, self.slabs)
        cr.cr_encode_tree(self.plan, mask)
        cr.cr_decode_root(self.plan, self.g)
        return self.g

    def close(self):
        cr.cr_synchronize(self.plan)
        cr.cr_plan_destroy(self.plan)


def data(points: int, positions: int, inputs: int, classes: int, seed: int):
    """Tokens around a centre per class."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    targets = torch.randint(0, classes, (points,), generator=gen, device="cuda")
    centres = torch.randn(classes, inputs, generator=gen, device="cuda")
    return centres[targets][:, None, :] + 2.0 * torch.randn(points, positions, inputs, generator=gen, device="cuda"), targets


def train(points=600, positions=16, inputs=24, channels=64, classes=10, blocks=2, groups=8, rate=0.1, steps=30, lr=1.0, tree=(2, 3, 1), seed=7, say=print):
    """Returns the mean loss per step, and the largest relative distance of a decoded gradient from the uncoded one."""
    x, targets = data(points, positions, inputs, classes, seed)
    net = Network(inputs, channels, classes, blocks, groups, rate, seed)
    workers = Tree(*tree, points, net.size)
    rng = np.random.default_rng(seed)
    n, s = tree[1], tree[2]
    losses, worst = [], 0.0
    for step in range(steps):
        mask = np.zeros(workers.info.num_workers, dtype=np.uint8)
        for group in range(workers.info.num_groups):
            mask[group * n + rng.choice(n, size=s, replace=False)] = 1
        loss, kept = net.forward(x, targets, step)
        runs = net.gradients(kept, workers.bounds)
        g, whole = workers.aggregate(runs, mask), runs.double().sum(dim=0)
        worst = max(worst, float((g.double() - whole).norm() / whole.norm()))
        net.w -= lr / points * g
        losses.append(float(loss.mean()))
        if say and step % 5 == 0:
            say(f"step {step:3d}  loss {losses[-1]:.4f}  stragglers {int(mask.sum())} of {len(mask)}  decoded against uncoded gradient {worst:.1e}")
    workers.close()
    return losses, worst


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--points", type=int, default=600)
    parser.add_argument("--steps", type=int, default=30)
    args = parser.parse_args()
    train(points=args.points, steps=args.steps)
