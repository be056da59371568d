"""The layers of a network that trains under coded aggregation, as cases whose time can be taken.

A case is a dict of plain values.  Three operators, each over data points of `positions` rows of `channels` columns:

  norm      group norm with an activation, channels last; training: with all gradients, the parameters' per run of consecutive points
  dropout   bias, dropout and residual, the mask from a counter; training: with the gradients, the bias's per run
  loss      softmax loss per row from logits (a sum over rows, weighted, some rows without a target), with its gradient or without

Where `own` is false they are computed in their plain form, else by the framework's entry points.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

GOLDEN = 0x9E3779B97F4A7C15
MIX = (0xBF58476D1CE4E5B9, 0x94D049BB133111EB)
MOST_ELEMENTS = 8192 * 131_071                           # of the largest listed case


def _norm(points, positions, channels, groups, bf16=False, train=False, activation="silu", runs=1):
    return {"kind": "norm", "points": points, "positions": positions, "channels": channels, "groups": groups, "bf16": bf16, "train": train,
            "activation": activation, "runs": runs}


def _dropout(points, positions, channels, rate, bf16=False, train=False, residual=True, runs=1):
    return {"kind": "dropout", "points": points, "positions": positions, "channels": channels, "rate": rate, "bf16": bf16, "train": train,
            "residual": residual, "runs": runs}


def _loss(rows, classes, bf16=False, train=True, masked=0):
    return {"kind": "loss", "rows": rows, "classes": classes, "bf16": bf16, "train": train, "masked": masked}


def listed():
    return [
        # one point answered by a small network: launches and the call itself
        dict(_norm(1, 64, 64, 8, activation="relu"), name="norm 1x64x64"),
        # the first layer of the paper's simulated network (16 channels on 32 x 32) for the 320 points of one of its 156 workers
        dict(_norm(320, 1024, 16, 4, bf16=True, train=True), name="norm train 320x1024x16 bf16"),
        # an odd number of positions, groups of ten channels, a gradient for each of twelve runs of points
        dict(_norm(96, 255, 320, 32, train=True, runs=12), name="norm train 96x255x320"),
        # token rows normalised head by head: a point is one row
        dict(_norm(16_384, 1, 4_096, 32, bf16=True, train=True), name="norm train 16384x1x4096 bf16"),
        # large feature maps: a point's groups do not fit a compute unit
        dict(_norm(64, 4_096, 512, 32, bf16=True, train=True), name="norm train 64x4096x512 bf16"),
        # one token on its way through a residual branch
        dict(_dropout(1, 1, 1_024, 0.1, bf16=True), name="dropout 1x1x1024 bf16"),
        # odd sizes, no residual, a bias gradient for each of twelve runs
        dict(_dropout(683, 9, 1_027, 0.25, train=True, residual=False, runs=12), name="dropout train 683x9x1027"),
        # the rows of a large training step
        dict(_dropout(64, 512, 4_096, 0.1, bf16=True, train=True), name="dropout train 64x512x4096 bf16"),
        # the ten classes of the paper's network, the points of one worker
        dict(_loss(320, 10), name="loss 320x10"),
        # a few rows over many classes, the padded ones masked
        dict(_loss(3, 131_072, masked=72), name="loss 3x131072"),
        # as wide as the widest rows of the framework's benchmark
        dict(_loss(4_099, 50_008, bf16=True), name="loss 4099x50008 bf16"),
        # a large step over a large set of classes: an odd number of them
        dict(_loss(8_192, 131_071, bf16=True), name="loss 8192x131071 bf16"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "dropout", "loss"])
    bf16, train = rng.random() < 0.6, rng.random() < 0.6
    if kind == "loss":
        classes = _log_uniform(rng, 2, 200_000)
        rows = max(1, min(65_536, _log_uniform(rng, 1_000, MOST_ELEMENTS // 8) // classes))
        return _loss(rows, classes, bf16, train, masked=rng.choice([0, 0, classes // 20]))
    elements = _log_uniform(rng, 1_000, 134_217_728)
    if kind == "dropout":
        channels = _log_uniform(rng, 8, 12_000)
        positions = _log_uniform(rng, 1, 600)
        points = max(1, min(65_536, elements // (positions * channels)))
        return _dropout(points, positions, channels, round(rng.uniform(0.05, 0.6), 3), bf16, train, rng.random() < 0.6, min(points, rng.choice([1, 1, 5, 12])))
    groups = rng.choice([1, 2, 4, 8, 16, 32])
    channels = groups * max(1, _log_uniform(rng, 8, 4_500) // groups)
    positions = _log_uniform(rng, 1, 5_000)
    points = max(1, min(65_536, elements // (positions * channels)))
    return _norm(points, positions, channels, groups, bf16, train, "silu" if train else rng.choice(["none", "relu", "silu"]), min(points, rng.choice([1, 1, 5, 12])))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng([seed, 5])
    dtype = torch.bfloat16 if case["bf16"] else torch.float32
    state = {"case": case}

    def normal(*shape, dtype=torch.float32):
        return torch.empty(*shape, device="cuda", dtype=dtype).normal_(generator=gen)

    if case["kind"] == "loss":
        N, V = case["rows"], case["classes"]
        x = normal(N, V, dtype=dtype).mul_(3.0)
        if case["masked"]:
            x[:, V - case["masked"]:] = -math.inf
        targets = torch.randint(0, V - case["masked"], (N,), generator=gen, device="cuda")
        targets[torch.rand(N, generator=gen, device="cuda") < 0.05] = -1           # rows without a target
        state.update(x=x, targets=targets, weights=0.5 + torch.rand(N, generator=gen, device="cuda"), loss=torch.empty(N, device="cuda"),
                     lse=torch.empty(N, device="cuda"), dx=torch.empty_like(x) if case["train"] else None)
        return state
    N, P, C = case["points"], case["positions"], case["channels"]
    bounds = np.concatenate([[0], np.sort(rng.integers(0, N + 1, case["runs"] - 1)), [N]]).astype(np.int64)
    member = np.zeros((case["runs"], N), dtype=np.float32)                         # member[r][n]: is point n in run r?
    for r in range(case["runs"]):
        member[r, bounds[r]:bounds[r + 1]] = 1.0
    state.update(bounds=bounds, member=torch.from_numpy(member).cuda())
    x = normal(N, P, C, dtype=dtype)
    state.update(x=x, y=torch.empty_like(x))
    if case["train"]:
        state.update(dy=normal(N, P, C, dtype=dtype), dx=torch.empty_like(x))
    if case["kind"] == "dropout":
        state.update(bias=normal(C), residual=normal(N, P, C, dtype=dtype) if case["residual"] else None, seed=int(rng.integers(1 << 62)),
                     draw=int(rng.integers(1 << 20)), first=int(rng.integers(1 << 33)), dbias=torch.empty(case["runs"], C, device="cuda"))
        return state
    x.mul_((0.5 + torch.rand(C, generator=gen, device="cuda")).to(dtype)).add_((1.0 + 0.3 * normal(C)).to(dtype))
    G = case["groups"]
    state.update(gamma=1.0 + 0.2 * normal(C), beta=0.2 * normal(C), eps=1e-5, mean=torch.empty(N, G, device="cuda"), rstd=torch.empty(N, G, device="cuda"),
                 dgamma=torch.empty(case["runs"], C, device="cuda"), dbeta=torch.empty(case["runs"], C, device="cuda"))
    return state


def run(state):
    return {"norm": _run_norm, "dropout": _run_dropout, "loss": _run_loss}[state["case"]["kind"]](state)


def _run_norm(s):
    case = s["case"]
    if own:
        import paper_1902_01981_amd as cr

        act = {"none": cr.CR_ACT_NONE, "relu": cr.CR_ACT_RELU, "silu": cr.CR_ACT_SILU}[case["activation"]]
        if not case["train"]:
            cr.cr_group_norm_forward(s["x"], s["gamma"], s["beta"], case["groups"], s["y"], eps=s["eps"], activation=act)
            return {"y": s["y"]}
        cr.cr_group_norm_forward(s["x"], s["gamma"], s["beta"], case["groups"], s["y"], s["mean"], s["rstd"], eps=s["eps"], activation=act)
        cr.cr_group_norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["gamma"], s["beta"], case["groups"], s["dx"], s["dgamma"], s["dbeta"],
                                  activation=act, bounds=s["bounds"])
        return {k: s[k] for k in ("y", "mean", "rstd", "dx", "dgamma", "dbeta")}
    N, P, C, G = case["points"], case["positions"], case["channels"], case["groups"]
    x = s["x"].float().view(N, P, G, C // G)
    gamma, beta = s["gamma"].view(G, C // G), s["beta"].view(G, C // G)
    mean = x.mean(dim=(1, 3), keepdim=True)
    h = x - mean
    rstd = torch.rsqrt(h.square().mean(dim=(1, 3), keepdim=True) + s["eps"])
    h = h * rstd
    z = gamma * h + beta
    sig = 1.0 / (1.0 + torch.exp(-z))
    y = {"none": z, "relu": torch.where(z > 0, z, torch.zeros_like(z)), "silu": z * sig}[case["activation"]].to(s["x"].dtype).view(N, P, C)
    if not case["train"]:
        return {"y": y}
    dz = s["dy"].float().view(N, P, G, C // G)
    if case["activation"] == "silu":
        dz = dz * sig * (1.0 + z * (1.0 - sig))
    dgamma = s["member"] @ (dz * h).sum(dim=1).view(N, C)
    dbeta = s["member"] @ dz.sum(dim=1).view(N, C)
    dz = dz * gamma
    dx = rstd * (dz - dz.mean(dim=(1, 3), keepdim=True) - h * (dz * h).mean(dim=(1, 3), keepdim=True))
    return {"y": y, "mean": mean.view(N, G), "rstd": rstd.view(N, G), "dx": dx.to(s["x"].dtype).view(N, P, C), "dgamma": dgamma, "dbeta": dbeta}


def _signed(v):
    """The signed 64-bit integer with the bits of v modulo 2^64."""
    v &= (1 << 64) - 1
    return v - (1 << 64) if v >> 63 else v


def _mixed(z):
    """The mixing function of the splitmix64 generator on signed 64-bit integers (arithmetic wraps; shifts are made logical)."""
    z = (z ^ (z >> 30 & (1 << 34) - 1)) * _signed(MIX[0])
    z = (z ^ (z >> 27 & (1 << 37) - 1)) * _signed(MIX[1])
    return z ^ (z >> 31 & (1 << 33) - 1)


def _run_dropout(s):
    case = s["case"]
    if own:
        import paper_1902_01981_amd as cr

        cr.cr_dropout_forward(s["x"], s["y"], case["rate"], s["seed"], s["draw"], bias=s["bias"], residual=s["residual"], first_point=s["first"])
        if not case["train"]:
            return {"y": s["y"]}
        cr.cr_dropout_backward(s["dy"], s["dx"], case["rate"], s["seed"], s["draw"], dbias=s["dbias"], bounds=s["bounds"], first_point=s["first"])
        return {k: s[k] for k in ("y", "dx", "dbias")}
    N, P, C = case["points"], case["positions"], case["channels"]
    words = -(-C // 4)                                   # four draws of 16 bits each per word
    first = s["first"] * P * words                       # the counter goes on over points, positions and words
    key = _mixed(torch.tensor(_signed(s["seed"] + (s["draw"] + 1) * GOLDEN), device="cuda"))
    z = torch.arange(1, N * P * words + 1, device="cuda").add_(_signed(first)).mul_(_signed(GOLDEN)).add_(key)
    fields = _mixed(z).view(N, P, words, 1) >> torch.tensor([0, 16, 32, 48], device="cuda") & 0xFFFF
    least = round(case["rate"] * 65536)
    keep = fields.view(N, P, 4 * words)[..., :C] >= least
    scale = 65536.0 / (65536 - least)
    zero = torch.zeros((), device="cuda")
    y = torch.where(keep, (s["x"].float() + s["bias"]) * scale, zero)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    y = y.to(s["x"].dtype)
    if not case["train"]:
        return {"y": y}
    dx = torch.where(keep, s["dy"].float() * scale, zero)
    return {"y": y, "dx": dx.to(s["x"].dtype), "dbias": s["member"] @ dx.sum(dim=1)}


def _run_loss(s):
    case = s["case"]
    if own:
        import paper_1902_01981_amd as cr

        cr.cr_softmax_loss(s["x"], s["targets"], s["loss"], lse=s["lse"], dlogits=s["dx"], weights=s["weights"])
        return {k: s[k] for k in ("loss", "lse", "dx") if s[k] is not None}
    x = s["x"].float()
    top = x.amax(dim=1, keepdim=True)
    p = torch.exp(x - top)
    total = p.sum(dim=1, keepdim=True)
    lse = (top + torch.log(total)).view(-1)
    at = s["targets"].clamp(min=0).view(-1, 1)
    weight = torch.where(s["targets"] >= 0, s["weights"], torch.zeros_like(s["weights"]))
    loss = weight * (lse - x.gather(1, at).view(-1))
    if not case["train"]:
        return {"loss": loss, "lse": lse}
    p = p.mul_(weight.view(-1, 1) / total)
    p.scatter_add_(1, at, -weight.view(-1, 1))
    return {"loss": loss, "lse": lse, "dx": p.to(s["x"].dtype)}


def work(case):
    """Bytes and operations the results cannot do without: inputs read once, outputs written once (a training step's two passes: what each reads and
    writes); the operations of the formulas, an exponential or a quotient counted as one, a draw of the mask as eight."""
    e = 2 if case["bf16"] else 4
    if case["kind"] == "loss":
        N, V = case["rows"], case["classes"]
        return {"bytes": e * N * V * (2 if case["train"] else 1) + N * (8 + 4 + 4 + 4), "flops": N * V * (7 if case["train"] else 4)}
    N, C, R = case["points"], case["channels"], case["runs"]
    elements = N * case["positions"] * C
    if case["kind"] == "dropout":
        forward = (3 if case["residual"] else 2) * e * elements + 4 * C
        if not case["train"]:
            return {"bytes": forward, "flops": 12 * elements}
        return {"bytes": forward + 2 * e * elements + 4 * R * C, "flops": 23 * elements}
    if not case["train"]:
        return {"bytes": 2 * e * elements + 8 * C, "flops": 11 * elements}
    return {"bytes": 5 * e * elements + 16 * N * case["groups"] + 16 * C + 8 * R * C, "flops": 31 * elements}


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "dropout": _exact_dropout, "loss": _exact_loss}[case["kind"]](s)


def _exact_norm(s):
    """Point by point or a few at a time; a group's channels side by side, positions below each other."""
    case = s["case"]
    N, P, C, G = case["points"], case["positions"], case["channels"], case["groups"]
    M = P * (C // G)
    out = {"y": []} if not case["train"] else {k: [] for k in ("y", "mean", "rstd", "dx", "gh", "g")}
    gamma, beta = s["gamma"].double(), s["beta"].double()
    step = max(1, (1 << 25) // (P * C))
    for lo in range(0, N, step):
        x = s["x"][lo:lo + step].double()
        n = x.shape[0]

        def over_groups(v):                              # the mean over each group of a point, for each of its channels
            m = v.sum(dim=1).reshape(n, G, -1).sum(dim=2) / M
            return m, m.repeat_interleave(C // G, dim=1)[:, None, :]

        mean, wide = over_groups(x)
        x -= wide
        var, wide = over_groups(x * x)
        x /= torch.sqrt(wide + s["eps"])
        z = torch.addcmul(beta, gamma, x)
        s_z = torch.special.expit(z)
        out["y"].append({"none": z, "relu": z.clamp(min=0), "silu": z * s_z}[case["activation"]])
        if not case["train"]:
            continue
        d = s["dy"][lo:lo + step].double()
        if case["activation"] == "silu":
            d *= s_z + z * s_z * (1 - s_z)
        out["mean"].append(mean)
        out["rstd"].append((var + s["eps"]) ** -0.5)
        out["g"].append(d.sum(dim=1))
        out["gh"].append((d * x).sum(dim=1))
        d *= gamma
        out["dx"].append((d - over_groups(d)[1] - x * over_groups(d * x)[1]) * out["rstd"][-1].repeat_interleave(C // G, dim=1)[:, None, :])
    out = {k: torch.cat(v) for k, v in out.items()}
    if case["train"]:
        b = s["bounds"]
        for name, per_point in (("dgamma", out.pop("gh")), ("dbeta", out.pop("g"))):
            out[name] = torch.stack([per_point[b[r]:b[r + 1]].sum(dim=0) for r in range(case["runs"])])
    return out


def _exact_dropout(s):
    """The mask from unsigned 64-bit words on the host, a word's four 16-bit fields as they lie in memory, lowest first."""
    case = s["case"]
    N, P, C = case["points"], case["positions"], case["channels"]
    words = (C + 3) // 4
    least = int(math.floor(case["rate"] * 65536 + 0.5))
    with np.errstate(over="ignore"):
        def output(start, number):                       # of the splitmix64 stream that starts at `start`
            v = start + (number + np.uint64(1)) * np.uint64(GOLDEN)
            v ^= v >> np.uint64(30)
            v *= np.uint64(MIX[0])
            v ^= v >> np.uint64(27)
            v *= np.uint64(MIX[1])
            return v ^ (v >> np.uint64(31))

        key = output(np.array([s["seed"]], dtype=np.uint64), np.array([s["draw"]], dtype=np.uint64))
        number = np.uint64(s["first"] * P * words % (1 << 64)) + np.arange(N * P * words, dtype=np.uint64)
        fields = output(key, number).view("<u2").reshape(N, P, 4 * words)[:, :, :C]
    keep = torch.from_numpy(np.ascontiguousarray(fields >= least)).cuda()
    by = 1.0 / (1.0 - least / 65536)
    y = (s["x"].double() + s["bias"].double()) * by * keep
    if s["residual"] is not None:
        y += s["residual"].double()
    if not case["train"]:
        return {"y": y}
    dx = s["dy"].double() * by * keep
    b = s["bounds"]
    return {"y": y, "dx": dx, "dbias": torch.stack([dx[b[r]:b[r + 1]].sum(dim=(0, 1)) for r in range(case["runs"])])}


def _exact_loss(s):
    case = s["case"]
    N, V = case["rows"], case["classes"]
    loss, lse = torch.empty(N, dtype=torch.float64, device="cuda"), torch.empty(N, dtype=torch.float64, device="cuda")
    dx = torch.empty(N, V, dtype=torch.float32, device="cuda") if case["train"] else None      # of more bits than the outputs are compared in
    step = max(1, (1 << 26) // V)
    for lo in range(0, N, step):
        x = s["x"][lo:lo + step].double()
        t, w = s["targets"][lo:lo + step], s["weights"][lo:lo + step].double()
        w = w * (t >= 0)
        row = torch.arange(x.shape[0], device="cuda")
        lse[lo:lo + step] = z = torch.logsumexp(x, dim=1)
        loss[lo:lo + step] = w * (z - x[row, t.clamp(min=0)])
        if case["train"]:
            p = torch.exp(x - z[:, None]) * w[:, None]
            p[row, t.clamp(min=0)] -= w
            dx[lo:lo + step] = p
    return {"loss": loss, "lse": lse, "dx": dx} if case["train"] else {"loss": loss, "lse": lse}
