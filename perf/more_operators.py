"""The two ends of a network over tokens that trains under coded aggregation, as cases whose time can be taken.

A case is a dict of plain values.  Three operators:

  embed      rows of a table looked up by tokens and scaled; training: with the table's gradient, per run of consecutive points
  log_probs  log probability of a token per row of logits, the entropy and the most probable alternatives; training: with the gradient of the first two
  distill    loss of a row of logits against the largest logits that a teacher gave, training: with its gradient

Where `own` is false they are computed in their plain form, else by the framework's entry points.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

MOST_ELEMENTS = 8192 * 131_071                           # of the largest listed case
PADDED = 0.1                                             # of a batch's positions, about: points end early


def _embed(points, positions, channels, vocabulary, bf16=False, table_bf16=False, train=True, runs=1):
    return {"kind": "embed", "points": points, "positions": positions, "channels": channels, "vocabulary": vocabulary, "bf16": bf16,
            "table_bf16": table_bf16, "train": train, "runs": runs}


def _log_probs(rows, classes, top, bf16=False, train=False, masked=0):
    return {"kind": "log_probs", "rows": rows, "classes": classes, "top": top, "bf16": bf16, "train": train, "masked": masked}


def _distill(rows, classes, top, temperature, bf16=False, train=True):
    return {"kind": "distill", "rows": rows, "classes": classes, "top": top, "temperature": temperature, "bf16": bf16, "train": train}


def listed():
    return [
        # the next token of one sequence on its way into a network: the call itself
        dict(_embed(1, 1, 1_024, 50_008, bf16=True, train=False), name="embed 1x1x1024"),
        # a small step of odd sizes, a gradient for each of twelve runs: the dense gradient is most of it
        dict(_embed(683, 9, 1_027, 5_003, runs=12), name="embed train 683x9x1027"),
        # many short points and narrow rows, frequent tokens many thousand times each
        dict(_embed(8_192, 120, 512, 50_008, bf16=True, table_bf16=True), name="embed train 8192x120x512 bf16"),
        # the rows of a large training step, over a large set of tokens
        dict(_embed(64, 512, 4_096, 131_072, bf16=True, table_bf16=True), name="embed train 64x512x4096 bf16"),
        # one sampled token's probability, with the twenty next to it, the padded classes masked
        dict(_log_probs(1, 131_072, 20, masked=72), name="log_probs 1x131072 top 20"),
        # a policy's gradient: log probabilities and entropies of a batch, no alternatives
        dict(_log_probs(2_047, 32_003, 0, train=True), name="log_probs train 2047x32003"),
        # a teacher's answers written down for its students: many alternatives
        dict(_log_probs(4_099, 50_008, 64, bf16=True), name="log_probs 4099x50008 top 64"),
        # a large step with a few alternatives and the gradient
        dict(_log_probs(8_192, 131_071, 8, bf16=True, train=True), name="log_probs train 8192x131071"),
        # a small student of few classes, a teacher that gave five of them
        dict(_distill(320, 1_003, 5, 2.0), name="distill 320x1003 top 5"),
        # distillation over as wide rows as the framework's benchmark has, from long lists
        dict(_distill(4_099, 50_008, 64, 2.0, bf16=True), name="distill 4099x50008 top 64"),
        # wide rows in 32 bits, the loss alone: validation
        dict(_distill(2_048, 128_000, 100, 1.0, train=False), name="distill 2048x128000 top 100"),
        # a large step: an odd number of classes
        dict(_distill(8_192, 131_071, 20, 1.5, bf16=True), name="distill 8192x131071 top 20"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["embed", "log_probs", "distill"])
    bf16, train = rng.random() < 0.6, rng.random() < 0.6
    if kind == "embed":
        channels, vocabulary = _log_uniform(rng, 8, 6_000), _log_uniform(rng, 20, 200_000)
        vocabulary = min(vocabulary, MOST_ELEMENTS // 4 // channels)
        positions = _log_uniform(rng, 1, 600)
        points = max(1, min(65_536, _log_uniform(rng, 1_000, MOST_ELEMENTS // 8) // (positions * channels)))
        most_runs = max(1, MOST_ELEMENTS // 4 // (vocabulary * channels))
        return _embed(points, positions, channels, vocabulary, bf16, rng.random() < 0.5, train, min(points, most_runs, rng.choice([1, 1, 5, 12])))
    classes = _log_uniform(rng, 3, 200_000)
    rows = max(1, min(65_536, _log_uniform(rng, 1_000, MOST_ELEMENTS // 8) // classes))
    if kind == "log_probs":
        return _log_probs(rows, classes, min(classes, rng.choice([0, 1, 5, 20, 64, 128])), bf16, train, masked=rng.choice([0, 0, classes // 20]))
    return _distill(rows, classes, min(classes, _log_uniform(rng, 1, 128)), round(rng.uniform(0.5, 4.0), 2), bf16, train)


def _frequencies(vocabulary):
    """How often tokens are met: the i-th most frequent one as 1 / (i + 2.7)."""
    f = 1.0 / (np.arange(1, vocabulary + 1) + 2.7)
    return f / f.sum()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = torch.bfloat16 if case["bf16"] else torch.float32

    def normal(*shape, dtype=torch.float32):
        return torch.empty(*shape, device="cuda", dtype=dtype).normal_(generator=gen)

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device="cuda")

    if case["kind"] == "embed":
        return _prepare_embed(case, seed, gen, dtype, normal, uniform)
    N, V, K = case["rows"], case["classes"], case["top"]
    x = normal(N, V, dtype=dtype).mul_(3.0)
    state = {"case": case, "x": x, "dx": torch.empty_like(x) if case["train"] else None}
    if case["kind"] == "log_probs":
        if case["masked"]:
            x[:, V - case["masked"]:] = -math.inf
        tokens = torch.randint(0, V - case["masked"], (N,), generator=gen, device="cuda")
        tokens[uniform(N) < 0.05] = -1                   # rows without a token
        state.update(tokens=tokens, logp=torch.empty(N, device="cuda"), entropy=torch.empty(N, device="cuda"))
        if K:
            state.update(top_index=torch.empty(N, K, dtype=torch.int64, device="cuda"), top_logp=torch.empty(N, K, device="cuda"))
        if case["train"]:
            state.update(largest=torch.empty(N, device="cuda"), log_sum=torch.empty(N, device="cuda"), dlogp=normal(N), dentropy=0.1 * normal(N))
        return state
    # a teacher that is near the student: other noise on the same logits, its K largest; some gave fewer, some rows have none
    index, logits = torch.empty(N, K, dtype=torch.int64, device="cuda"), torch.empty(N, K, device="cuda")
    step = max(1, (1 << 28) // V)
    for lo in range(0, N, step):
        near = x[lo:lo + step].float()
        near.add_(normal(*near.shape))
        logits[lo:lo + step], index[lo:lo + step] = torch.topk(near, K, dim=1)
    given = torch.where(uniform(N) < 0.2, uniform(N), torch.ones((), device="cuda"))
    given[uniform(N) < 0.03] = 0.0
    index[torch.arange(K, device="cuda") >= (given * K).ceil()[:, None]] = -1
    state.update(index=index, logits=logits, weights=0.5 + uniform(N), loss=torch.empty(N, device="cuda"))
    return state


def _prepare_embed(case, seed, gen, dtype, normal, uniform):
    N, P, C, V, R = case["points"], case["positions"], case["channels"], case["vocabulary"], case["runs"]
    rng = np.random.default_rng([seed, 5])
    at = torch.from_numpy(np.cumsum(_frequencies(V))).cuda()
    tokens = torch.searchsorted(at, torch.rand(N, P, generator=gen, device="cuda", dtype=torch.float64)).clamp_(max=V - 1)
    tokens = torch.randperm(V, generator=gen, device="cuda")[tokens]
    lengths = torch.where(uniform(N) < 2 * PADDED, uniform(N), torch.ones((), device="cuda"))
    tokens[torch.arange(P, device="cuda") >= (lengths * P).ceil()[:, None]] = -1
    bounds = np.concatenate([[0], np.sort(rng.integers(0, N + 1, R - 1)), [N]]).astype(np.int64)
    table = normal(V, C, dtype=torch.bfloat16 if case["table_bf16"] else torch.float32)
    state = {"case": case, "tokens": tokens, "table": table, "scale": math.sqrt(C), "bounds": bounds, "y": torch.empty(N, P, C, dtype=dtype, device="cuda"),
             "run": torch.from_numpy(np.searchsorted(bounds, np.arange(N), side="right") - 1).cuda()}
    if case["train"]:
        state.update(dy=normal(N, P, C, dtype=dtype), dtable=torch.empty(R, V, C, device="cuda"))
    return state


def run(state):
    return {"embed": _run_embed, "log_probs": _run_log_probs, "distill": _run_distill}[state["case"]["kind"]](state)


def _run_embed(s):
    case = s["case"]
    if own:
        import paper_1902_01981_amd as cr

        cr.cr_embedding_forward(s["tokens"], s["table"], s["y"], scale=s["scale"])
        if not case["train"]:
            return {"y": s["y"]}
        cr.cr_embedding_backward(s["dy"], s["tokens"], s["dtable"], scale=s["scale"], bounds=s["bounds"])
        return {"y": s["y"], "dtable": s["dtable"]}
    tokens = s["tokens"]
    there = tokens >= 0
    y = s["table"][tokens.clamp(min=0)].float() * s["scale"]
    y = torch.where(there[..., None], y, torch.zeros((), device="cuda")).to(s["y"].dtype)
    if not case["train"]:
        return {"y": y}
    R, V, C = case["runs"], case["vocabulary"], case["channels"]
    place = (s["run"][:, None] * V + tokens)[there]
    # a frequent token's row is a sum of many thousand: in 64 bits
    dtable = torch.zeros(R * V, C, dtype=torch.float64, device="cuda").index_add_(0, place, s["dy"][there].double())
    return {"y": y, "dtable": (dtable * s["scale"]).float().view(R, V, C)}


def _ordered(x):
    """Whole numbers in the order of the values of x (zeros of both signs the same)."""
    bits = (x.float() + 0.0).view(torch.int32).long()
    return torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)


def _run_log_probs(s):
    case = s["case"]
    if own:
        import paper_1902_01981_amd as cr

        cr.cr_log_probs(s["x"], s["tokens"], s["logp"], entropy=s["entropy"], top_index=s.get("top_index"), top_logp=s.get("top_logp"),
                        largest=s.get("largest"), log_sum=s.get("log_sum"))
        out = {k: s[k] for k in ("logp", "entropy", "top_index", "top_logp") if k in s}
        if case["train"]:
            cr.cr_log_probs_backward(s["x"], s["tokens"], s["largest"], s["log_sum"], s["entropy"], s["dlogp"], s["dentropy"], s["dx"])
            out["dx"] = s["dx"]
        return out
    V, K = case["classes"], case["top"]
    x = s["x"].float()
    d = x - x.amax(dim=1, keepdim=True)
    total = torch.exp(d).sum(dim=1, keepdim=True, dtype=torch.float64)
    logp = d - torch.log(total).float()
    p = torch.exp(logp)
    log_p = torch.where(p > 0, logp, torch.zeros((), device="cuda"))               # a class that cannot be adds nothing
    entropy = -(p * log_p).sum(dim=1)
    at, there = s["tokens"].clamp(min=0)[:, None], s["tokens"] >= 0
    zero = torch.zeros((), device="cuda")
    out = {"logp": torch.where(there, logp.gather(1, at)[:, 0], zero), "entropy": entropy}
    if K:
        # the value above, the index's complement below: every number is another, and of equal values the lowest index is the largest
        key = (_ordered(s["x"]) << 28) + (V - 1 - torch.arange(V, device="cuda"))
        index = V - 1 - (torch.topk(key, K, dim=1).values & (1 << 28) - 1)
        there_is = x.gather(1, index) > -math.inf
        out["top_logp"] = torch.where(there_is, logp.gather(1, index), torch.full((), -math.inf, device="cuda"))
        out["top_index"] = torch.where(there_is, index, torch.full((), -1, device="cuda"))
    if case["train"]:
        a, b = torch.where(there, s["dlogp"], zero)[:, None], s["dentropy"][:, None]
        dx = -p * (a + b * (log_p + entropy[:, None]))
        out["dx"] = dx.scatter_add_(1, at, a).to(s["x"].dtype)
    return out


def _run_distill(s):
    case = s["case"]
    if own:
        import paper_1902_01981_amd as cr

        cr.cr_distill_loss(s["x"], s["index"], s["logits"], s["loss"], temperature=case["temperature"], dlogits=s["dx"], weights=s["weights"])
        return {"loss": s["loss"], "dx": s["dx"]} if case["train"] else {"loss": s["loss"]}
    T, zero = case["temperature"], torch.zeros((), device="cuda")
    given = s["index"] >= 0
    at, counts = s["index"].clamp(min=0), given.any(dim=1)
    z = torch.where(given, s["logits"] / T, torch.full((), -math.inf, device="cuda"))
    z = z - torch.where(counts, z.amax(dim=1), zero)[:, None]
    q = torch.exp(z)
    sum_q = torch.where(counts, q.sum(dim=1), torch.ones((), device="cuda"))[:, None]
    q = q / sum_q
    x = s["x"].float() / T
    x = x - x.amax(dim=1, keepdim=True)
    p = torch.exp(x)
    sum_p = p.sum(dim=1, keepdim=True, dtype=torch.float64)
    terms = torch.where(given, q * ((z - torch.log(sum_q)) - (x.gather(1, at) - torch.log(sum_p).float())), zero)
    weight = torch.where(counts, s["weights"], zero)
    loss = weight * T * T * terms.sum(dim=1)
    if not case["train"]:
        return {"loss": loss}
    dx = p * (weight[:, None] * T / sum_p).float()
    dx = dx.scatter_add_(1, at, -weight[:, None] * T * q)
    return {"loss": loss, "dx": dx.to(s["x"].dtype)}


def work(case):
    """Bytes and operations the results cannot do without: inputs read once, outputs written once (a training step of two passes: what each reads and writes);
    the operations of the formulas, an exponential counted as one.  Of a table the rows of the tokens that are met."""
    e = 2 if case["bf16"] else 4
    if case["kind"] == "embed":
        N, C, V, R = case["points"] * case["positions"], case["channels"], case["vocabulary"], case["runs"]
        met = float(-np.expm1(N * (1 - PADDED) * np.log1p(-_frequencies(V))).sum()) if V > 1 else 1.0
        forward = 8 * N + met * C * (2 if case["table_bf16"] else 4) + e * N * C
        if not case["train"]:
            return {"bytes": forward, "flops": N * C}
        return {"bytes": forward + 8 * N + e * N * (1 - PADDED) * C + 4 * R * V * C, "flops": 2 * N * C + met * C}
    N, V, K = case["rows"], case["classes"], case["top"]
    if case["kind"] == "log_probs":
        forward = e * N * V + N * (8 + 4 + 4) + 12 * N * K
        if not case["train"]:
            return {"bytes": forward, "flops": 6 * N * V}
        return {"bytes": forward + 8 * N + 2 * e * N * V + N * (8 + 5 * 4), "flops": 12 * N * V}
    return {"bytes": e * N * V * (2 if case["train"] else 1) + 12 * N * K + N * (4 + 4), "flops": N * V * (7 if case["train"] else 4)}


def exact(case, seed):
    s = prepare(case, seed)
    return {"embed": _exact_embed, "log_probs": _exact_log_probs, "distill": _exact_distill}[case["kind"]](s)


def _exact_embed(s):
    """The gradient from sums along the tokens in their order: what a token's stretch adds to the running sum."""
    case = s["case"]
    N, P, C, V, R = case["points"], case["positions"], case["channels"], case["vocabulary"], case["runs"]
    flat = s["tokens"].reshape(-1)
    y = torch.zeros(N * P, C, dtype=torch.float64, device="cuda")
    used = torch.nonzero(flat != -1)[:, 0]
    y[used] = s["table"].double()[flat[used]] * s["scale"]
    if not case["train"]:
        return {"y": y.view(N, P, C)}
    cell = s["run"].repeat_interleave(P)[used] * V + flat[used]
    cell, order = torch.sort(cell, stable=True)
    met, counts = torch.unique_consecutive(cell, return_counts=True)
    last = torch.cumsum(counts, 0) - 1
    dtable = torch.zeros(R * V, C, dtype=torch.float32, device="cuda")             # of more bits than the outputs are compared in
    step = max(1, (1 << 28) // max(1, len(used)))
    for lo in range(0, C, step):
        run_sum = torch.cumsum(s["dy"].view(N * P, C)[:, lo:lo + step][used][order].double(), dim=0)[last] * s["scale"]
        run_sum[1:] -= run_sum[:-1].clone()
        dtable[met, lo:lo + step] = run_sum.float()
    return {"y": y.view(N, P, C), "dtable": dtable.view(R, V, C)}


def _exact_log_probs(s):
    case = s["case"]
    N, V, K = case["rows"], case["classes"], case["top"]
    names = ["logp", "entropy"] + (["top_logp"] if K else [])
    out = {k: torch.empty((N, K) if k == "top_logp" else (N,), dtype=torch.float64, device="cuda") for k in names}
    if K:
        out["top_index"] = torch.empty(N, K, dtype=torch.int64, device="cuda")
    if case["train"]:
        out["dx"] = torch.empty(N, V, dtype=torch.float32, device="cuda")          # of more bits than the outputs are compared in
    step = max(1, (1 << 26) // V)
    for lo in range(0, N, step):
        x = s["x"][lo:lo + step].double()
        t = s["tokens"][lo:lo + step]
        row, i = torch.arange(x.shape[0], device="cuda"), t.clamp(min=0)
        logp = x - torch.logsumexp(x, dim=1)[:, None]
        h = torch.special.entr(torch.softmax(x, dim=1))
        out["entropy"][lo:lo + step] = H = h.sum(dim=1)
        out["logp"][lo:lo + step] = logp[row, i] * (t >= 0)
        if K:
            ranked, which = torch.sort(x, dim=1, descending=True, stable=True)
            which, ranked = which[:, :K], ranked[:, :K]
            out["top_index"][lo:lo + step] = torch.where(ranked == -math.inf, torch.full_like(which, -1), which)
            out["top_logp"][lo:lo + step] = logp.gather(1, which)
        if case["train"]:
            a, b = s["dlogp"][lo:lo + step].double() * (t >= 0), s["dentropy"][lo:lo + step].double()
            p = torch.exp(logp)
            dx = b[:, None] * (h - p * H[:, None]) - a[:, None] * p                # -p log p is the class's part of the entropy
            dx[row, i] += a
            out["dx"][lo:lo + step] = dx
    return out


def _exact_distill(s):
    """The divergence as cross entropy less entropy."""
    case = s["case"]
    N, V, T = case["rows"], case["classes"], case["temperature"]
    loss = torch.empty(N, dtype=torch.float64, device="cuda")
    dx = torch.empty(N, V, dtype=torch.float32, device="cuda") if case["train"] else None      # of more bits than the outputs are compared in
    step = max(1, (1 << 26) // V)
    for lo in range(0, N, step):
        x, index = s["x"][lo:lo + step].double() / T, s["index"][lo:lo + step]
        none, counts = index < 0, (index >= 0).sum(dim=1) > 0
        q = torch.softmax(s["logits"][lo:lo + step].double().masked_fill(none, -math.inf) / T, dim=1)
        q = torch.where(counts[:, None], q, torch.zeros_like(q))
        w = s["weights"][lo:lo + step].double() * counts
        lse = torch.logsumexp(x, dim=1)
        here = x.gather(1, index.clamp(min=0))
        cross = (q * (lse[:, None] - here)).sum(dim=1)
        loss[lo:lo + step] = w * T ** 2 * (cross - torch.special.entr(q).sum(dim=1))
        if case["train"]:
            p = torch.exp(x - lse[:, None])
            p.scatter_add_(1, index.clamp(min=0), -q)
            dx[lo:lo + step] = p * (w * T)[:, None]
    return {"loss": loss, "dx": dx} if case["train"] else {"loss": loss}
