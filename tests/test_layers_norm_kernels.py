"""Which kernels a group norm takes: the planner, compiled for the host, has to send the shapes below where they are meant to go, so that each kernel and
each of its variants stays tested when the rules are tuned; and what it lays out has to fit the kernels.  On the GPU the same shapes run against the formulas."""
import ctypes
import os
import random
import shutil
import subprocess

import pytest

import paper_1902_01981_amd as cr

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
WRAPPER = r"""
#include "norm_plan.h"
extern "C" void plan(int64_t points, int positions, int channels, int bf16, int groups, int backward, int64_t *out)
{
    const cr::LayerShape s = {points, positions, channels, bf16 != 0};
    const cr::RowsPlan r = cr::rows_plan(s, groups, backward != 0);
    cr::Tiling t = {};
    int kind = 0;
    int64_t length = 0;
    if (!r.lanes) {
        t = cr::tile(s, groups, backward != 0);
        kind = t.deep ? 2 : 1;
        if (!t.k) {
            t = cr::cut(s, groups);
            kind = 3;
        }
    }
    if (backward) {
        const cr::BackwardPlan b = cr::plan_backward(s, groups);
        length = b.length;
        if (b.cut != (kind == 3) || (b.rows.lanes > 0) != (kind == 0)) kind = -1;
    }
    const int64_t v[] = {kind, r.lanes, r.chunks, r.wide, r.down, t.tiles, t.slices, t.unit, t.across, t.down, t.side, t.threads, t.k, t.pieces, t.deep, t.fold, length,
                         kind == 3 ? cr::batch_points(s, t) : 0, kind == 0 ? 0 : cr::most_groups(t, groups)};
    for (int64_t x : v) *out++ = x;
}
"""
NAMES = ["kind", "lanes", "chunks", "wide", "rows_down", "tiles", "slices", "unit", "across", "down", "side", "threads", "k", "pieces", "deep", "fold", "length", "batch",
         "most_groups"]
KINDS = ["rows", "tile", "deep", "pieces"]

# points, positions, channels, groups, bf16; the forward's kernel and the gradient's, with the points of a thread of the deep ones, and their points side by side
CASES = [
    ((2101, 1, 2004, 334, True), "deep 2", "deep 2"), ((4101, 1, 2004, 334, True), "deep 4", "deep 2"), ((4101, 1, 1000, 500, True), "deep 2 side", "deep 2 side"),
    ((8201, 1, 1000, 500, True), "deep 4 side", "deep 2 side"), ((4101, 1, 999, 333, True), "deep 2 side", "tile"), ((30_001, 1, 160, 32, True), "deep 2 side", "deep 2 side"),
    ((2101, 1, 3000, 1, True), "rows", "deep 2"), ((5001, 1, 3000, 1, True), "rows", "deep 4"), ((2101, 5, 384, 128, True), "tile", "deep 2"),
    ((2101, 1, 999, 333, False), "deep 2", "deep 2"), ((4101, 1, 999, 333, False), "deep 4", "deep 2"), ((4101, 1, 384, 128, False), "deep 2 side", "deep 2 side"),
    ((8201, 1, 384, 128, False), "deep 4 side", "deep 2 side"), ((2101, 1, 1000, 500, False), "deep 2", "deep 2"), ((4101, 1, 1000, 500, False), "deep 4", "deep 2"),
    ((30_001, 1, 96, 48, False), "deep 2 side", "deep 2 side"), ((44_267, 1, 96, 48, False), "deep 4 side", "deep 2 side"),
    # groups wider than a workgroup's registers, many points: slices of a group, whose parameters' sums come from every point
    ((301, 1, 4104, 1, True), "tile", "pieces"), ((403, 1, 8192, 1, True), "tile", "pieces"), ((201, 2, 4096, 1, True), "tile", "pieces"),
    ((301, 1, 5001, 1, True), "tile", "pieces"), ((205, 1, 4096, 1, False), "tile", "pieces"), ((203, 1, 9001, 1, False), "pieces", "pieces"),
    ((501, 1, 2047, 1, False), "rows", "rows"), ((303, 1, 4095, 1, True), "rows", "tile"),
]


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    gxx = shutil.which("g++")
    if not gxx or not os.path.exists(os.path.join(ROCM, "include", "hip", "hip_runtime_api.h")):
        pytest.skip("needs a host compiler and the runtime's headers")
    d = tmp_path_factory.mktemp("plan")
    (d / "w.cpp").write_text(WRAPPER)
    subprocess.run([gxx, "-O1", "-std=c++17", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROCM, "include"), "-I",
                    os.path.join(ROOT, "paper_1902_01981_amd", "csrc"), str(d / "w.cpp"), "-o", str(d / "w.so")], check=True)
    lib = ctypes.CDLL(str(d / "w.so"))

    def call(points, positions, channels, groups, bf16, backward):
        out = (ctypes.c_int64 * len(NAMES))()
        lib.plan(ctypes.c_int64(points), positions, channels, int(bf16), groups, int(backward), out)
        return dict(zip(NAMES, out))

    return call


def _said(p):
    kind = KINDS[p["kind"]]
    return kind if kind != "deep" else f"deep {p['deep']}" + (" side" if p["side"] > 1 else "")


@pytest.mark.parametrize("case,forward,gradient", CASES, ids=lambda c: "x".join(map(str, c)) if isinstance(c, tuple) else None)
def test_where_the_shapes_go(plan, case, forward, gradient):
    assert (_said(plan(*case, False)), _said(plan(*case, True))) == (forward, gradient)


def test_every_kind_is_among_them():
    for bf16 in (False, True):
        of_type = [c for c in CASES if c[0][4] == bf16]
        assert {c[1] for c in of_type} >= {"rows", "deep 2", "deep 4", "deep 2 side", "deep 4 side", "tile"}
        assert {c[2] for c in of_type} >= {"deep 2", "deep 2 side", "pieces"}
    assert "deep 4" in {c[2] for c in CASES} and "pieces" in {c[1] for c in CASES}


def test_what_is_laid_out_fits(plan):
    """Seats, registers, LDS, grids and pieces, over shapes of all sizes."""
    rng = random.Random(5)

    def number(most):
        return max(1, int(most ** rng.random()))

    kinds = set()
    for _ in range(20_000):
        groups = number(rng.choice([40, 5000]))
        channels = groups * number(max(1, min(20_000, 200_000 // groups)))
        positions, points, bf16, backward = number(rng.choice([50, 100_000])), number(100_000), rng.random() < 0.5, rng.random() < 0.5
        p = plan(points, positions, channels, groups, bf16, backward)
        cg, vec = channels // groups, 8 if bf16 else 4
        kinds.add((p["kind"], backward))
        where = (points, positions, channels, groups, bf16, backward, p)
        if p["kind"] == 0:
            assert positions == 1 and cg >= vec and p["lanes"] in (1, 2, 4, 8, 16, 32, 64) and (p["chunks"] == 1 or p["lanes"] == 64), where
            assert p["lanes"] * p["chunks"] * vec >= cg and p["chunks"] <= (4 if backward and bf16 else 8) and p["lanes"] * p["wide"] * p["rows_down"] <= 256, where
            assert not backward or p["length"] >= 1, where
            continue
        vec = 1 if channels < vec else vec
        unit = vec
        while cg % unit:
            unit //= 2
        assert 64 <= p["threads"] <= 1024 and p["threads"] % 64 == 0 and p["across"] * p["down"] * p["side"] <= p["threads"] and p["side"] >= 1, where
        assert p["tiles"] <= 65535 and p["threads"] <= (512 if backward or p["deep"] else 1024), where
        if p["slices"] == 1:
            fewest, most = channels // cg // p["tiles"] * cg, -(-groups // p["tiles"]) * cg
        else:
            assert p["tiles"] == groups * p["slices"], where
            fewest, most = cg // p["unit"] // p["slices"] * p["unit"], -(-(cg // p["unit"]) // p["slices"]) * p["unit"]
        assert vec <= fewest and most <= p["across"] * vec, where                        # a chunk lies in its tile, and the tile's in its seats
        assert p["most_groups"] == (1 if p["slices"] > 1 else -(-groups // p["tiles"])), where
        values, tables = vec // unit, 2 * p["side"] * p["most_groups"]
        at_once = max(p["deep"], 1)
        lds = 4 * at_once * (p["threads"] * values * (2 if backward else 1) + tables)
        assert max(lds, 4 * p["threads"] * vec if backward else 0) <= 64 << 10, where
        if p["fold"]:
            assert p["across"] <= 32 and 64 % p["across"] == 0 and p["across"] * p["down"] % 64 == 0, where
        if p["kind"] == 3:
            assert p["pieces"] * p["down"] * p["k"] >= positions > (p["pieces"] - 1) * p["down"] * p["k"] and p["k"] in (8, 16, 32, 64), where
            assert 1 <= p["batch"] <= points and (p["batch"] == 1 or p["batch"] * p["pieces"] <= 1 << 22), where
        else:
            assert p["down"] * p["k"] >= positions and p["k"] in (1, 2, 4, 8) and (not p["deep"] or p["k"] == 1 and p["deep"] in (2, 4)), where
            assert not (backward and p["deep"] == 4 and values > 1), where
    assert kinds == {(k, b) for k in range(4) for b in (False, True)}


@pytest.mark.gpu
@pytest.mark.parametrize("case", [c[0] for c in CASES], ids=lambda c: "x".join(map(str, c)))
def test_against_the_formulas(case):
    from test_layers_norm import _bounds, _check_backward, _check_forward, _parameters, _run, _x

    N, P, C, G, bf16 = case
    dtype, kind = (torch.bfloat16 if bf16 else torch.float32), ("silu" if N % 4 == 1 else "none")
    x, dy = _x((N, P, C), dtype, 71), _x((N, P, C), dtype, 72, offset=0.1)
    gamma, beta = _parameters(C, 73)
    bounds = _bounds(N, 4, 74)
    out = _run(x, dy, gamma, beta, G, kind, bounds)
    y, mean, rstd, dx, dgamma, dbeta = out
    _check_forward(x, gamma, beta, G, kind, y, mean, rstd)
    _check_backward(dy, x, mean, rstd, gamma, beta, G, kind, bounds, dx, dgamma, dbeta)
    assert all(torch.equal(a, b) for a, b in zip(_run(x, dy, gamma, beta, G, kind, bounds), out))
    over_x, over_dy = x.clone(), dy.clone()              # in place
    cr.cr_group_norm_forward(over_x, gamma, beta, G, over_x, activation=("none", "relu", "silu").index(kind))
    cr.cr_group_norm_backward(over_dy, x, mean, rstd, gamma, beta, G, over_dy, activation=("none", "relu", "silu").index(kind))
    assert torch.equal(over_x, y) and torch.equal(over_dy, dx)
