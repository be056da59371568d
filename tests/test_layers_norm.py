"""Group norm with an activation against its formulas in 64 bits.

What may differ, in units of u = 2^-24: mean, variance and the sums of the gradient are sums of up to 2^18 terms, added up in parts; their
errors stay far below 64 u of the sum of the terms' sizes.  h and z inherit the mean's error times rstd.  The result is rounded once more to
its type."""
import numpy as np
import pytest

import paper_1902_01981_amd as cr
from _layers import ACTS, HALF_ULP, U, norm_backward, norm_forward, wide

torch = pytest.importorskip("torch")
ROUNDS = 64.0

# points, positions, channels, groups: one value per group; groups of less than a load, of odd sizes, across loads; rows of odd lengths; a point that
# fits a few threads, one workgroup, none; points in numbers
SHAPES = [(1, 1, 1, 1), (1, 1, 8, 8), (2, 1, 64, 4), (3, 5, 6, 2), (1, 64, 64, 8), (2, 7, 10, 10), (5, 3, 33, 11), (4, 49, 96, 32), (3, 17, 1027, 1),
          (2, 255, 320, 32), (7, 1, 4096, 32), (130, 1, 257, 1), (300, 4, 24, 3), (2, 1024, 16, 4), (1, 5000, 12, 4), (2, 4096, 64, 32), (1, 3000, 520, 5),
          (40, 9, 200, 25), (1, 40, 4104, 3), (1000, 1, 8, 2), (1, 30001, 8, 1), (2, 9, 20_000, 4), (1, 2, 70_000, 7)]


def _x(shape, dtype, seed, offset=0.5):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(*shape, generator=gen) * (0.5 + torch.rand(shape[-1], generator=gen)) + offset
    return x.to(dtype).cuda()


def _parameters(C, seed):
    gen = torch.Generator().manual_seed(seed + 1)
    return (1 + 0.3 * torch.randn(C, generator=gen)).cuda(), (0.3 * torch.randn(C, generator=gen)).cuda()


def _bounds(N, runs, seed):
    rng = np.random.default_rng(seed)
    return np.concatenate([[0], np.sort(rng.integers(0, N + 1, runs - 1)), [N]]).astype(np.int64)


def _check_forward(x, gamma, beta, groups, kind, y, mean, rstd, eps=1e-5):
    C = x.shape[-1]
    x64 = wide(x).reshape(x.shape[0], -1, C)
    g64, b64 = (torch.ones(C, dtype=torch.float64) if gamma is None else wide(gamma)), (torch.zeros(C, dtype=torch.float64) if beta is None else wide(beta))
    want, m, r = norm_forward(x64, g64, b64, groups, eps, kind)
    most = x64.abs().amax(dim=1).reshape(x.shape[0], groups, -1).amax(dim=2)             # of a group
    if mean is not None:
        assert (wide(mean) - m).abs().sub(ROUNDS * U * most).max() <= 0
        assert ((wide(rstd) - r).abs() / r).sub(ROUNDS * U * (1 + (most * r) ** 2 / 16)).max() <= 0
    spread = (most * r).repeat_interleave(C // groups, dim=1)[:, None, :]
    z_error = ROUNDS * U * (g64.abs() * spread * (1 + spread / 16) + b64.abs() + 1)
    assert ((wide(y).reshape(want.shape) - want).abs() - 1.1 * z_error - HALF_ULP[x.dtype] * want.abs()).max() <= 0


def _check_backward(dy, x, mean, rstd, gamma, beta, groups, kind, bounds, dx, dgamma, dbeta):
    C = x.shape[-1]
    g64, b64 = (torch.ones(C, dtype=torch.float64) if gamma is None else wide(gamma)), (torch.zeros(C, dtype=torch.float64) if beta is None else wide(beta))
    x64, dy64 = (wide(t).reshape(x.shape[0], -1, C) for t in (x, dy))
    want, dg, db, dg_size, db_size = norm_backward(dy64, x64, wide(mean), wide(rstd), g64, b64, groups, kind, bounds)
    spread = wide(rstd).repeat_interleave(C // groups, dim=1)[:, None, :]
    h = (x64.abs() + wide(mean).abs().repeat_interleave(C // groups, dim=1)[:, None, :]) * spread
    most_h, most_d = h.max(), (g64 * dy64).abs().max()
    if dx is not None:
        # the slope of an activation moves by less than half of what z moves, z by a few u of its terms
        allowed = ROUNDS * U * spread * most_d * (1 + most_h) * (2 + g64.abs().max())
        assert ((wide(dx).reshape(want.shape) - want).abs() - allowed - HALF_ULP[x.dtype] * want.abs()).max() <= 0
    size = dy64.abs().sum(dim=1)
    size = torch.stack([size[bounds[r]:bounds[r + 1]].sum(dim=0) for r in range(len(bounds) - 1)])
    slack = ROUNDS * U * size * (1 + most_h) * (1 + g64.abs().max()) / 8
    if dgamma is not None:
        assert ((wide(dgamma) - dg).abs() - ROUNDS * U * dg_size - slack).max() <= 0
    if dbeta is not None:
        assert ((wide(dbeta) - db).abs() - ROUNDS * U * db_size - slack).max() <= 0


def _run(x, dy, gamma, beta, groups, kind, bounds=None, y=None, dx=None, eps=1e-5):
    N, C = x.shape[0], x.shape[-1]
    runs = 1 if bounds is None else len(bounds) - 1
    out = lambda *s: torch.full(s, float("nan"), device="cuda")                          # noqa: E731
    y = torch.full_like(x, float("nan")) if y is None else y
    dx = torch.full_like(x, float("nan")) if dx is None else dx
    mean, rstd, dgamma, dbeta = out(N, groups), out(N, groups), out(runs, C), out(runs, C)
    cr.cr_group_norm_forward(x, gamma, beta, groups, y, mean, rstd, eps=eps, activation=ACTS.index(kind))
    cr.cr_group_norm_backward(dy, x, mean, rstd, gamma, beta, groups, dx, dgamma, dbeta, activation=ACTS.index(kind), bounds=bounds)
    return y, mean, rstd, dx, dgamma, dbeta


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_against_the_formulas(shape, dtype):
    N, P, C, G = shape
    kind = ACTS[(N + P + C + G) % 3]
    x, dy = _x((N, P, C), dtype, 1), _x((N, P, C), dtype, 2, offset=0.1)
    if kind == "relu":                                   # a slope that jumps: keep z away from 0 by more than it can be off
        x = _away_from_the_jump(x, *_parameters(C, 3), G)
    gamma, beta = _parameters(C, 3)
    bounds = _bounds(N, 1 + N % 4, 4)
    y, mean, rstd, dx, dgamma, dbeta = _run(x, dy, gamma, beta, G, kind, bounds)
    _check_forward(x, gamma, beta, G, kind, y, mean, rstd)
    _check_backward(dy, x, mean, rstd, gamma, beta, G, kind, bounds, dx, dgamma, dbeta)
    serving = torch.full_like(x, float("nan"))           # no statistics kept: the same bits
    cr.cr_group_norm_forward(x, gamma, beta, G, serving, activation=ACTS.index(kind))
    assert torch.equal(serving, y)
    again = _run(x, dy, gamma, beta, G, kind, bounds)    # every sum has its order
    assert all(torch.equal(a, b) for a, b in zip(again, (y, mean, rstd, dx, dgamma, dbeta)))


def _away_from_the_jump(x, gamma, beta, groups):
    """x with the values moved whose z is within 1e-2 of 0 (where one move brings another value there, again)."""
    C = x.shape[-1]
    for _ in range(20):
        x64 = wide(x)
        z = norm_forward(x64, wide(gamma), wide(beta), groups, 1e-5, "none")[0]
        near = z.abs() < 1e-2
        if not near.any():
            break
        x = torch.where(near, x64 + 0.25, x64).to(x.dtype).cuda()
    return x


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ACTS)
@pytest.mark.parametrize("shape", [(3, 20, 48, 4), (2, 33, 37, 1), (2, 2500, 64, 8)], ids=lambda s: "x".join(map(str, s)))
def test_without_parameters_and_in_place(shape, kind):
    N, P, C, G = shape
    x, dy = _x((N, P, C), torch.float32, 5), _x((N, P, C), torch.float32, 6, offset=0.0)
    if kind == "relu":
        x = _away_from_the_jump(x, torch.ones(C), torch.zeros(C), G)
    y, mean, rstd, dx, dgamma, dbeta = _run(x, dy, None, None, G, kind)
    _check_forward(x, None, None, G, kind, y, mean, rstd)
    _check_backward(dy, x, mean, rstd, None, None, G, kind, [0, N], dx, dgamma, dbeta)
    over_dy, over_x = dy.clone(), x.clone()
    cr.cr_group_norm_backward(over_dy, x, mean, rstd, None, None, G, over_dy, activation=ACTS.index(kind))
    cr.cr_group_norm_backward(dy, over_x, mean, rstd, None, None, G, over_x, activation=ACTS.index(kind))
    assert torch.equal(over_dy, dx) and torch.equal(over_x, dx)
    over_x = x.clone()
    cr.cr_group_norm_forward(over_x, None, None, G, over_x, activation=ACTS.index(kind))
    assert torch.equal(over_x, y)
    only = torch.full_like(dbeta, float("nan"))          # one of the parameters' gradients, no dx
    cr.cr_group_norm_backward(dy, x, mean, rstd, None, None, G, dbeta=only, activation=ACTS.index(kind))
    assert torch.equal(only, dbeta)
    only.fill_(float("nan"))
    cr.cr_group_norm_backward(dy, x, mean, rstd, None, None, G, dgamma=only, activation=ACTS.index(kind))
    assert torch.equal(only, dgamma)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_strides(dtype):
    """Channels out of wider rows, at an odd element; points inside positions; one point for all; several dimensions of positions."""
    big = _x((6, 10, 45), dtype, 7)
    for x in (big[:, :, 3:39], big[1::2, ::3, 5:41].contiguous().transpose(0, 1), big[:1, :, 1:37].expand(4, 10, 36), big[:, :, :36].view(6, 2, 5, 36)):
        G, C = 6, x.shape[-1]
        gamma, beta = _parameters(C, 8)
        dy = _x(x.shape, dtype, 9, offset=0.0)
        y = torch.empty_strided(x.shape, dy.stride(), dtype=dtype, device="cuda")
        room = torch.full((x.shape[0], x.numel() // x.shape[0] // C, C + 7), 5.0, dtype=dtype, device="cuda")
        dx = room[:, :, 2:2 + C].view(x.shape)           # rows with a gap
        got = _run(x, dy, gamma, beta, G, "silu", y=y, dx=dx)
        want = _run(x.contiguous(), dy, gamma, beta, G, "silu")
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert bool((room[:, :, :2] == 5).all() and (room[:, :, 2 + C:] == 5).all())


@pytest.mark.gpu
def test_a_large_mean():
    """A mean of a thousand deviations: a variance from sums of squares would be lost."""
    x = _x((4, 300, 40), torch.float32, 10, offset=0.0) + 1000.0
    y, mean, rstd = _run(x, torch.zeros_like(x), None, None, 5, "none")[:3]
    _, m, r = norm_forward(wide(x), torch.ones(40).double(), torch.zeros(40).double(), 5, 1e-5, "none")
    assert ((wide(mean) - m).abs() / m).max() <= 4 * U * np.log2(2400)
    assert ((wide(rstd) - r).abs() / r).max() <= 1e-4     # a mean off by 4 u log2(M) of itself moves the variance by the square of 2e-3 ...
    assert (wide(y) - norm_forward(wide(x), torch.ones(40).double(), torch.zeros(40).double(), 5, 1e-5, "none")[0]).abs().max() <= 5e-3   # ... and h by that


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(3, 12, 40, 5), (2, 2100, 64, 4), (9, 1, 36, 4)], ids=lambda s: "x".join(map(str, s)))
def test_values_that_are_not_finite(shape, dtype):
    """They reach their own group of their own point, and the gradients of the parameters of that group's channels."""
    N, P, C, G = shape
    for bad in (float("nan"), float("inf"), -float("inf")):
        x, dy = _x((N, P, C), dtype, 11), _x((N, P, C), dtype, 12)
        clean = _run(x, dy, None, None, G, "silu")
        x[1, P // 2, C // G + 1] = bad                   # in the second group of the second point
        got = _run(x, dy, None, None, G, "silu")
        hit = torch.zeros(N, P, C, dtype=torch.bool, device="cuda")
        hit[1, :, C // G:2 * (C // G)] = True
        for a, b in ((got[0], clean[0]), (got[3], clean[3])):
            assert bool(a[hit].isnan().all()) and torch.equal(a[~hit], b[~hit])
        assert bool(got[1][1, 1].isnan() or got[1][1, 1].isinf()) and bool(got[2][1, 1].isnan())
        columns = hit[1, 0]
        for a, b in ((got[4], clean[4]), (got[5], clean[5])):
            assert bool(a[0, columns].isnan().all()) and torch.equal(a[0, ~columns], b[0, ~columns])


@pytest.mark.gpu
def test_equal_values():
    """A group of one value, and groups of equal values: the variance is 0, h is 0, the gradient is finite."""
    x = torch.full((2, 6, 8), 3.0, device="cuda")
    for G in (2, 8):
        y, mean, rstd, dx, dgamma, dbeta = _run(x, torch.ones_like(x), None, None, G, "none")
        assert bool((y == 0).all()) and bool((mean == 3).all()) and bool((dgamma == 0).all()) and bool((dbeta == 12).all())
        assert ((wide(rstd) - 1e-5 ** -0.5).abs() / 1e-5 ** -0.5).max() <= 4 * U
        assert dx.abs().max() <= 8 * U * 1e-5 ** -0.5
    x = torch.randn(5, 1, 8, device="cuda")
    y, mean, rstd, dx, *_ = _run(x, torch.randn_like(x), None, None, 8, "none")
    assert bool((y == 0).all()) and torch.equal(mean, x.view(5, 8)) and bool((dx == 0).all())


@pytest.mark.gpu
def test_a_gradient_against_differences():
    """<dx, v>, <dgamma, v> and <dbeta, v> against central differences of sum(dy y) in 64 bits."""
    N, P, C, G = 3, 10, 24, 4
    x, dy = _x((N, P, C), torch.float32, 13), _x((N, P, C), torch.float32, 14, offset=0.0)
    gamma, beta = _parameters(C, 15)
    _, _, _, dx, dgamma, dbeta = _run(x, dy, gamma, beta, G, "silu")

    def total(x, g, b):
        return float((norm_forward(x, g, b, G, 1e-5, "silu")[0] * wide(dy)).sum())

    gen = torch.Generator().manual_seed(16)
    step = 1e-5
    for at, grad in ((0, dx), (1, dgamma[0]), (2, dbeta[0])):
        where = [wide(x), wide(gamma), wide(beta)]
        v = torch.randn(where[at].shape, generator=gen, dtype=torch.float64)
        up, down = list(where), list(where)
        up[at], down[at] = where[at] + step * v, where[at] - step * v
        slope = (total(*up) - total(*down)) / (2 * step)
        size = float((wide(grad).abs() * v.abs()).sum())
        assert abs(float((wide(grad) * v).sum()) - slope) <= 1e-5 * size      # the differences' own error: step^2 times third derivatives


@pytest.mark.gpu
def test_points_of_a_holder():
    """A worker that holds some of the points forms the same bits for them as a call over all, and runs are sums of their own points only."""
    x, dy = _x((24, 30, 40), torch.bfloat16, 17), _x((24, 30, 40), torch.bfloat16, 18)
    gamma, beta = _parameters(40, 19)
    bounds = np.array([0, 5, 5, 11, 24])
    y, mean, rstd, dx, dgamma, dbeta = _run(x, dy, gamma, beta, 8, "silu", bounds)
    for r in range(4):
        lo, hi = bounds[r], bounds[r + 1]
        if lo == hi:
            assert bool((dgamma[r] == 0).all()) and bool((dbeta[r] == 0).all())
            continue
        own = _run(x[lo:hi], dy[lo:hi], gamma, beta, 8, "silu")
        assert all(torch.equal(a, b[lo:hi]) for a, b in zip(own[:4], (y, mean, rstd, dx)))
        _check_backward(dy[lo:hi], x[lo:hi], mean[lo:hi], rstd[lo:hi], gamma, beta, 8, "silu", [0, hi - lo], own[3], own[4], own[5])
        for a, b in ((own[4][0], dgamma[r]), (own[5][0], dbeta[r])):
            assert (a - b).abs().max() <= 1e-5 * a.abs().max()


@pytest.mark.gpu
@pytest.mark.parametrize("positions,channels", [(3, 20), (700, 72)])
def test_many_runs(positions, channels):
    """More runs than a launch takes, most of one point, some of none."""
    N = 400
    x, dy = _x((N, positions, channels), torch.float32, 20), _x((N, positions, channels), torch.float32, 21)
    bounds = np.sort(np.concatenate([np.arange(N + 1), [7, 7, 200, 400, 400]]))
    y, mean, rstd, dx, dgamma, dbeta = _run(x, dy, None, None, 4, "silu", bounds)
    _check_backward(dy, x, mean, rstd, None, None, 4, "silu", bounds, dx, dgamma, dbeta)


@pytest.mark.gpu
def test_no_points():
    x = torch.empty(0, 3, 8, device="cuda")
    y, mean, rstd, dx, dgamma, dbeta = _run(x, x, None, None, 2, "relu", np.array([0, 0, 0]))
    assert bool((dgamma == 0).all()) and bool((dbeta == 0).all()) and dgamma.shape == (2, 8)


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    """Two points more than 2^32 elements apart."""
    block = torch.empty((1 << 32) + 4096, dtype=torch.bfloat16, device="cuda")
    x = block.as_strided((2, 8, 64), (1 << 32, 64, 1))
    x.copy_(_x((2, 8, 64), torch.bfloat16, 22))
    dy = _x((2, 8, 64), torch.bfloat16, 23)
    got, want = _run(x, dy, None, None, 8, "silu"), _run(x.contiguous(), dy, None, None, 8, "silu")
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(2, 12, 40, 5), (3, 3000, 64, 4), (50, 40, 32, 4)], ids=lambda s: "x".join(map(str, s)))
def test_in_a_graph(shape):
    """Captured once, replayed on new contents, with eager work in between."""
    N, P, C, G = shape
    x, dy = _x((N, P, C), torch.bfloat16, 24), _x((N, P, C), torch.bfloat16, 25)
    gamma, beta = _parameters(C, 26)
    bounds = np.array([0, 1, N])
    _run(x, dy, gamma, beta, G, "silu", bounds)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = _run(x, dy, gamma, beta, G, "silu", bounds)
    for k in range(3):
        x.copy_(_x((N, P, C), torch.bfloat16, 30 + k))
        for t in captured:
            t.fill_(7.0)
        graph.replay()
        eager = _run(x, dy, gamma, beta, G, "silu", bounds)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, eager))


@pytest.mark.gpu
def test_on_another_stream():
    x, dy = _x((8, 1500, 64), torch.bfloat16, 27), _x((8, 1500, 64), torch.bfloat16, 28)
    want = _run(x, dy, None, None, 8, "silu")
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        got = _run(x, dy, None, None, 8, "silu")
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
