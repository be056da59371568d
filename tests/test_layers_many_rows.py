"""The layers where a wavefront or a workgroup goes through many points or rows: what it carries from one to the next, and what it reads ahead.

The bounds are those of the tests of each layer; where a call on a part of the rows has to give the same bits, no bound is needed."""
import numpy as np
import pytest

import paper_1902_01981_amd as cr
from _layers import ACTS, HALF_ULP, U, kept, wide
from test_layers_norm import _check_backward, _check_forward, _away_from_the_jump, _bounds, _parameters, _run, _x

torch = pytest.importorskip("torch")

# points, positions, channels, groups: several points of few positions to a thread, groups of whole loads, halves, quarters, odd; groups of 5 to 8 chunks a lane
NORM = [(4100, 2, 640, 32), (4100, 2, 320, 10), (4200, 3, 300, 100), (4100, 1, 2004, 334), (2100, 1, 3000, 1), (2100, 1, 2999, 1), (2100, 4, 251, 1), (2100, 5, 384, 128), (2100, 5, 387, 43), (4200, 17, 90, 2),
        (600, 20, 256, 32), (700, 1, 3001, 1), (300, 1, 1250, 1), (300, 1, 1501, 1), (300, 1, 1800, 1), (300, 1, 2040, 1), (300, 1, 2500, 1), (300, 1, 3500, 1),
        (300, 1, 4090, 1)]
# a wavefront per row, twice around; workgroups of 8 and 16 chunks a thread
LOSS = [(7300, 9), (7300, 517), (7300, 1100), (3200, 4201), (2100, 9002), (600, 40_001), (600, 66_001)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", NORM, ids=lambda s: "x".join(map(str, s)))
def test_norm(shape, dtype):
    N, P, C, G = shape
    kind = ACTS[(N // 100 + P + C + G) % 3]
    x, dy = _x((N, P, C), dtype, 21), _x((N, P, C), dtype, 22, offset=0.1)
    gamma, beta = _parameters(C, 23)
    if kind == "relu":
        x = _away_from_the_jump(x, gamma, beta, G)
    bounds = _bounds(N, 3, 24)
    y, mean, rstd, dx, dgamma, dbeta = _run(x, dy, gamma, beta, G, kind, bounds)
    _check_forward(x, gamma, beta, G, kind, y, mean, rstd)
    _check_backward(dy, x, mean, rstd, gamma, beta, G, kind, bounds, dx, dgamma, dbeta)
    again = _run(x, dy, gamma, beta, G, kind, bounds)
    assert all(torch.equal(a, b) for a, b in zip(again, (y, mean, rstd, dx, dgamma, dbeta)))
    over_x, over_dy = x.clone(), dy.clone()              # in place, where the last chunk of a group is shared
    cr.cr_group_norm_forward(over_x, gamma, beta, G, over_x, activation=ACTS.index(kind))
    cr.cr_group_norm_backward(over_dy, x, mean, rstd, gamma, beta, G, over_dy, activation=ACTS.index(kind))
    assert torch.equal(over_x, y) and torch.equal(over_dy, dx)


@pytest.mark.gpu
def test_one_run_each_and_one_of_all():
    """Sums of runs that one workgroup adds up, and of a run of more pieces than one workgroup adds up: the same terms."""
    for shape, groups in (((40, 9, 200), 25), ((9000, 1, 24), 3), ((70, 2100, 16), 4)):
        x, dy = _x(shape, torch.float32, 31), _x(shape, torch.float32, 32)
        N, P, C = shape
        gamma, beta = _parameters(C, 33)
        for bounds in (np.arange(N + 1), np.array([0, N]), np.array([0, 0, N, N])):
            out = _run(x, dy, gamma, beta, groups, "silu", bounds)
            _check_backward(dy, x, out[1], out[2], gamma, beta, groups, "silu", bounds, *out[3:])
        only = torch.full((N, C), float("nan"), device="cuda")
        each = _run(x, dy, gamma, beta, groups, "silu", np.arange(N + 1))
        cr.cr_group_norm_backward(dy, x, each[1], each[2], gamma, beta, groups, dgamma=only, activation=2, bounds=np.arange(N + 1))
        assert torch.equal(only, each[4])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", LOSS, ids=lambda s: "x".join(map(str, s)))
def test_loss(shape, dtype):
    rows, classes = shape
    gen = torch.Generator(device="cuda").manual_seed(41)
    x = (3 * torch.randn(rows, classes, generator=gen, device="cuda")).to(dtype)
    targets = torch.randint(0, classes, (rows,), generator=gen, device="cuda")
    targets[5::7] = -1
    targets[6::301] = classes
    x[3::50, classes // 3:] = -float("inf")
    x[11::170] = -float("inf")
    targets[3::50] %= classes // 3
    weights = 0.5 + torch.rand(rows, generator=gen, device="cuda")

    def run(a, b, gradient=True, over=None):
        loss, lse = torch.full((2, b - a), float("nan"), device="cuda")
        d = (torch.full_like(x[a:b], 7.0) if over is None else over) if gradient else None
        cr.cr_softmax_loss(x[a:b] if over is None else over, targets[a:b], loss, weights=weights[a:b], lse=lse, dlogits=d)
        return (loss, lse, d) if gradient else (loss, lse)

    def same(p, q):
        return all(torch.equal(s.nan_to_num(123.0), t.nan_to_num(123.0)) and torch.equal(s.isnan(), t.isnan()) for s, t in zip(p, q))

    loss, lse, dlogits = whole = run(0, rows)
    step = 250                                           # few enough rows that nobody has a second one
    parts = [run(a, min(a + step, rows)) for a in range(0, rows, step)]
    assert same(whole, [torch.cat(t) for t in zip(*parts)])
    parts = [run(a, min(a + step, rows), False) for a in range(0, rows, step)]
    assert same(run(0, rows, False), [torch.cat(t) for t in zip(*parts)])
    over = x.clone()
    assert same(run(0, rows, True, over), whole)

    # the definition, in 64 bits; a part of the rows at a time
    t, w = targets.cpu(), wide(weights)
    for a in range(0, rows, step):
        z, at, wt = wide(x[a:a + step]), t[a:a + step], w[a:a + step]
        none = (z == -float("inf")).all(dim=1)
        want_lse = torch.logsumexp(z, dim=1)
        valid = (at >= 0) & (at < classes)
        safe = torch.where(valid, at, torch.zeros_like(at))
        want = torch.where(none, torch.full_like(wt, float("inf")), wt * (want_lse - z.gather(1, safe[:, None])[:, 0]))
        want = torch.where(valid, want, torch.where(at < 0, torch.zeros_like(wt), torch.full_like(wt, float("nan"))))
        most = z.where(z > -float("inf"), torch.zeros_like(z)).abs().amax(dim=1)
        # relative error of an exponential (its argument is off by u of itself, its power of two by 2 u) and of their sum
        error = 32 * U * (2 + most + np.log(classes))
        ok = valid & ~none
        got_loss, got_lse, got = wide(loss[a:a + step]), wide(lse[a:a + step]), wide(dlogits[a:a + step])
        assert ((got_lse - want_lse).abs()[~none] <= error[~none]).all() and torch.equal(got_lse[none], want_lse[none])
        assert ((got_loss - want).abs()[ok] <= (wt * 2 * error)[ok]).all() and torch.equal(got_loss[~ok].nan_to_num(5.0), want[~ok].nan_to_num(5.0))
        share = wt[:, None] * torch.exp(z - want_lse[:, None])
        grad = share.clone()
        grad[torch.arange(len(at)), safe] -= wt
        size = share.clone()
        size[torch.arange(len(at)), safe] += 2 * wt
        bad = (got - grad).abs() - size * 2 * error[:, None] - HALF_ULP[dtype] * grad.abs() - 1e-37
        assert bad[ok].max() <= 0
        assert (got[(at < 0) | (none & valid)] == 0).all() and got[at >= classes].isnan().all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_sliced_rows_in_place(dtype):
    """The gradient in the logits' place, from many workgroups per row: the target's logit is read before any of them replaces it."""
    rows, classes = 40, 150_001
    gen = torch.Generator(device="cuda").manual_seed(51)
    x = torch.randn(rows, classes, generator=gen, device="cuda").to(dtype)
    targets = torch.randint(0, classes, (rows,), generator=gen, device="cuda")
    loss, over = torch.empty(2, rows, device="cuda"), x.clone()
    dlogits = torch.empty_like(x)
    cr.cr_softmax_loss(x, targets, loss[0], dlogits=dlogits)
    cr.cr_softmax_loss(over, targets, loss[1], dlogits=over)
    assert torch.equal(loss[0], loss[1]) and torch.equal(over, dlogits)
    want = torch.logsumexp(x.double(), 1) - x.double().gather(1, targets[:, None])[:, 0]
    assert (loss[0].double() - want).abs().max() <= 2 * 32 * U * (2 + 6 + np.log(classes))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", [(9000, 3, 37), (20_000, 1, 10), (700, 40, 264), (3, 9000, 130)], ids=lambda s: "x".join(map(str, s)))
def test_dropout(shape, dtype):
    N, P, C = shape
    gen = torch.Generator(device="cuda").manual_seed(61)
    big = torch.randn(N, P, C + 3, generator=gen, device="cuda").to(dtype)
    x, dy = big[:, :, 1:C + 1], torch.randn(N, P, C, generator=gen, device="cuda").to(dtype)
    bias, residual = torch.randn(C, generator=gen, device="cuda"), torch.randn(N, P, C, generator=gen, device="cuda").to(dtype)
    mask, scale = kept(np.arange(100, 100 + N), P, C, 0.25, 77, 3)
    y = torch.full((N, P, C), float("nan"), dtype=dtype, device="cuda")
    cr.cr_dropout_forward(x, y, 0.25, 77, 3, bias=bias, residual=residual, first_point=100)
    kept_x = torch.where(mask, wide(x) + wide(bias), torch.zeros(1, dtype=torch.float64)) * scale
    want = wide(residual) + kept_x
    slack = 4 * U * (wide(residual).abs() + 2 * scale * (wide(x).abs() + wide(bias).abs()))
    assert ((wide(y) - want).abs() - slack - HALF_ULP[dtype] * want.abs()).max() <= 0
    bounds = np.array([0, N // 3, N // 3, N])
    dx, dbias = torch.full((N, P, C + 3), 9.0, dtype=dtype, device="cuda"), torch.full((3, C), float("nan"), device="cuda")
    cr.cr_dropout_backward(dy, dx[:, :, 1:C + 1], 0.25, 77, 3, dbias=dbias, bounds=bounds, first_point=100)
    want = torch.where(mask, wide(dy), torch.zeros(1, dtype=torch.float64)) * scale
    assert ((wide(dx[:, :, 1:C + 1]) - want).abs() - 2 * U * want.abs() - HALF_ULP[dtype] * want.abs()).max() <= 0
    assert bool((dx[:, :, 0] == 9).all()) and bool((dx[:, :, C + 1:] == 9).all())
    for r in range(3):
        part = want[bounds[r]:bounds[r + 1]]
        assert ((wide(dbias[r]) - part.sum(dim=(0, 1))).abs() - 64 * U * part.abs().sum(dim=(0, 1))).max() <= 0
