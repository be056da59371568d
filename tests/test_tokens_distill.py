"""The distillation loss and its gradient against the definition in 64 bits.

What may differ, in half steps of 32 bits (U).  exp(d / T) is off by 2 |d| / T + 2 of itself (the unit is rounded), sums of positive terms by at most
ADDS = 192 (a thread adds up 128 of them at most, joins follow); a log share by 3 of its size and ADDS + 16 absolutely, a share by as much of itself.  The loss is a
sum of 128 terms at most, in order of lanes: 8 of their sizes."""
import pytest

import paper_1902_01981_amd as cr
from _layers import HALF_ULP, U, wide
from _tokens import INF, distill, log_softmax

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
NAN = float("nan")
TYPES = [torch.float32, torch.bfloat16]
ADDS = 192

# rows, classes, entries, temperature: as those of the losses of one target
SHAPES = [(1, 1, 1, 1.0), (3, 2, 5, 2.0), (5, 3, 2, 0.5), (4, 7, 7, 1.0), (320, 10, 3, 2.0), (9, 63, 64, 1.5), (70, 64, 20, 4.0), (33, 65, 65, 1.0), (17, 500, 128, 2.0), (6, 1000, 5, 1.0),
          (3, 1027, 20, 3.0), (4, 4096, 64, 1.0), (5, 4097, 100, 2.0), (3, 5001, 127, 0.7), (3, 20_003, 20, 2.0), (2, 50_008, 64, 2.0), (1, 65_536, 8, 1.0), (2, 131_071, 20, 1.5),
          (1, 131_080, 64, 2.0), (1, 250_001, 128, 1.0), (700, 40, 10, 1.0), (300, 257, 16, 2.5), (2000, 7, 2, 1.0)]


def _inputs(rows, classes, top, dtype, seed, spread=3.0):
    gen = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, classes, generator=gen) * spread).to(dtype)
    index = torch.randint(0, classes, (rows, top), generator=gen)                  # several times the same, where classes are few
    z = torch.randn(rows, top, generator=gen) * spread
    index[torch.rand(rows, top, generator=gen) < 0.1] = -1
    index[2::9] = -1
    return x.cuda(), index.cuda(), z.cuda(), (0.5 + torch.rand(rows, generator=gen)).cuda()


def _run(x, index, z, T, weights, dlogits=None, gradient=True):
    loss = torch.full((x.shape[0],), 9.0, device="cuda")
    if gradient and dlogits is None:
        dlogits = torch.full_like(x, 9.0)
    cr.cr_distill_loss(x, index, z, loss, temperature=T, dlogits=dlogits, weights=weights)
    return loss, dlogits


def _same(a, b, allowed):
    odd = ~b.isfinite()
    assert torch.equal(a[odd].isnan(), b[odd].isnan()) and bool(((a[odd] == b[odd]) | b[odd].isnan()).all())
    assert bool(((a - b).abs() <= allowed)[~odd].all()), float(((a - b).abs() - allowed)[~odd].max())


def _check(x, index, z, T, weights, loss, dlogits):
    T = float(torch.tensor(T, dtype=torch.float32))
    x64, z64, i = wide(x), wide(z), index.cpu()
    want_loss, want, size = distill(x64, i, z64, T, None if weights is None else wide(weights))
    most = torch.finfo(torch.float32).max                # a loss past what 32 bits hold is infinite
    want_loss = torch.where(want_loss.abs() > most, want_loss.sign() * INF, want_loss)
    there = (i >= 0) & (z64 != -INF)
    zt = torch.where(there, z64 / T, torch.full_like(z64, -INF))
    most_z = torch.where(zt.isfinite(), zt, torch.full_like(zt, -INF)).amax(dim=1, keepdim=True)
    spread_z = torch.where(zt.isfinite() & (zt - most_z > -100), (zt - most_z).abs(), torch.zeros_like(zt)).amax(dim=1)
    _same(wide(loss), want_loss, size * (2 * (ADDS + 16) + 4 * spread_z + 8) * U + 1e-37)
    if dlogits is None:
        return
    c = torch.where(x64.isfinite(), x64, torch.full_like(x64, -INF)).amax(dim=1, keepdim=True)
    d = torch.where(x64.isfinite() & c.isfinite(), (x64 - c).abs() / T, torch.zeros_like(x64))
    w = torch.ones(x.shape[0], 1).double() if weights is None else wide(weights)[:, None]
    log_p = log_softmax(x64 / T)
    p = torch.where(log_p.isfinite(), torch.exp(log_p), torch.zeros_like(log_p))
    q = torch.zeros_like(p)                              # at the teacher's classes both shares' sizes count
    shares = torch.where(there, torch.softmax(torch.where(there.any(dim=1, keepdim=True), zt, torch.zeros_like(zt)), dim=1), torch.zeros_like(zt))
    q.scatter_add_(1, i.clamp(0, x.shape[1] - 1), torch.where(shares.isfinite(), shares, torch.zeros_like(shares)))
    allowed = w * T * (p * (2 * d + ADDS + 16) + q * (3 * spread_z[:, None] + ADDS + 24)) * U
    _same(wide(dlogits), want, allowed * (1 + 2 * HALF_ULP[x.dtype]) + HALF_ULP[x.dtype] * torch.where(want.isfinite(), want, torch.zeros(()).double()).abs() + 1e-36 * T)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_against_the_definition(shape, dtype):
    rows, classes, top, T = shape
    x, index, z, weights = _inputs(rows, classes, top, dtype, 1)
    loss, dlogits = _run(x, index, z, T, weights)
    _check(x, index, z, T, weights, loss, dlogits)
    without = _run(x, index, z, T, weights, gradient=False)
    assert torch.equal(without[0], loss)
    _check(x, index, z, T, None, *_run(x, index, z, T, None))
    again = _run(x, index, z, T, weights)
    assert torch.equal(again[0], loss) and torch.equal(again[1], dlogits)
    over = x.clone()                                     # the gradient in the logits' place
    in_place = _run(over, index, z, T, weights, dlogits=over)
    assert torch.equal(in_place[0], loss) and torch.equal(over, dlogits)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("classes", [10, 77, 1000, 5003, 140_000])
def test_masks_and_infinities(classes, dtype):
    x, index, z, weights = _inputs(20, classes, 6, dtype, 2)
    index = index.clamp(min=0)
    lowest = torch.finfo(dtype).min
    x[0, classes // 2:] = -INF
    index[0] = index[0] % (classes // 2)
    x[1, :] = -INF                                       # nothing can be
    x[2, index[2, 1]] = -INF                             # a class that the teacher gives a share
    x[3, 1:] = lowest
    x[4, :] = lowest
    x[5, classes - 1] = NAN
    x[6, 0] = INF
    x[7, :] = NAN
    index[8, :] = -1                                     # no entry, whatever the logits are
    x[8, 3] = NAN
    index[9, 1:] = -5
    z[10, 2] = -INF                                      # not there: neither its class nor its number counts
    index[10, 2] = classes + 7
    z[11, :] = -INF
    z[12, 0] = NAN
    z[13, 0] = INF
    z[14, 3], index[14, 3] = NAN, -1                     # not there
    index[15, 5] = classes
    index[16, 0] = 1 << 40
    z[17] = torch.tensor([0.0, -200.0, -300.0, -1000.0, -3e38, -50.0])              # shares of 0
    x[17, index[17, 4]] = -INF if int((index[17] == index[17, 4]).sum()) == 1 else 0.0
    index[18] = index[18, 0]                             # one class six times
    x[19, :-1] = -INF
    index[19] = classes - 1
    for T in (1.0, 2.0, 0.25):
        loss, dlogits = _run(x, index, z, T, weights)
        _check(x, index, z, T, weights, loss, dlogits)
        assert float(loss[1]) == INF and float(loss[2]) == INF and float(loss[8]) == 0 and float(loss[11]) == 0 and bool((dlogits[8] == 0).all()) and bool((dlogits[1] == 0).all())
        assert bool(loss[[12, 13, 15, 16]].isnan().all()) and bool(dlogits[15].isnan().all()) and float(loss[17]) < INF


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("T", [2.0 ** -40, 1e-3, 0.3, 50.0, 2.0 ** 40])
def test_temperatures(T, dtype):
    x, index, z, weights = _inputs(12, 700, 9, dtype, 3)
    loss, dlogits = _run(x, index, z, T, weights)
    if T > 1e-3:
        _check(x, index, z, T, weights, loss, dlogits)
    else:                                                # all on the largest: what is the largest of both has no gradient
        assert bool((loss >= 0).all()) and bool(dlogits.isfinite().all())
        assert float(dlogits.double().sum(dim=1).abs().max()) <= 1e-5 * T


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("classes", [12, 301, 9001])
def test_extreme_logits(classes, dtype):
    for shift, spread in ((3e4, 1.0), (-3e4, 1.0), (0.0, 1e4)):
        x, index, z, weights = _inputs(8, classes, 6, torch.float32, 4, spread)
        x = (wide(x) + shift).to(dtype).cuda()
        _check(x, index, z + shift, 2.0, weights, *_run(x, index, z + shift, 2.0, weights))


def test_a_constant_of_the_teachers_row_changes_nothing():
    """Log probabilities instead of logits."""
    x, index, z, weights = _inputs(20, 3000, 16, torch.float32, 5)
    a, b = _run(x, index, z, 2.0, weights), _run(x, index, z - 4.0, 2.0, weights)
    assert (a[0] - b[0]).abs().max() <= 1e-4 and (a[1] - b[1]).abs().max() <= 1e-5


def test_strides():
    big, index, z, _ = _inputs(30, 800, 25, torch.bfloat16, 6)
    index = torch.where(index >= 500, index - 400, index)
    for x in (big[:, 3:503], big[:1, 7:507].expand(30, 500), big[::2, 1:501]):
        n = x.shape[0]
        for i, zz in ((index[:n], z[:n]), (index[:n, 5:20], z[:n, 5:20]), (index[:1].expand(n, 25), z[:1].expand(n, 25))):
            want = _run(x.contiguous(), i.contiguous(), zz.contiguous(), 2.0, None)
            room = torch.full((n, 511), 4.0, dtype=torch.bfloat16, device="cuda")
            got = _run(x, i, zz, 2.0, None, dlogits=room[:, 5:505])
            assert all(torch.equal(a, b) for a, b in zip(got, want))
            assert bool((room[:, :5] == 4).all()) and bool((room[:, 505:] == 4).all())


@pytest.mark.parametrize("classes", [20, 3000, 150_000])
def test_a_gradient_against_differences(classes):
    x, index, z, weights = _inputs(6, classes, 8, torch.float32, 7)
    dlogits = wide(_run(x, index, z, 1.7, weights)[1])
    v, step = torch.randn(6, classes, generator=torch.Generator().manual_seed(8), dtype=torch.float64), 1e-4
    T = float(torch.tensor(1.7, dtype=torch.float32))
    total = [float(distill(wide(x) + s * step * v, index.cpu(), wide(z), T, wide(weights))[0].sum()) for s in (1, -1)]
    assert abs(float((dlogits * v).sum()) - (total[0] - total[1]) / (2 * step)) <= 1e-5 * float((dlogits.abs() * v.abs()).sum())


def test_the_loss_of_a_student_that_is_the_teacher():
    """All classes given, and the same logits: no divergence, no gradient."""
    x, _, _, _ = _inputs(10, 100, 1, torch.float32, 9)
    index = torch.arange(100, device="cuda").expand(10, 100)
    loss, dlogits = _run(x, index.contiguous(), x, 1.0, None)
    assert loss.abs().max() <= 1e-5 and dlogits.abs().max() <= 1e-6


def test_offsets_beyond_32_bits():
    block = torch.empty((1 << 32) + 30_000, dtype=torch.bfloat16, device="cuda")
    for classes in (600, 20_000, 140_000):
        if classes > 30_000:
            block = torch.empty((1 << 32) + classes, dtype=torch.bfloat16, device="cuda")
        x = block.as_strided((2, classes), (1 << 32, 1))
        values, index, z, weights = _inputs(2, classes, 9, torch.bfloat16, 10)
        x.copy_(values)
        want, got = _run(values, index, z, 2.0, weights), _run(x, index, z, 2.0, weights, dlogits=x)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_no_rows():
    x = torch.empty(0, 12, device="cuda")
    cr.cr_distill_loss(x, torch.empty(0, 3, dtype=torch.int64, device="cuda"), torch.empty(0, 3, device="cuda"), torch.empty(0, device="cuda"), dlogits=x.clone())


@pytest.mark.parametrize("few,many,classes", [(1, 3000, 10), (7, 2000, 1100), (2, 900, 9002), (3, 40, 150_001)])
def test_two_holders_of_the_same_rows(few, many, classes):
    x, index, z, weights = _inputs(many, classes, 20, torch.bfloat16, 11)
    own, all_ = (_run(x[:n], index[:n], z[:n], 2.0, weights[:n]) for n in (few, many))
    assert all(torch.equal(a, b[:few]) for a, b in zip(own, all_))


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,classes", [(5000, 9), (4000, 300), (3000, 4000), (2500, 9000), (700, 70_000)])
def test_many_rows(rows, classes, dtype):
    """What a workgroup carries from one row to the next: rows of every kind after each other, each the bits that it has alone."""
    x, index, z, weights = _inputs(60, classes, 12, dtype, 12)
    x[7], x[8, 0], index[9, 3], z[10, 0] = -INF, NAN, classes, NAN
    index[11] = index[11, 0]
    place = torch.randint(0, 60, (rows,), generator=torch.Generator().manual_seed(13)).cuda()
    want = _run(x, index, z, 2.0, weights)
    wide_x = x[place]
    got = _run(wide_x, index[place], z[place], 2.0, weights[place])
    for a, b in zip(got, want):
        b = b[place]
        assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(), b.nan_to_num())
    over = _run(wide_x, index[place], z[place], 2.0, weights[place], dlogits=wide_x)
    assert torch.equal(over[1].nan_to_num(), got[1].nan_to_num())


@pytest.mark.parametrize("shape", [(100, 10), (20, 5000), (2, 200_000)])
def test_in_a_graph(shape):
    x, index, z, weights = _inputs(*shape, 7, torch.bfloat16, 14)
    _run(x, index, z, 2.0, weights)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = _run(x, index, z, 2.0, weights)
    for k in range(3):
        for a, b in zip((x, index, z, weights), _inputs(*shape, 7, torch.bfloat16, 20 + k)):
            a.copy_(b)
        for t in captured:
            t.fill_(7.0)
        graph.replay()
        eager = _run(x, index, z, 2.0, weights)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, eager))
