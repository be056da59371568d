"""Log probabilities, entropy and alternatives, and their gradient, against the definition in 64 bits.

What may differ, in half steps of 32 bits (U).  exp(d) is off by |d| + 2 of itself; a thread adds up 64 of them at most and 16 joins follow, so that a sum of
positive terms is off by at most ADDS = 96 of itself, log S by as much absolutely and a few more.  l = x - c - L: its two differences, and L's error.  The
entropy: L's error, and that of E / S, whose terms p |d| are off by |d| + 2 and whose sum by 2 ADDS.  Indices are equal: ties are decided on the logits."""
import pytest

import paper_1902_01981_amd as cr
from _layers import HALF_ULP, U, wide
from _tokens import INF, log_probs, log_probs_gradient

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
NAN = float("nan")
TYPES = [torch.float32, torch.bfloat16]
ADDS = 96

# rows, classes, alternatives: fewer classes than a load has, all of them as alternatives; a wavefront's rows of one to eight chunks; their border; a workgroup's;
# rows of several slices, whole and not; many rows
SHAPES = [(1, 1, 1), (3, 2, 2), (5, 3, 0), (4, 7, 9), (320, 10, 10), (9, 63, 5), (70, 64, 64), (33, 65, 128), (17, 511, 3), (9, 513, 128), (6, 1025, 20), (3, 2047, 128), (4, 2049, 64),
          (5, 4095, 128), (3, 4096, 1), (4, 4097, 20), (2, 8192, 128), (3, 8193, 64), (2, 16_385, 128), (3, 20_003, 20), (2, 50_008, 64), (1, 131_071, 128), (1, 131_072, 0),
          (2, 300_001, 128), (700, 40, 4), (300, 257, 50), (2001, 7, 2)]


def _logits(rows, classes, dtype, seed, spread=3.0):
    return (torch.randn(rows, classes, generator=torch.Generator().manual_seed(seed)) * spread).to(dtype).cuda()


def _tokens(rows, classes, seed):
    t = torch.randint(0, classes, (rows,), generator=torch.Generator().manual_seed(seed))
    t[1::7] = -1
    return t.cuda()


def _run(x, tokens, top, statistics=True):
    N = x.shape[0]
    out = {k: torch.full((N,), 9.0, device="cuda") for k in ("logp", "entropy") + (("largest", "log_sum") if statistics else ())}
    if tokens is None:
        del out["logp"]
    if top:
        out.update(top_index=torch.full((N, top), 9, device="cuda"), top_logp=torch.full((N, top), 9.0, device="cuda"))
    cr.cr_log_probs(x, tokens, **out)
    return out


def _errors(x64):
    """For each row: c, logits' distances and log probabilities (0 and -infinity for classes that cannot be), and what log probabilities and entropy may be off by."""
    c = torch.where(x64.isfinite(), x64, torch.full_like(x64, -INF)).amax(dim=1, keepdim=True)
    c = torch.where(c.isfinite(), c, torch.zeros_like(c))
    d = x64 - c
    L = torch.logsumexp(d, dim=1)
    L = torch.where(L == -INF, torch.zeros_like(L), L)   # rows of no class: their entropy is 0, and nothing rounds
    l = d - L[:, None]
    p = torch.exp(l)
    size = torch.where(p > 0, d.abs(), torch.zeros_like(d))
    of_L = (ADDS + 8 + 2 * L.abs()) * U
    of_l = (torch.where(l.isfinite(), d.abs() + l.abs(), torch.zeros_like(d))) * U + of_L[:, None]
    of_H = of_L + (p * size * (size + 2 * ADDS + 8)).sum(dim=1) * U + 4 * U * L.abs()
    return l, p, of_l, of_H


def _same(a, b, allowed):
    odd = ~b.isfinite()
    assert torch.equal(a[odd].isnan(), b[odd].isnan()) and bool(((a[odd] == b[odd]) | b[odd].isnan()).all())
    assert bool(((a - b).abs() <= allowed)[~odd].all()), float(((a - b).abs() - allowed)[~odd].max())


def _check(x, tokens, top, out):
    x64 = wide(x)
    logp, entropy, index, values = log_probs(x64, None if tokens is None else tokens.cpu(), top)
    l, p, of_l, of_H = _errors(x64)
    if tokens is not None:
        at = tokens.cpu().clamp(0, x.shape[1] - 1)[:, None]
        _same(wide(out["logp"]), logp, of_l.gather(1, at)[:, 0])
    _same(wide(out["entropy"]), entropy, of_H)
    if top:
        assert torch.equal(out["top_index"].cpu(), index)
        _same(wide(out["top_logp"]), values, of_l.gather(1, index.clamp(min=0)))
    if "largest" in out:
        finite = x64.isnan().any(dim=1) | (x64 == INF).any(dim=1)
        want = torch.where(finite, torch.full((), NAN).double(), x64.amax(dim=1))
        _same(wide(out["largest"]), want, torch.zeros(()).double())


def _gradient(x, tokens, out, dlogp, dentropy, dlogits=None):
    dlogits = torch.full_like(x, 9.0) if dlogits is None else dlogits
    cr.cr_log_probs_backward(x, tokens, out["largest"], out["log_sum"], None if dentropy is None else out["entropy"], dlogp, dentropy, dlogits)
    return dlogits


def _check_gradient(x, tokens, dlogp, dentropy, got):
    x64 = wide(x)
    t = None if tokens is None else tokens.cpu()
    a = torch.zeros(x.shape[0]).double() if t is None else torch.where(t >= 0, wide(dlogp), torch.zeros(()).double())
    b = torch.zeros(x.shape[0]).double() if dentropy is None else wide(dentropy)
    want = log_probs_gradient(x64, t, None if t is None else wide(dlogp), None if dentropy is None else wide(dentropy))
    l, p, of_l, of_H = _errors(x64)
    size = torch.where(p > 0, l.abs(), torch.zeros_like(l))
    H = (p * size).sum(dim=1)[:, None]
    a, b = a.abs()[:, None], b.abs()[:, None]
    allowed = p * ((a + b * (H + size)) * (of_l + (size + 12) * U) + b * (of_l + of_H[:, None]))
    if t is not None:
        here = (t >= 0) & (t < x.shape[1])
        allowed[here, t[here]] += 2 * U * a[here, 0]
    allowed = allowed * (1 + 2 * HALF_ULP[x.dtype]) + HALF_ULP[x.dtype] * want.abs() + 1e-36
    _same(wide(got), want, allowed)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_against_the_definition(shape, dtype):
    rows, classes, top = shape
    x, tokens = _logits(rows, classes, dtype, 1), _tokens(rows, classes, 2)
    out = _run(x, tokens, top)
    _check(x, tokens, top, out)
    again = _run(x, tokens, top)
    assert all(torch.equal(out[k], again[k]) for k in out)
    less = _run(x, tokens, 0, statistics=False)
    assert torch.equal(less["logp"], out["logp"]) and torch.equal(less["entropy"], out["entropy"])
    if top > 1:
        fewer = _run(x, None, top // 2)
        assert torch.equal(fewer["top_index"], out["top_index"][:, :top // 2]) and torch.equal(fewer["top_logp"], out["top_logp"][:, :top // 2])


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_gradient(shape, dtype):
    rows, classes, _ = shape
    x, tokens = _logits(rows, classes, dtype, 3), _tokens(rows, classes, 4)
    gen = torch.Generator().manual_seed(5)
    dlogp, dentropy = torch.randn(rows, generator=gen).cuda(), torch.randn(rows, generator=gen).cuda()
    out = _run(x, tokens, 0)
    dx = _gradient(x, tokens, out, dlogp, dentropy)
    _check_gradient(x, tokens, dlogp, dentropy, dx)
    _check_gradient(x, tokens, dlogp, None, _gradient(x, tokens, out, dlogp, None))
    _check_gradient(x, None, None, dentropy, _gradient(x, None, out, None, dentropy))
    over = x.clone()                                     # the gradient in the logits' place
    assert torch.equal(_gradient(over, tokens, out, dlogp, dentropy, over), dx)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("classes", [1, 10, 77, 1000, 3001, 5003, 40_001])
def test_masks_and_infinities(classes, dtype):
    """Classes that cannot be, rows of none, tokens that cannot be, the type's lowest value, NaN and infinity, tokens that are no class."""
    x, tokens = _logits(16, classes, dtype, 6), torch.arange(16).cuda() % classes
    lowest = torch.finfo(dtype).min
    x[0, classes // 2:] = -INF
    x[1, :] = -INF
    x[2, int(tokens[2])] = -INF
    x[3, 1:] = lowest
    x[4, :] = lowest
    x[5, classes - 1] = NAN
    x[6, 0] = INF
    x[7, :] = NAN
    x[8, :-1] = -INF
    tokens[8] = classes - 1
    x[9, :] = -INF
    x[9, 0] = NAN
    tokens[10] = classes
    tokens[11] = -100
    x[12, :] = -INF
    tokens[12] = -1
    tokens[13] = 1 << 40
    x[14, :] = -INF
    x[14, classes // 2] = lowest
    x[15, :] = torch.where(x[15] > 0, 0.0, -0.0)         # equal, whatever their sign
    gen = torch.Generator().manual_seed(7)
    dlogp, dentropy = torch.randn(16, generator=gen).cuda(), torch.randn(16, generator=gen).cuda()
    for top in (0, 1, 40, 128):
        out = _run(x, tokens, top)
        _check(x, tokens, top, out)
    assert float(out["entropy"][1]) == 0 and float(out["logp"][1]) == -INF and float(out["logp"][12]) == 0
    assert out["top_index"][15, :min(128, classes)].tolist() == list(range(min(128, classes)))
    dx = _gradient(x, tokens, out, dlogp, dentropy)
    _check_gradient(x, tokens, dlogp, dentropy, dx)
    assert bool((dx[1] == 0).all()) and bool(dx[10].isnan().all()) and bool(dx[13].isnan().all())


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("classes", [300, 1000, 4096, 4097, 9000, 60_000])
def test_ties_and_orders(classes, dtype):
    """All equal; two values; ascending and descending; the largest ones side by side, at the ends, and in one thread's places; few that can be."""
    j = torch.arange(classes)
    rows = [torch.zeros(classes), (j % 2).float(), (j % 97 == 3).float(), j.float() / classes, -j.float() / classes, torch.where(j < 130, 5.0, 0.0), torch.where(j >= classes - 130, 5.0, 0.0),
            torch.where((j // 8) % 256 == 7, 3.0, -1.0) - (j % 8) * 0.25, torch.where(j % 50 == 0, j.float() / classes, -INF), torch.where(j == classes - 1, 1.0, -INF),
            torch.where(j // 64 == 1, 2.0, -INF), 1e-40 * (j % 5).float(), -(j % 7).float() * 1e30]
    x = torch.stack([r.double() for r in rows]).to(dtype).cuda()
    for top in (1, 2, 64, 127, 128):
        _check(x, None, top, _run(x, None, top))


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("classes", [12, 301, 9001])
def test_extreme_logits(classes, dtype):
    """Large values of both signs: nothing overflows, and log probabilities beside large logits are as good as beside small ones."""
    for shift, spread in ((3e4, 1.0), (-3e4, 1.0), (0.0, 1e4)):
        x = (wide(_logits(8, classes, torch.float32, 8, spread)) + shift).to(dtype).cuda()
        tokens = _tokens(8, classes, 9)
        out = _run(x, tokens, 20)
        _check(x, tokens, 20, out)
        ones = torch.ones(8, device="cuda")
        _check_gradient(x, tokens, ones, ones, _gradient(x, tokens, out, ones, ones))


def test_strides():
    """Rows out of wider ones at odd elements, one row for all, gradients into rows with gaps."""
    big, tokens = _logits(30, 800, torch.bfloat16, 10), _tokens(30, 500, 11)
    ones = torch.ones(30, device="cuda")
    for x in (big[:, 3:503], big[:1, 7:507].expand(30, 500), big[::2, 1:501]):
        t, n = tokens[:x.shape[0]], x.shape[0]
        want, got = _run(x.contiguous(), t, 20), _run(x, t, 20)
        assert all(torch.equal(want[k], got[k]) for k in want)
        room = torch.full((n, 511), 4.0, dtype=torch.bfloat16, device="cuda")
        assert torch.equal(_gradient(x, t, got, ones[:n], ones[:n], room[:, 5:505]), _gradient(x.contiguous(), t, got, ones[:n], ones[:n]))
        assert bool((room[:, :5] == 4).all()) and bool((room[:, 505:] == 4).all())


def test_offsets_beyond_32_bits():
    block = torch.empty((1 << 32) + 30_000, dtype=torch.bfloat16, device="cuda")
    for classes in (600, 20_000):
        x = block.as_strided((2, classes), (1 << 32, 1))
        x.copy_(_logits(2, classes, torch.bfloat16, 12))
        tokens, ones = torch.tensor([5, 9], device="cuda"), torch.ones(2, device="cuda")
        want, got = _run(x.contiguous(), tokens, 30), _run(x, tokens, 30)
        assert all(torch.equal(want[k], got[k]) for k in want)
        dx = _gradient(x.contiguous(), tokens, want, ones, ones)
        assert torch.equal(_gradient(x, tokens, got, ones, ones, x), dx)


@pytest.mark.parametrize("classes", [20, 3000, 50_000])
def test_a_gradient_against_differences(classes):
    """<dlogits, v> against central differences of the weighted sum of log probabilities and entropies, in 64 bits."""
    x, tokens = _logits(6, classes, torch.float32, 13), _tokens(6, classes, 14)
    gen = torch.Generator().manual_seed(15)
    a, b = torch.randn(6, generator=gen), torch.randn(6, generator=gen)
    dx = wide(_gradient(x, tokens, _run(x, tokens, 0), a.cuda(), b.cuda()))
    v, step = torch.randn(6, classes, generator=gen, dtype=torch.float64), 1e-4
    total = []
    for s in (1, -1):
        logp, entropy, _, _ = log_probs(wide(x) + s * step * v, tokens.cpu(), 0)
        total.append(float((a.double() * logp + b.double() * entropy).sum()))
    assert abs(float((dx * v).sum()) - (total[0] - total[1]) / (2 * step)) <= 1e-5 * float((dx.abs() * v.abs()).sum()) + 1e-7


def test_no_rows():
    x, none = torch.empty(0, 12, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    _run(x, none, 5)
    cr.cr_log_probs_backward(x, none, *(torch.empty(0, device="cuda") for _ in range(5)), x.clone())


@pytest.mark.parametrize("few,many,classes", [(1, 3000, 10), (7, 2000, 1100), (2, 900, 9002), (3, 40, 150_001)])
def test_two_holders_of_the_same_rows(few, many, classes):
    x, tokens = _logits(many, classes, torch.bfloat16, 16), _tokens(many, classes, 17)
    own, all_ = _run(x[:few], tokens[:few], 30), _run(x, tokens, 30)
    assert all(torch.equal(own[k], all_[k][:few]) for k in own)
    ones = torch.ones(many, device="cuda")
    assert torch.equal(_gradient(x[:few], tokens[:few], own, ones[:few], ones[:few]), _gradient(x, tokens, all_, ones, ones)[:few])


def test_rows_of_several_batches():
    """More rows of several slices than the workspace has room for at once."""
    x, tokens = _logits(3, 140_000, torch.bfloat16, 18), _tokens(3, 140_000, 19)
    rows = 9000
    need, one = (cr.cr_log_probs_workspace_bytes(n, 140_000, cr.CR_BF16, 128) for n in (rows, 1))
    assert need < rows * one
    place = torch.arange(rows, device="cuda") % 3
    wide_x = x[place]
    want, got = _run(x, tokens, 128), _run(wide_x, tokens[place], 128)
    assert all(torch.equal(want[k][place], got[k]) for k in want)


@pytest.mark.parametrize("shape", [(100, 10, 3), (20, 5000, 64), (2, 200_000, 128)])
def test_in_a_graph(shape):
    rows, classes, top = shape
    x, tokens = _logits(rows, classes, torch.bfloat16, 20), _tokens(rows, classes, 21)
    ones = torch.ones(rows, device="cuda")
    _run(x, tokens, top)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = _run(x, tokens, top)
        dx = _gradient(x, tokens, captured, ones, ones)
    for k in range(3):
        x.copy_(_logits(rows, classes, torch.bfloat16, 30 + k))
        for t in captured.values():
            t.fill_(7)
        graph.replay()
        eager = _run(x, tokens, top)
        torch.cuda.synchronize()
        assert all(torch.equal(captured[n], eager[n]) for n in eager)
        assert torch.equal(dx, _gradient(x, tokens, eager, ones, ones))
