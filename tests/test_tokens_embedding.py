"""Token embedding and its gradient against the definition in 64 bits.

What may differ.  Forward: a product in 32 bits, rounded once more to the type: half a step of each.  Gradient: the terms are exact, a sum of n of them in
32 bits is off by at most n half steps of the sum of their sizes (a piece has no more than 256 of them, pieces are added up in 64 bits and rounded to 32:
two more), and the product with the scale by one."""
import numpy as np
import pytest

import paper_1902_01981_amd as cr
from _layers import HALF_ULP, U, wide
from _tokens import embedding, embedding_gradient

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16]
MOST = 256                                               # terms that are added up in 32 bits

# points, positions, channels, vocabulary: one of everything; fewer channels than a load has; odd ones; tokens met once and thousands of times; vocabularies on
# both sides of a byte's and two bytes' borders, with the number that stands for no token; rows of more than a wavefront's chunks, of many workgroups'
SHAPES = [(1, 1, 1, 1), (1, 1, 1024, 1000), (3, 5, 7, 20), (2, 1, 3, 255), (9, 33, 12, 256), (4, 100, 65, 257), (1, 1000, 16, 3), (700, 9, 37, 5003), (60, 70, 128, 65_535),
          (60, 70, 130, 65_536), (5, 64, 1027, 300), (2, 40, 4099, 50), (33, 500, 24, 70_001), (3, 3, 40_000, 30)]


def _inputs(points, positions, channels, vocabulary, dtype, table_dtype, seed=1, skewed=True):
    gen = torch.Generator().manual_seed(seed)
    u = torch.rand(points, positions, generator=gen, dtype=torch.float64)
    tokens = ((u ** 3 if skewed else u) * vocabulary).long().clamp(max=vocabulary - 1)
    tokens[torch.rand(points, positions, generator=gen) < 0.1] = -1
    table = torch.randn(vocabulary, channels, generator=gen).to(table_dtype)
    dy = torch.randn(points, positions, channels, generator=gen).to(dtype)
    return tokens.cuda(), table.cuda(), dy.cuda()


def _forward(tokens, table, dtype, scale):
    y = torch.full((*tokens.shape, table.shape[1]), 9.0, dtype=dtype, device="cuda")
    cr.cr_embedding_forward(tokens, table, y, scale=scale)
    return y


def _backward(dy, tokens, vocabulary, scale, bounds=None, **more):
    runs = 1 if bounds is None else len(bounds) - 1
    dtable = torch.full((runs, vocabulary, dy.shape[-1]), 9.0, device="cuda")
    cr.cr_embedding_backward(dy, tokens, dtable, scale=scale, bounds=bounds, **more)
    return dtable


def _check_forward(y, tokens, table, scale):
    want, got = embedding(tokens.cpu(), wide(table), scale), wide(y)
    assert torch.equal(want.isnan(), got.isnan())
    there = ~want.isnan()
    allowed = want.abs() * (U + HALF_ULP[y.dtype] * (1 + U)) * 1.0001 + 1e-44
    assert ((want - got).abs() - allowed)[there].max() <= 0 if bool(there.any()) else True


def _check_gradient(dtable, dy, tokens, scale, bounds):
    want, size, count = embedding_gradient(wide(dy), tokens.cpu(), dtable.shape[1], scale, bounds)
    got = wide(dtable)
    allowed = size * (count.clamp(max=MOST) + 3) * U * 1.0001
    assert ((got - want).abs() - allowed).max() <= 0
    assert bool((got[(count == 0).expand_as(got)] == 0).all())


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("table_dtype", TYPES, ids=["table-f32", "table-bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_forward(shape, table_dtype, dtype):
    tokens, table, _ = _inputs(*shape, dtype, table_dtype)
    scale = np.float32(shape[2] ** 0.5).item()
    y = _forward(tokens, table, dtype, scale)
    _check_forward(y, tokens, table, scale)
    assert torch.equal(_forward(tokens, table, dtype, scale), y)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_gradient(shape, dtype):
    points, positions, channels, vocabulary = shape
    tokens, _, dy = _inputs(*shape, dtype, torch.float32, seed=2)
    got = _backward(dy, tokens, vocabulary, 1.5)
    _check_gradient(got, dy, tokens, 1.5, [0, points])
    assert torch.equal(_backward(dy, tokens, vocabulary, 1.5), got)
    bounds = [0, 0, points // 3, points // 3, points // 2, points]
    _check_gradient(_backward(dy, tokens, vocabulary, -0.5, bounds), dy, tokens, -0.5, bounds)


@pytest.mark.parametrize("runs", [127, 128, 129, 300])
def test_many_runs(runs):
    """More runs than one launch takes, empty ones at every border among them."""
    points = 211
    tokens, _, dy = _inputs(points, 6, 20, 70, torch.bfloat16, torch.float32, seed=3)
    rng = np.random.default_rng(runs)
    bounds = np.concatenate([[0, 0], np.sort(rng.integers(0, points + 1, runs - 3)), [points, points]])
    _check_gradient(_backward(dy, tokens, 70, 1.0, bounds), dy, tokens, 1.0, bounds)
    bounds = np.concatenate([np.zeros(runs), [points]]).astype(np.int64)           # all in the last
    _check_gradient(_backward(dy, tokens, 70, 1.0, bounds), dy, tokens, 1.0, bounds)
    bounds = np.concatenate([[0], np.full(runs, points)]).astype(np.int64)         # all in the first
    _check_gradient(_backward(dy, tokens, 70, 1.0, bounds), dy, tokens, 1.0, bounds)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("points,positions,channels", [(300, 101, 8), (40, 50, 520), (1, 70_001, 3)])
def test_one_token_everywhere(points, positions, channels, dtype):
    """A cell of many pieces, alone, beside one position of another, and cut by runs."""
    _, _, dy = _inputs(points, positions, channels, 9, dtype, torch.float32, seed=4)
    tokens = torch.full((points, positions), 5, device="cuda")
    _check_gradient(_backward(dy, tokens, 9, 1.0), dy, tokens, 1.0, [0, points])
    tokens[0, 0], tokens[-1, -1] = 8, 0
    bounds = [0, points // 2, points // 2, points]
    _check_gradient(_backward(dy, tokens, 9, 1.0, bounds), dy, tokens, 1.0, bounds)


@pytest.mark.parametrize("positions", [15, 16, 17, 31, 32, 33, 255, 256, 257, 1023, 1024, 1025, 8191, 8192, 8193, 9217])
def test_lengths_around_pieces_and_tiles(positions):
    for vocabulary in (2, 40, 5000):
        tokens, table, dy = _inputs(1, positions, 5, vocabulary, torch.float32, torch.float32, seed=positions)
        _check_gradient(_backward(dy, tokens, vocabulary, 1.0), dy, tokens, 1.0, [0, 1])
        _check_forward(_forward(tokens, table, torch.float32, 2.0), tokens, table, 2.0)


@pytest.mark.parametrize("positions", [43_691, 349_525, 349_526, 900_001])
def test_many_positions(positions):
    """A tile each for some workgroups of the sort, full ones for 128 of them, twice as many, several tiles each."""
    points, vocabulary = 3, 1000
    tokens, _, dy = _inputs(points, positions, 1, vocabulary, torch.bfloat16, torch.float32, seed=5)
    bounds = [0, 1, 3]
    _check_gradient(_backward(dy, tokens, vocabulary, 1.0, bounds), dy, tokens, 1.0, bounds)


@pytest.mark.parametrize("vocabulary", [1 << 24, (1 << 24) + 5, 1 << 28])
def test_large_vocabularies(vocabulary):
    gen = torch.Generator().manual_seed(6)
    tokens = torch.randint(vocabulary - 40, vocabulary + 2, (5, 60), generator=gen)
    tokens[0, :3] = torch.tensor([0, 1 << 23, 255])
    dy = torch.randn(5, 60, 1, generator=gen).cuda()
    got = _backward(dy, tokens.cuda(), vocabulary, 1.0)[0, :, 0]
    met = torch.unique(tokens[tokens < vocabulary])
    flat, d = tokens.reshape(-1), wide(dy).reshape(-1)
    for t in met.tolist():
        terms = d[flat == t]
        assert abs(float(got[t]) - float(terms.sum())) <= float(terms.abs().sum()) * (len(terms) + 3) * U
    got[met.cuda()] = 0.0
    assert int(torch.count_nonzero(got)) == 0


def test_no_tokens_and_tokens_of_no_row():
    """What they point at has no influence, whatever is there."""
    tokens, table, dy = _inputs(6, 11, 40, 30, torch.bfloat16, torch.float32, seed=7)
    tokens[1, :] = -1
    tokens[2, 3], tokens[3, 0], tokens[5, 10], tokens[5, 9] = 30, 1 << 40, -(1 << 50), (1 << 32) + 3
    bad = (tokens < 0) | (tokens >= 30)
    dy[bad] = float("nan")
    dy[4, 4] = float("inf")
    tokens[4, 4] = 29
    tokens[(tokens == 29) & ~((torch.arange(6).cuda()[:, None] == 4) & (torch.arange(11).cuda()[None] == 4))] = 28
    _check_forward(_forward(tokens, table, torch.bfloat16, 3.0), tokens, table, 3.0)
    got = _backward(dy, tokens, 30, 2.0)
    assert bool((got[0, 29] == float("inf")).all()) and bool(got[0, :29].isfinite().all())
    dy[4, 4] = 0.0
    dy[bad] = 1.0
    assert torch.equal(_backward(dy, tokens, 30, 2.0)[0, :29], got[0, :29])
    nobody = torch.full((6, 11), -7, device="cuda")
    assert bool((_backward(dy, nobody, 30, 2.0) == 0).all()) and bool((_forward(nobody, table, torch.bfloat16, 2.0) == 0).all())


@pytest.mark.parametrize("channels", [6, 700])
def test_many_positions_without_tokens(channels):
    """More positions than one workgroup sorts, whose end, or all of which, have no row: NaN there has no influence, and every row is written."""
    tokens, _, dy = _inputs(40, 500, channels, 60, torch.bfloat16, torch.float32, seed=15)
    tokens[10:, 100:] = -1
    tokens[20:] = torch.where(tokens[20:] == 3, 60, tokens[20:])
    dy[(tokens < 0) | (tokens >= 60)] = float("nan")
    got = _backward(dy, tokens, 60, 1.0, [0, 15, 15, 40])
    assert bool(got.isfinite().all())
    clean = torch.where(dy.isnan(), torch.zeros((), dtype=dy.dtype, device="cuda"), dy)
    _check_gradient(got, clean, tokens, 1.0, [0, 15, 15, 40])
    assert bool((_backward(dy, torch.full_like(tokens, -1), 60, 1.0, [0, 15, 40]) == 0).all())


def test_no_points():
    tokens, table = torch.empty(0, 4, dtype=torch.int64, device="cuda"), torch.ones(10, 6, device="cuda")
    assert _forward(tokens, table, torch.float32, 1.0).shape == (0, 4, 6)
    for bounds in (None, [0, 0, 0], [0] * 200):
        assert bool((_backward(torch.empty(0, 4, 6, device="cuda"), tokens, 10, 1.0, bounds) == 0).all())


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
def test_strides(dtype):
    """Tokens out of longer rows, transposed, of one point for all; outputs and gradients with gaps, transposed, broadcast, at odd elements."""
    points, positions, channels, vocabulary = 13, 21, 44, 90
    tokens, table, dy = _inputs(points, positions, channels, vocabulary, dtype, dtype, seed=8)
    y, g = _forward(tokens, table, dtype, 1.0), _backward(dy, tokens, vocabulary, 1.0)
    long = torch.full((points, positions + 5), 3, device="cuda")
    long[:, 2:2 + positions] = tokens
    turned = tokens.t().contiguous().t()
    room = torch.full((points, positions + 2, channels + 7), 4.0, dtype=dtype, device="cuda")
    for t in (long[:, 2:2 + positions], turned):
        out = room[:, 1:1 + positions, 3:3 + channels]
        cr.cr_embedding_forward(t, table, out)
        assert torch.equal(out, y)
        room[:, 1:1 + positions, 3:3 + channels] = 4.0
        assert bool((room == 4).all())
        crossed = torch.empty(positions, points, channels, dtype=dtype, device="cuda").transpose(0, 1)
        cr.cr_embedding_forward(t, table, crossed)
        assert torch.equal(crossed, y)
        room[:, 1:1 + positions, 3:3 + channels] = dy
        assert torch.equal(_backward(room[:, 1:1 + positions, 3:3 + channels], t, vocabulary, 1.0), g)
        crossed.copy_(dy)
        assert torch.equal(_backward(crossed, t, vocabulary, 1.0), g)
        room.fill_(4.0)
    one = tokens[:1].expand(points, positions)
    _check_forward(_forward(one, table, dtype, 1.0), one, table, 1.0)
    same = dy[:, :1].expand(points, positions, channels)                           # the gradient of a mean over positions
    _check_gradient(_backward(same, one, vocabulary, 1.0), same, one, 1.0, [0, points])
    flat = tokens[:, 0]                                                            # points of one position
    assert torch.equal(_forward(flat, table, dtype, 1.0), y[:, 0])
    _check_gradient(_backward(dy[:, 0], flat, vocabulary, 1.0), dy[:, :1], tokens[:, :1], 1.0, [0, points])
    deep = tokens[:, :20].reshape(points, 4, 5)
    assert torch.equal(_forward(deep, table, dtype, 1.0).view(points, 20, channels), y[:, :20])
    offset = torch.empty(vocabulary * channels + 1, dtype=dtype, device="cuda")[1:].view(vocabulary, channels)
    offset.copy_(table)
    assert torch.equal(_forward(tokens, offset, dtype, 1.0), y)


def test_offsets_beyond_32_bits():
    block = torch.empty((1 << 32) + 4096, dtype=torch.bfloat16, device="cuda")
    tokens, table, dy = _inputs(2, 6, 40, 7, torch.bfloat16, torch.bfloat16, seed=9)
    for far in (block.as_strided((2, 6, 40), (1 << 32, 40, 1)), block.as_strided((6, 2, 40), (40, 1 << 32, 1)).transpose(0, 1)):
        cr.cr_embedding_forward(tokens, table, far)
        assert torch.equal(far, _forward(tokens, table, torch.bfloat16, 1.0))
        far.copy_(dy)
        assert torch.equal(_backward(far, tokens, 7, 1.0), _backward(dy, tokens, 7, 1.0))
    big = block[:70_000 * 61_000].view(70_000, 61_000)                             # a table
    big[69_999] = 2.0
    big[0] = 1.0
    got = _forward(torch.tensor([[69_999, 0]], device="cuda"), big, torch.float32, 1.0)
    assert bool((got[0, 0] == 2).all()) and bool((got[0, 1] == 1).all())


def test_a_gradient_of_more_than_32_bits():
    vocabulary, channels = 70_000, 31_000
    tokens = torch.tensor([[69_999, 3, 69_999]], device="cuda")
    dy = torch.randn(1, 3, channels, generator=torch.Generator().manual_seed(1)).cuda()
    dtable = torch.full((2, vocabulary, channels), 5.0, device="cuda")
    cr.cr_embedding_backward(dy, tokens, dtable, bounds=[0, 0, 1])
    assert torch.equal(dtable[1, 3], dy[0, 1])
    assert (dtable[1, 69_999] - (dy[0, 0] + dy[0, 2])).abs().max() <= 1e-6
    dtable[1, 3], dtable[1, 69_999] = 0.0, 0.0
    assert int(torch.count_nonzero(dtable)) == 0


def test_against_differences():
    """<dtable, v> is the derivative of <y, dy> along v, which is linear."""
    tokens, table, dy = _inputs(20, 30, 50, 40, torch.float32, torch.float32, seed=10)
    dtable = wide(_backward(dy, tokens, 40, 0.7))[0]
    v = torch.randn(40, 50, generator=torch.Generator().manual_seed(11), dtype=torch.float64)
    step = 2.0 ** -4
    there = [float((embedding(tokens.cpu(), wide(table) + s * step * v, 0.7) * wide(dy)).sum()) for s in (1, -1)]
    assert abs(float((dtable * v).sum()) - (there[0] - there[1]) / (2 * step)) <= 1e-5 * float((dtable.abs() * v.abs()).sum())


@pytest.mark.parametrize("shape", [(2, 40, 24, 60), (30, 700, 16, 3000)])
def test_in_a_graph(shape):
    points, positions, channels, vocabulary = shape
    bounds = [0, points // 2, points]
    tokens, table, dy = _inputs(*shape, torch.bfloat16, torch.float32, seed=12)
    y, dtable = torch.empty_like(dy), torch.empty(2, vocabulary, channels, device="cuda")

    def step():
        cr.cr_embedding_forward(tokens, table, y, scale=2.0)
        cr.cr_embedding_backward(dy, tokens, dtable, bounds=bounds)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        new = _inputs(*shape, torch.bfloat16, torch.float32, seed=20 + k)
        for a, b in zip((tokens, table, dy), new):
            a.copy_(b)
        y.fill_(7.0), dtable.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, _forward(tokens, table, torch.bfloat16, 2.0))
        assert torch.equal(dtable, _backward(dy, tokens, vocabulary, 1.0, bounds))


def test_another_stream_with_a_workspace_of_its_own():
    tokens, table, dy = _inputs(40, 60, 96, 500, torch.bfloat16, torch.float32, seed=13)
    want = _backward(dy, tokens, 500, 1.0)
    stream = torch.cuda.Stream()
    need = cr.cr_embedding_workspace_bytes(dy, 500)
    workspace = torch.full((need + 256,), 0xAB, dtype=torch.uint8, device="cuda")
    dtable = torch.full((1, 500, 96), 9.0, device="cuda")
    stream.wait_stream(torch.cuda.current_stream())
    cr.cr_embedding_backward(dy, tokens, dtable, workspace=workspace[:need], stream=stream.cuda_stream)
    stream.synchronize()
    assert torch.equal(dtable, want) and bool((workspace[need:] == 0xAB).all())
    with pytest.raises(ValueError):
        cr.cr_embedding_backward(dy, tokens, dtable, stream=stream.cuda_stream)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
def test_two_holders_of_the_same_points(dtype):
    """What is looked up for a point is the same bits among other points; gradients of runs of the same points are the same up to rounding."""
    tokens, table, dy = _inputs(90, 17, 76, 40, dtype, dtype, seed=14)
    assert torch.equal(_forward(tokens[30:50], table, dtype, 3.0), _forward(tokens, table, dtype, 3.0)[30:50])
    all_ = _backward(dy, tokens, 40, 1.0, [0, 30, 50, 90])[1]
    own = _backward(dy[30:50], tokens[30:50], 40, 1.0)[0]
    _, size, count = embedding_gradient(wide(dy[30:50]), tokens[30:50].cpu(), 40, 1.0, [0, 20])
    assert ((wide(own) - wide(all_)).abs() - 2 * size[0] * (count[0].clamp(max=MOST) + 3) * U).max() <= 0
