"""The table's gradient where its positions are sorted by many workgroups: digits of three and four passes, workgroups of several tiles, with one run and several, many runs;
and the largest shapes.

What may differ is what test_tokens_embedding.py says: sums of at most 256 terms in 32 bits, and three more roundings."""
import numpy as np
import pytest

import paper_1902_01981_amd as cr
from _layers import U, wide
from test_tokens_embedding import MOST, _backward, _check_gradient, _inputs

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16]


@pytest.mark.parametrize("positions", [699_050, 699_051, 1_500_001])
def test_tiles(positions):
    """256 workgroups whose tile is full, but for two positions; one position more than those hold, so that each has a second tile; several tiles."""
    points, vocabulary = 3, 1000
    tokens, _, dy = _inputs(points, positions, 1, vocabulary, torch.bfloat16, torch.float32, seed=5)
    for bounds in ([0, 3], [0, 1, 1, 3]):
        _check_gradient(_backward(dy, tokens, vocabulary, 1.0, bounds), dy, tokens, 1.0, bounds)


def _check_cells(dtable, dy, tokens, bounds):
    """The rows that positions have against sums in 64 bits, all others are 0: for tables whose gradient in 64 bits would not fit the host."""
    R, V, C = dtable.shape
    t, d = tokens.cpu().reshape(-1).numpy(), wide(dy).reshape(-1, C)
    run = np.repeat(np.searchsorted(np.asarray(bounds), np.arange(tokens.shape[0]), side="right") - 1, tokens.shape[1])
    known = (t >= 0) & (t < V)
    cells, which, counts = np.unique(run[known] * V + t[known], return_inverse=True, return_counts=True)
    which, d = torch.from_numpy(which.reshape(-1)), d[torch.from_numpy(known)]
    want, size = torch.zeros(len(cells), C, dtype=torch.float64), torch.zeros(len(cells), C, dtype=torch.float64)
    want.index_add_(0, which, d)
    size.index_add_(0, which, d.abs())
    at = torch.from_numpy(cells).cuda()
    flat = dtable.view(R * V, C)
    got = wide(flat[at])
    allowed = size * (torch.from_numpy(counts).clamp(max=MOST)[:, None] + 3) * U * 1.0001
    assert ((got - want).abs() - allowed).max() <= 0
    flat[at] = 0.0
    assert int(torch.count_nonzero(flat)) == 0


# numbers up to the vocabulary, which stands for no token: two passes of nine bits, three of seven, four of seven and of eight; on both sides of a pass
@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("vocabulary", [511, 512, 262_143, 262_144, (1 << 27) - 1, 1 << 27, 1 << 28])
def test_passes(vocabulary, dtype):
    points, positions = 30, 701
    gen = torch.Generator().manual_seed(vocabulary % 1009)
    # tokens from all over the vocabulary, a few very often, the first and last ones, none, and some of no row
    tokens = torch.randint(0, vocabulary, (points, positions), generator=gen)
    often = torch.rand(points, positions, generator=gen) < 0.3
    tokens[often] = (torch.rand(int(often.sum()), generator=gen) ** 3 * 40).long() * (vocabulary // 41)
    tokens[torch.rand(points, positions, generator=gen) < 0.05] = -1
    tokens[torch.rand(points, positions, generator=gen) < 0.05] = vocabulary
    tokens[torch.rand(points, positions, generator=gen) < 0.02] = vocabulary - 1
    tokens[torch.rand(points, positions, generator=gen) < 0.02] = 0
    channels = 1 if vocabulary > 1 << 20 else 24
    dy = torch.randn(points, positions, channels, generator=gen).to(dtype).cuda()
    dy[(tokens < 0) | (tokens >= vocabulary)] = float("nan")             # without influence
    tokens = tokens.cuda()
    clean = torch.where(dy.isnan(), torch.zeros((), dtype=dtype, device="cuda"), dy)
    for bounds in ([0, points], [0, 0, 11, 11, points]):
        runs = len(bounds) - 1
        got = _backward(dy, tokens, vocabulary, 1.0, bounds)
        if runs == 1:
            assert torch.equal(_backward(dy, tokens, vocabulary, 1.0), got)
        _check_cells(got, clean, tokens, bounds)
        del got


def test_passes_in_a_graph():
    """Three passes, replayed with new tokens."""
    points, positions, channels, vocabulary, bounds = 20, 1000, 8, 300_000, [0, 7, 20]
    tokens, _, dy = _inputs(points, positions, channels, vocabulary, torch.bfloat16, torch.float32, seed=1)
    dtable = torch.empty(2, vocabulary, channels, device="cuda")
    cr.cr_embedding_backward(dy, tokens, dtable, bounds=bounds)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cr.cr_embedding_backward(dy, tokens, dtable, bounds=bounds)
    for seed in (2, 3, 4):
        new_tokens, _, new_dy = _inputs(points, positions, channels, vocabulary, torch.bfloat16, torch.float32, seed=seed)
        tokens.copy_(new_tokens), dy.copy_(new_dy), dtable.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(dtable, _backward(dy, tokens, vocabulary, 1.0, bounds))


@pytest.mark.parametrize("runs", [129, 300])
def test_many_runs(runs):
    """Several batches of runs, each of more positions than one workgroup sorts; a batch without points between them."""
    points, positions, channels, vocabulary = 700, 60, 12, 530
    tokens, _, dy = _inputs(points, positions, channels, vocabulary, torch.bfloat16, torch.float32, seed=3)
    rng = np.random.default_rng(runs)
    bounds = np.concatenate([[0, 0], np.sort(rng.integers(0, points + 1, runs - 3)), [points, points]])
    _check_gradient(_backward(dy, tokens, vocabulary, 1.0, bounds), dy, tokens, 1.0, bounds)
    bounds = np.concatenate([[0], np.full(127, 300), np.full(130, 300), np.full(runs, points)])
    _check_gradient(_backward(dy, tokens, vocabulary, 1.0, bounds), dy, tokens, 1.0, bounds)


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("channels", [5, 60, 1030])
def test_strides(channels, dtype):
    """Many positions whose tokens and gradients lie apart, in either order, or are the same for all points."""
    points, positions, vocabulary, bounds = 130, 71, 300, [0, 50, 130]
    tokens, _, dy = _inputs(points, positions, channels, vocabulary, dtype, dtype, seed=8)
    want = _backward(dy, tokens, vocabulary, 1.0, bounds)
    _check_gradient(want, dy, tokens, 1.0, bounds)
    room = torch.full((points, positions + 2, channels + 7), 4.0, dtype=dtype, device="cuda")
    room[:, 1:1 + positions, 3:3 + channels] = dy
    apart = room[:, 1:1 + positions, 3:3 + channels]
    crossed = dy.transpose(0, 1).contiguous().transpose(0, 1)
    long = torch.full((points, positions + 5), 3, device="cuda")
    long[:, 2:2 + positions] = tokens
    for d, t in ((apart, tokens), (crossed, tokens), (dy, long[:, 2:2 + positions]), (apart, tokens.t().contiguous().t())):
        assert torch.equal(_backward(d, t, vocabulary, 1.0, bounds), want)
    one, same = tokens[:1].expand(points, positions), dy[:, :1].expand(points, positions, channels)
    _check_gradient(_backward(same, one, vocabulary, 1.0, bounds), same, one, 1.0, bounds)


def test_the_most_positions():
    """2^31 - 2 positions of one channel, near the limit of points and positions together.  The terms are small whole numbers, whose sums 32 bits hold: all is exact."""
    points, positions, vocabulary = 2, (1 << 30) - 1, 1000
    gen = torch.Generator(device="cuda").manual_seed(1)
    tokens = torch.empty(points, positions, dtype=torch.int64, device="cuda").random_(0, vocabulary + 1, generator=gen)
    tokens -= 1                                          # -1: no token
    dy = torch.empty(points, positions, 1, dtype=torch.bfloat16, device="cuda").random_(0, 4, generator=gen)
    table = torch.randn(vocabulary, 1, generator=gen, device="cuda")
    want = torch.zeros(2, vocabulary + 1, dtype=torch.float64, device="cuda")
    y = torch.full((points, positions, 1), 9.0, dtype=torch.bfloat16, device="cuda")
    cr.cr_embedding_forward(tokens, table, y, scale=0.5)
    rows = torch.cat([table[:, 0] * 0.5, torch.zeros(1, device="cuda")]).bfloat16()            # -1 is the last one
    step = 1 << 27
    for p in range(points):
        for lo in range(0, positions, step):
            t = tokens[p, lo:lo + step]
            want[p] += torch.bincount(t + 1, weights=dy[p, lo:lo + step, 0].double(), minlength=vocabulary + 1)
            assert torch.equal(y[p, lo:lo + step, 0], rows[t])
    del y
    assert float(want.max()) < 2 ** 24
    dtable = torch.full((2, vocabulary, 1), 9.0, device="cuda")
    cr.cr_embedding_backward(dy, tokens, dtable, bounds=[0, 1, 2])
    assert torch.equal(dtable[..., 0].double(), want[:, 1:])
    cr.cr_embedding_backward(dy, tokens, dtable[:1], scale=2.0)
    assert torch.equal(dtable[0, :, 0].double(), 2 * want[:, 1:].sum(dim=0))


@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
def test_the_most_channels(dtype):
    """2^24 and a few less, of cells that lie in a piece and that go on behind it.  Whole numbers again: all is exact."""
    for channels in (1 << 24, (1 << 24) - 3):
        gen = torch.Generator(device="cuda").manual_seed(channels)
        tokens = torch.tensor([[1] * 20 + [0, -1, 3], [1] * 20 + [3, 4, 0]], device="cuda")           # 4: no row
        dy = torch.empty(2, 23, channels, dtype=dtype, device="cuda").random_(0, 4, generator=gen)
        table = torch.empty(4, channels, dtype=dtype, device="cuda").random_(0, 4, generator=gen)
        for bounds in ([0, 2], [0, 1, 2]):
            got = _backward(dy, tokens, 4, 0.5, bounds)
            for r in range(len(bounds) - 1):
                part, t = dy[bounds[r]:bounds[r + 1]].reshape(-1, channels), tokens[bounds[r]:bounds[r + 1]].reshape(-1)
                for v in range(4):
                    assert torch.equal(got[r, v], 0.5 * part[t == v].float().sum(dim=0))
        del got
        y = torch.full_like(dy, 9.0)
        cr.cr_embedding_forward(tokens, table, y, scale=2.0)
        for v in range(4):
            assert bool((y[tokens == v] == 2 * table[v]).all())
        assert bool((y[tokens < 0] == 0).all()) and bool(y[tokens == 4].isnan().all())
        del dy, y, table
