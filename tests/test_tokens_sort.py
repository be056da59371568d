"""The table's gradient where its positions are sorted by many workgroups: digits of three and four passes, workgroups of several tiles, with one run and several.

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
