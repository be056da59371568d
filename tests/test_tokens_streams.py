"""The layers over tokens as a program calls them: on several streams at once, in graphs that share a workspace, in workspaces that hold anything, at the largest
sizes."""
import pytest

import paper_1902_01981_amd as cr
from _layers import U

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _embed(seed, points=60, positions=200, channels=72, vocabulary=900):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    tokens = torch.randint(-1, vocabulary, (points, positions), generator=gen, device="cuda")
    dy = torch.randn(points, positions, channels, generator=gen, device="cuda").bfloat16()
    out = torch.full((2, vocabulary, channels), 9.0, device="cuda")
    need = cr.cr_embedding_workspace_bytes(dy, vocabulary, [0, points // 3, points])

    def call(workspace=None, stream=None):
        cr.cr_embedding_backward(dy, tokens, out, scale=2.0, bounds=[0, points // 3, points], workspace=workspace, stream=stream)

    return call, [out], need, (tokens, dy)


def _score(seed, rows=30, classes=40_000, top=50):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, classes, generator=gen, device="cuda").bfloat16()
    tokens = torch.randint(0, classes, (rows,), generator=gen, device="cuda")
    logp, entropy, values = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda"), torch.zeros(rows, top, device="cuda")
    index = torch.zeros(rows, top, dtype=torch.int64, device="cuda")

    def call(workspace=None, stream=None):
        cr.cr_log_probs(x, tokens, logp, entropy=entropy, top_index=index, top_logp=values, workspace=workspace, stream=stream)

    return call, [logp, entropy, index, values], cr.cr_log_probs_workspace_bytes(rows, classes, cr.CR_BF16, top), (x, tokens)


def _distil(seed, rows=40, classes=150_000, top=30):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, classes, generator=gen, device="cuda").bfloat16()
    index = torch.randint(-1, classes, (rows, top), generator=gen, device="cuda")
    z = torch.randn(rows, top, generator=gen, device="cuda")
    loss, dx = torch.zeros(rows, device="cuda"), torch.zeros_like(x)

    def call(workspace=None, stream=None):
        cr.cr_distill_loss(x, index, z, loss, temperature=2.0, dlogits=dx, workspace=workspace, stream=stream)

    return call, [loss, dx], cr.cr_distill_loss_workspace_bytes(rows, classes, cr.CR_BF16, top), (x, index, z)


MAKERS = [_embed, _score, _distil]


def _expected(make, seed):
    call, out, _, _ = make(seed)
    call()
    torch.cuda.synchronize()
    return [t.clone() for t in out]


@pytest.mark.parametrize("make", MAKERS)
def test_two_streams_at_once(make):
    """Two calls that overlap, each in a workspace of its own, several times over."""
    want = [_expected(make, seed) for seed in (1, 2)]
    calls, streams = [make(1), make(2)], [torch.cuda.Stream(), torch.cuda.Stream()]
    spaces = [torch.empty(c[2], dtype=torch.uint8, device="cuda") for c in calls]
    for _ in range(5):
        for c in calls:
            for t in c[1]:
                t.fill_(7)
        torch.cuda.synchronize()
        for c, s, w in zip(calls, streams, spaces):
            c[0](workspace=w, stream=s.cuda_stream)
        torch.cuda.synchronize()
        for c, expected in zip(calls, want):
            assert all(torch.equal(a, b) for a, b in zip(c[1], expected))


@pytest.mark.parametrize("make", MAKERS)
def test_workspaces_that_hold_anything(make):
    want = _expected(make, 3)
    call, out, need, _ = make(3)
    assert need > 0
    for fill in (0x00, 0xFF, 0x7F):
        workspace = torch.full((need + 512,), fill, dtype=torch.uint8, device="cuda")
        for t in out:
            t.fill_(7)
        call(workspace=workspace[:need])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)) and bool((workspace[need:] == fill).all())
    with pytest.raises(cr.CodedReduceError):
        call(workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("make", MAKERS)
def test_two_graphs_that_share_a_workspace(make):
    """Replayed one after the other, in either order, with eager calls in the same workspace between them and new inputs."""
    calls = [make(4), make(5)]
    workspace = torch.empty(max(c[2] for c in calls), dtype=torch.uint8, device="cuda")
    graphs = []
    for c in calls:
        c[0](workspace=workspace)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c[0](workspace=workspace)
        graphs.append(graph)
    for seed in (6, 7, 8):
        fresh = [make(seed), make(seed + 10)]
        want = [_expected(make, seed), _expected(make, seed + 10)]
        for c, f in zip(calls, fresh):
            for a, b in zip(c[3], f[3]):
                a.copy_(b)
            for t in c[1]:
                t.fill_(7)
        fresh[0][0](workspace=workspace)
        for i in (0, 1) if seed % 2 else (1, 0):
            graphs[i].replay()
        fresh[1][0](workspace=workspace)
        torch.cuda.synchronize()
        for c, expected in zip(calls, want):
            assert all(torch.equal(a, b) for a, b in zip(c[1], expected))


def test_a_row_of_all_classes():
    """2^28 classes: the row's slices are many, and the alternatives of few of them last."""
    V, top = 1 << 28, 128
    gen = torch.Generator(device="cuda").manual_seed(9)
    x = torch.empty(1, V, dtype=torch.bfloat16, device="cuda").normal_(generator=gen).abs_().neg_()
    places = torch.randperm(V, generator=gen, device="cuda")[:top]
    x[0, places] = (1.0 + torch.arange(top, device="cuda") / 64.0).bfloat16()      # ascending, some of them equal
    tokens = torch.tensor([V - 1], device="cuda")
    logp, entropy, index, values = torch.empty(1, device="cuda"), torch.empty(1, device="cuda"), torch.empty(1, top, dtype=torch.int64, device="cuda"), torch.empty(1, top, device="cuda")
    cr.cr_log_probs(x, tokens, logp, entropy=entropy, top_index=index, top_logp=values)
    order = sorted(places.tolist(), key=lambda j: (-float(x[0, j]), j))
    assert index[0].tolist() == order
    total = sum(float(torch.exp(x[0, lo:lo + (1 << 24)].double()).sum()) for lo in range(0, V, 1 << 24))
    lse = torch.log(torch.tensor(total, dtype=torch.float64))
    # sums of parts: 64 additions a thread, 8 a workgroup, 128 and 8 a row's slices, in 32 bits
    error = 256 * U * (1 + float(lse))
    assert abs(float(logp) - (float(x[0, -1]) - float(lse))) <= error
    assert (values[0].double().cpu() - (x[0, order].double().cpu() - lse)).abs().max() <= error
    z = values.clone()
    loss, dx = torch.empty(1, device="cuda"), torch.empty_like(x)
    cr.cr_distill_loss(x, index, z, loss, dlogits=dx)
    q = torch.softmax(z[0].double().cpu(), dim=0)
    log_p = x[0, order].double().cpu() - lse
    want = float((q * (q.log() - log_p)).sum())
    # chunks of a slice one after another: 256 additions a thread and more of the slices
    assert abs(float(loss) - want) <= 1024 * U * (1 + float((q * (q.log().abs() + log_p.abs())).sum()))
    got = dx[0, order].double().cpu()
    assert ((got - (torch.exp(log_p) - q)).abs() <= 2.0 ** -8 * got.abs() + 1e-6).all()
    assert abs(float(dx[0, 12345].double()) - float(torch.exp(x[0, 12345].double().cpu() - lse))) <= 2.0 ** -7 * float(torch.exp(x[0, 12345].double().cpu() - lse)) or 12345 in order
