"""More rows than a launch has: batches of launches, and workgroups that go on to further rows.  A row's bits are the same among any others, so that rows on both sides of
every such border are compared with calls on those rows alone, which other tests compare with the definition."""
import pytest

import paper_1902_01981_amd as cr

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
FILL = 2.0 ** 100                                        # what no output is, in either type


def _logits(rows, classes, dtype, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(rows, classes, dtype=dtype, device="cuda").normal_(generator=gen), gen


def _same(got, want):
    assert len(got) == len(want) > 0
    for a, b in zip(got, want):
        assert torch.equal(a, b)


# rows of one team each, 2^22 a batch, as sixteen lanes and as wavefronts; rows of eight slices and 128 alternatives, 8 065 a batch
@pytest.mark.parametrize("rows,classes,top,border", [((1 << 22) + 9, 5, 3, 1 << 22), ((1 << 22) + 9, 150, 2, 1 << 22), ((1 << 22) + 9, 270, 0, 1 << 22), (8_070, 131_071, 128, 8_065)])
def test_log_probs(rows, classes, top, border):
    x, gen = _logits(rows, classes, torch.bfloat16, 1)
    tokens = torch.randint(-1, classes, (rows,), generator=gen, device="cuda")

    def run(lo, hi):
        n = hi - lo
        out = {k: torch.full((n,), FILL, device="cuda") for k in ("logp", "entropy", "largest", "log_sum")}
        if top:
            out.update(top_index=torch.full((n, top), -9, device="cuda"), top_logp=torch.full((n, top), FILL, device="cuda"))
        cr.cr_log_probs(x[lo:hi], tokens[lo:hi], **out)
        return list(out.values())

    whole = run(0, rows)
    for lo, hi in ((0, 20), (border - 11, border), (border - 3, border + 4), (rows - 7, rows)):
        _same([t[lo:hi] for t in whole], run(lo, hi))
    assert not any(bool((t == (-9 if t.dtype == torch.int64 else FILL)).any()) for t in whole)


# units of a launch: 2^20 workgroups of 256 chunks beside each other, of whole chunks of one row
@pytest.mark.parametrize("rows,classes,border", [(11_000_000, 99, (1 << 28) // 27), ((1 << 20) + 50, 1_027, 1 << 20)])
def test_the_gradient_of_log_probs(rows, classes, border):
    x, gen = _logits(rows, classes, torch.float32, 2)
    tokens = torch.randint(-1, classes, (rows,), generator=gen, device="cuda")
    a, b = (torch.empty(rows, device="cuda").normal_(generator=gen) for _ in range(2))
    largest, log_sum, entropy = (torch.empty(rows, device="cuda") for _ in range(3))
    cr.cr_log_probs(x, None, None, entropy=entropy, largest=largest, log_sum=log_sum)

    def run(lo, hi, dx):
        cr.cr_log_probs_backward(x[lo:hi], tokens[lo:hi], largest[lo:hi], log_sum[lo:hi], entropy[lo:hi], a[lo:hi], b[lo:hi], dx)
        return dx

    whole = run(0, rows, torch.full_like(x, FILL))
    for lo, hi in ((0, 20), (border - 11, border), (border - 3, border + 4), (rows - 7, rows)):
        _same([whole[lo:hi]], [run(lo, hi, torch.full_like(x[lo:hi], FILL))])
    assert not bool((whole == FILL).any())


# sixteen lanes: 2^26 rows a launch; wavefronts: 2^22 rows at once; workgroups that stay, a row after another
@pytest.mark.parametrize("rows,classes,border", [((1 << 26) + 9, 2, 1 << 26), ((1 << 22) + 9, 130, 1 << 22), (60_000, 4_200, 2_560)])
def test_distill(rows, classes, border):
    top = 2
    x, gen = _logits(rows, classes, torch.bfloat16, 3)
    index = torch.randint(-1, classes, (rows, top), generator=gen, device="cuda")
    z, weights = torch.empty(rows, top, device="cuda").normal_(generator=gen), torch.rand(rows, generator=gen, device="cuda")

    def run(lo, hi, gradient=True):
        loss, dx = torch.full((hi - lo,), FILL, device="cuda"), torch.full_like(x[lo:hi], FILL) if gradient else None
        cr.cr_distill_loss(x[lo:hi], index[lo:hi], z[lo:hi], loss, temperature=2.0, dlogits=dx, weights=weights[lo:hi])
        return [loss, dx] if gradient else [loss]

    whole = run(0, rows)
    for lo, hi in ((0, 20), (border - 11, border), (border - 3, border + 4), (rows - 7, rows)):
        _same([t[lo:hi] for t in whole], run(lo, hi))
    assert not any(bool((t == FILL).any()) for t in whole)
    _same(run(0, rows, gradient=False), whole[:1])
