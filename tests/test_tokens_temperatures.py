"""The distillation loss at the lower end of its temperatures against a closed form.

Where the largest logit of a row, and of a teacher's entries, is ahead of the others by 1 or more and T <= 1/1000, the others' shares are exp(-1000) or less, which is
0 in 32 bits, and the first ones' are 1: with m the student's largest class and j the teacher's, loss = w T (x_m - x_j), the gradient w T at m and -w T at j, 0 where
they are the same, and 0 elsewhere.  What may differ, in half steps of 32 bits: the distance, w T and their product once each, and the powers of two are exact."""
import pytest

from _layers import HALF_ULP, U, wide
from test_tokens_distill import _run

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16]


# a row's kernel: sixteen lanes, a wavefront, a workgroup, slices (bf16 and fp32 from 138 248 and 69 124 classes on)
@pytest.mark.parametrize("dtype", TYPES, ids=["f32", "bf16"])
@pytest.mark.parametrize("T", [2.0 ** -40, 2.0 ** -39 * 1.1, 1e-6, 1e-3])
@pytest.mark.parametrize("classes", [5, 40, 700, 9000, 140_003])
def test_shares_of_one(classes, T, dtype):
    rows, top = 12, 5
    gen = torch.Generator().manual_seed(classes)
    x = torch.randn(rows, classes, generator=gen) * 3
    index = torch.stack([torch.randperm(classes, generator=gen)[:top] for _ in range(rows)])
    z = torch.randn(rows, top, generator=gen) * 3
    first, given = torch.randint(0, classes, (rows,), generator=gen), torch.randint(0, top, (rows,), generator=gen)
    first[:4] = index[torch.arange(4), given[:4]]        # the teacher and the student agree
    first[4], first[5] = 0, classes - 1
    x[torch.arange(rows), first] = x.amax(dim=1) + 2.0   # bf16 values here have steps of 1/8 at most
    z[torch.arange(rows), given] = z.amax(dim=1) + 1.5
    index[7, (int(given[7]) + 1) % top] = index[7, int(given[7])]          # the teacher's class once more, with a share of 0
    x, weights = x.to(dtype), 0.5 + torch.rand(rows, generator=gen)
    ahead = torch.topk(wide(x), 2, dim=1).values
    assert bool((ahead[:, 0] - ahead[:, 1] >= 1).all())
    loss, dlogits = _run(x.cuda(), index.cuda(), z.cuda(), T, weights.cuda())
    by = wide(weights) * float(torch.tensor(T, dtype=torch.float32))
    row, j = torch.arange(rows), index[torch.arange(rows), given]
    want_loss = by * (wide(x)[row, first] - wide(x)[row, j])
    want = torch.zeros(rows, classes, dtype=torch.float64)
    want[row, first] += by
    want[row, j] -= by
    assert bool((want_loss[:4] == 0).all()) and bool((want_loss[j != first] > 0).all()) and int((j != first).sum()) >= 1
    assert bool(((wide(loss) - want_loss).abs() <= 3 * U * 1.0001 * want_loss).all())
    assert bool(((wide(dlogits) - want).abs() <= (U + HALF_ULP[dtype] * (1 + U)) * 1.0001 * want.abs()).all())
    only, _ = _run(x.cuda(), index.cuda(), z.cuda(), T, weights.cuda(), gradient=False)
    assert torch.equal(only, loss)
