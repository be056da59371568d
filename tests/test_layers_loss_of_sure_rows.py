"""The softmax loss of rows that are already classified well, and of logits that are large beside it: the loss is small beside both, and has to come out as
exact as its own terms allow, whatever the logits' size.

With c the largest logit, S = sum_j exp(x_j - c), the loss is (c - x_t) + log S.  What may differ, in units of u = 2^-24, c being subtracted from every
logit first: an exponential's relative error is 3 u |x_j - c| (the subtraction, the product with log2(e), that constant) and 2 u of itself, a sum about a
smaller reference that is brought to c adds as much for the distance between the two and 3 u beside; a logit passes at most 24 such steps and 40 additions on
its way into S.  So S is off by at most u (120 + 4 E), E the mean of c - x_j under the shares, and the loss by that, 4 u of each of its two terms, and
10 u for a logarithm near 1.  Nothing in this grows with c."""
import pytest

import paper_1902_01981_amd as cr
from _layers import U, wide

torch = pytest.importorskip("torch")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,classes", [(300, 2), (320, 10), (40, 77), (30, 301), (20, 3001), (9, 9001), (5, 70_003), (3, 140_001)])
def test_loss_beside_large_logits(rows, classes, dtype):
    gen = torch.Generator().manual_seed(classes)
    targets = torch.randint(0, classes, (rows,), generator=gen)
    weights = 0.5 + torch.rand(rows, generator=gen)
    for shift in (0.0, 30.0, -300.0, 3000.0, 3e4):
        x = 1.5 * torch.randn(rows, classes, generator=gen)
        lead = torch.linspace(0.0, 14.0, rows)           # over the rest of the row
        x[torch.arange(rows), targets] = x.amax(dim=1) + lead
        x = (x + shift).to(dtype).cuda()
        z, at = wide(x), targets[:, None]
        c = z.amax(dim=1, keepdim=True)
        e = torch.exp(z - c)
        S = e.sum(dim=1, keepdim=True)
        apart = c - z.gather(1, at)
        want = (wide(weights)[:, None] * (apart + torch.log1p(S - 1)))[:, 0]
        mean = (e * (c - z)).sum(dim=1, keepdim=True) / S
        allowed = (wide(weights)[:, None] * U * (130 + 4 * mean + 4 * apart + 4 * torch.log(S)))[:, 0]
        for gradient in (False, True):
            loss, lse = torch.full((rows,), float("nan"), device="cuda"), torch.full((rows,), float("nan"), device="cuda")
            cr.cr_softmax_loss(x, targets.cuda(), loss, lse=lse, dlogits=torch.empty_like(x) if gradient else None, weights=weights.cuda())
            assert ((wide(loss) - want).abs() - allowed).max() <= 0
            assert (loss >= 0).all()
            # the sum itself is rounded once, at its size
            assert ((wide(lse) - (c + torch.log(S))[:, 0]).abs() - (allowed / wide(weights)) - U * (c.abs()[:, 0] + 1)).max() <= 0
