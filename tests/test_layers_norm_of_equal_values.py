"""Group norm where a group's values are equal, or it has one alone, far from 0 and with a small eps: the variance is 0, h is 0, and what rounding leaves of
it would be multiplied by 1 / sqrt(eps).

The values have few enough bits that every sum of them is exact in 32 bits and so is the mean, in either type.  So y is beta (rounded to its type), the
gradient of gamma is 0, and mean and rstd are those of the formulas; dx has the rounding of gamma dz and of its mean, times rstd."""
import pytest

import paper_1902_01981_amd as cr
from _layers import HALF_ULP, U, wide

torch = pytest.importorskip("torch")

# points, positions, channels, groups: one position by lanes (whole chunks, odd ones, more than a chunk a lane); a point in a workgroup; several points of one
# position at a time, of small groups; pieces; slices of a group; groups of one value
SHAPES = [(7, 1, 256, 2), (300, 1, 330, 33), (5, 1, 1027, 1), (3, 1, 4000, 1), (6, 49, 96, 32), (3, 17, 100, 10), (40, 9, 200, 25), (5000, 1, 24, 6), (4100, 1, 2004, 334),
          (30_001, 1, 96, 48), (2, 2100, 64, 4), (2, 5001, 12, 4), (1, 3, 20_000, 4), (4, 1, 24, 24), (3, 2, 9000, 1)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_equal_values_far_from_zero(shape, dtype):
    N, P, C, G = shape
    eps = 1e-6
    gen = torch.Generator().manual_seed(C)
    value = torch.tensor([300.0, -1000.0, 3.0, 0.0])[torch.randint(0, 4, (N, G), generator=gen)]
    x = value.repeat_interleave(C // G, dim=1)[:, None, :].expand(N, P, C).contiguous().to(dtype).cuda()
    assert torch.equal(x[:, 0, ::C // G].float().cpu(), value)
    dy = torch.randn(N, P, C, generator=gen).to(dtype).cuda()
    gamma, beta = (1 + 0.3 * torch.randn(C, generator=gen)).cuda(), torch.randn(C, generator=gen).cuda()
    y, dx = torch.full_like(x, float("nan")), torch.full_like(x, float("nan"))
    mean, rstd = torch.full((2, N, G), float("nan"), device="cuda")
    dgamma, dbeta = torch.full((2, 1, C), float("nan"), device="cuda")
    cr.cr_group_norm_forward(x, gamma, beta, G, y, mean, rstd, eps=eps)
    cr.cr_group_norm_backward(dy, x, mean, rstd, gamma, beta, G, dx, dgamma, dbeta)
    assert torch.equal(mean.cpu(), value)
    assert ((wide(rstd) * eps ** 0.5 - 1).abs() <= 4 * U).all()
    assert torch.equal(y, beta.to(dtype).expand_as(y))
    assert (dgamma == 0).all()
    size = wide(dy).abs().sum(dim=(0, 1))
    assert ((wide(dbeta)[0] - wide(dy).sum(dim=(0, 1))).abs() - 64 * U * size).max() <= 0
    t = wide(gamma) * wide(dy)
    mean_t = t.reshape(N, P, G, C // G).mean(dim=(1, 3)).repeat_interleave(C // G, dim=1)[:, None, :]
    want = (t - mean_t) * eps ** -0.5
    assert ((wide(dx) - want).abs() - 64 * U * eps ** -0.5 * t.abs().max() - HALF_ULP[dtype] * want.abs()).max() <= 0
