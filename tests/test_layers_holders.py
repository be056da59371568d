"""What two holders of the same data points form in calls of their own, with other numbers of points: rows of the loss and values of the dropout are the
same bits; of the group norm, whose tiles go by the number of points, they are the same up to rounding.

Each of the two is within the bounds of test_layers_norm.py of the formulas, so they are within twice that of each other."""
import pytest

import paper_1902_01981_amd as cr
from _layers import HALF_ULP, U

torch = pytest.importorskip("torch")
ROUNDS = 64.0

# points of the one holder and of the other, positions, channels, groups: other chunks of a thread and points side by side; several points a thread or one; other pieces
PAIRS = [(320, 4000, 4, 320, 32), (40, 5000, 1, 24, 6), (12, 30_001, 1, 96, 48), (20, 64, 4096, 512, 32), (3, 700, 49, 96, 32), (1, 300, 1, 1027, 1)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("pair", PAIRS, ids=lambda p: "x".join(map(str, p)))
def test_group_norm(pair, dtype):
    few, many, P, C, G = pair
    gen = torch.Generator(device="cuda").manual_seed(few)
    x, dy = (torch.randn(many, P, C, generator=gen, device="cuda").to(dtype) for _ in range(2))
    gamma, beta = 1 + 0.3 * torch.randn(C, generator=gen, device="cuda"), 0.3 * torch.randn(C, generator=gen, device="cuda")

    def run(x, dy):
        N = x.shape[0]
        y, dx = torch.empty_like(x), torch.empty_like(x)
        mean, rstd = torch.empty(2, N, G, device="cuda")
        cr.cr_group_norm_forward(x, gamma, beta, G, y, mean, rstd, activation=cr.CR_ACT_SILU)
        cr.cr_group_norm_backward(dy, x, mean, rstd, gamma, beta, G, dx, activation=cr.CR_ACT_SILU)
        return y, mean, rstd, dx

    own, all_ = run(x[:few], dy[:few]), [t[:few] for t in run(x, dy)]
    most = x[:few].abs().amax(dim=1).view(few, G, -1).amax(dim=2).double()               # of a group
    assert ((own[1].double() - all_[1]).abs() - 2 * ROUNDS * U * most).max() <= 0
    spread = most * own[2]
    assert ((own[2].double() - all_[2]).abs() / own[2] - 2 * ROUNDS * U * (1 + spread ** 2 / 16)).max() <= 0
    wide = spread.repeat_interleave(C // G, dim=1)[:, None, :]
    z_error = ROUNDS * U * (gamma.abs() * wide * (1 + wide / 16) + beta.abs() + 1)
    assert ((own[0].double() - all_[0]).abs() - 2 * (1.1 * z_error + HALF_ULP[dtype] * own[0].abs())).max() <= 0
    most_d = (gamma * dy[:few]).abs().max().double()
    allowed = ROUNDS * U * own[2].max() * most_d * (1 + 2 * spread.max()) * (2 + gamma.abs().max())
    assert ((own[3].double() - all_[3]).abs() - 2 * (allowed + HALF_ULP[dtype] * own[3].abs())).max() <= 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("few,many,classes", [(1, 3000, 10), (7, 2000, 1100), (2, 900, 9002), (3, 40, 150_001)])
def test_loss(few, many, classes, dtype):
    gen = torch.Generator(device="cuda").manual_seed(classes)
    x = (3 * torch.randn(many, classes, generator=gen, device="cuda")).to(dtype)
    targets = torch.randint(0, classes, (many,), generator=gen, device="cuda")

    def run(n):
        loss, lse, dx = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty_like(x[:n])
        cr.cr_softmax_loss(x[:n], targets[:n], loss, lse=lse, dlogits=dx)
        return loss, lse, dx

    assert all(torch.equal(a, b[:few]) for a, b in zip(run(few), run(many)))


@pytest.mark.gpu
@pytest.mark.parametrize("few,many,P,C", [(1, 5000, 3, 37), (5, 600, 40, 264), (2, 70, 1, 20_000)])
def test_dropout(few, many, P, C):
    gen = torch.Generator(device="cuda").manual_seed(C)
    x, bias = torch.randn(many, P, C, generator=gen, device="cuda"), torch.randn(C, generator=gen, device="cuda")

    def run(n):
        y, dx = torch.empty_like(x[:n]), torch.empty_like(x[:n])
        cr.cr_dropout_forward(x[:n], y, 0.3, 5, 2, bias=bias, residual=x[:n], first_point=77)
        cr.cr_dropout_backward(x[:n], dx, 0.3, 5, 2, first_point=77)
        return y, dx

    assert all(torch.equal(a, b[:few]) for a, b in zip(run(few), run(many)))
