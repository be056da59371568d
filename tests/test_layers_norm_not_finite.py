"""A NaN or an infinity in a group: mean and rstd of that group are NaN, as y and dx are there, wherever in the group it is; nothing else changes by a bit."""
import pytest

import paper_1902_01981_amd as cr

torch = pytest.importorskip("torch")

# one position by lanes; a point in a workgroup; several points of one position at a time; pieces; slices of a group
SHAPES = [(9, 1, 36, 4), (3, 1, 1027, 1), (3, 12, 40, 5), (5, 49, 96, 32), (30_001, 1, 96, 48), (2, 2100, 64, 4), (2, 5001, 12, 4), (2, 3, 20_000, 4)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_statistics_of_a_group(shape, dtype):
    N, P, C, G = shape
    gen = torch.Generator().manual_seed(P)
    x, dy = (torch.randn(N, P, C, generator=gen).to(dtype).cuda() for _ in range(2))

    def run(x):
        y, dx = torch.full_like(x, 5.0), torch.full_like(x, 5.0)
        mean, rstd = torch.full((2, N, G), 5.0, device="cuda")
        cr.cr_group_norm_forward(x, None, None, G, y, mean, rstd, activation=cr.CR_ACT_SILU)
        cr.cr_group_norm_backward(dy, x, mean, rstd, None, None, G, dx, activation=cr.CR_ACT_SILU)
        return y, mean, rstd, dx

    clean = run(x)
    n, g, width = N - 1, G - 1, C // G
    hit = torch.zeros(N, P, C, dtype=torch.bool, device="cuda")
    hit[n, :, g * width:] = True
    for bad in (float("nan"), float("inf"), -float("inf")):
        for p, c in ((0, 0), (P - 1, width - 1), (P // 2, width // 2)):
            broken = x.clone()
            broken[n, p, g * width + c] = bad
            got = run(broken)
            for a, b, where in ((got[0], clean[0], hit), (got[1], clean[1], hit[:, 0, ::width]), (got[2], clean[2], hit[:, 0, ::width]), (got[3], clean[3], hit)):
                assert bool(a[where].isnan().all()) and torch.equal(a[~where], b[~where])
