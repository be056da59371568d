"""Slabs of wide rows against 64 bits, with a bound that goes by the rows' terms: a residual <x, w> - y may be as near to 0 as its terms cancel, and a bound relative to
the slab then asks for more than 32 bits hold.

What may differ.  A workgroup of 256 threads or more forms a dot product: a thread adds up d / 256 + 8 terms at most, six additions join a wavefront and eight its
wavefronts, so that it is off by (d / 256 + 22) half steps of sum |x w|, and the residual by another one of itself; the logistic function's slope is at most 1/4, and its own
error (an exponential off by |z| + 2 half steps, a sum, a reciprocal off by two) at most 8 + |z|.  A slab's sum has 64 rows in 32 bits at most, and four
roundings follow."""
import pytest

import paper_1902_01981_amd as cr
from _layers import U

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
# those of test_rows_once.py's two passes
WIDE = [(24_577, 0, 13), (24_580, 1, 14), (30_003, 0, 897), (32_768, 1, 451), (24_583, 1, 1_801), (24_578, 0, 3_601)]


@pytest.mark.parametrize("logistic", [0, 1])
@pytest.mark.parametrize("near", [False, True], ids=["", "residuals near 0"])
@pytest.mark.parametrize("d,bf16,m", WIDE)
def test_slabs(d, bf16, m, near, logistic):
    gen = torch.Generator(device="cuda").manual_seed(d + m)
    X = torch.empty(m, d, device="cuda").normal_(generator=gen)
    X = X.bfloat16() if bf16 else X
    w = torch.empty(d, device="cuda").normal_(generator=gen) / d ** 0.5
    step = 512                                           # rows at a time in 64 bits
    z, size = torch.empty(m, dtype=torch.float64, device="cuda"), torch.empty(m, dtype=torch.float64, device="cuda")
    for lo in range(0, m, step):
        terms = X[lo:lo + step].double() * w.double()
        z[lo:lo + step], size[lo:lo + step] = terms.sum(dim=1), terms.abs().sum(dim=1)
    value = torch.sigmoid(z) if logistic else z
    y = value.float() if near else (torch.rand(m, generator=gen, device="cuda") < 0.5).float()
    residual = value - y.double()
    error = (d / 256 + 22) * U * size
    if logistic:
        error = error / 4 + (8 + z.abs()) * U * value
    error = error + U * residual.abs()
    for split in ((cr.CR_SPLIT_ROW_CELLS, 64), None, (cr.CR_SPLIT_ROWS_ONCE, 1), (cr.CR_SPLIT_ROWS_ONCE, 70)):
        if split and split[1] == 1 and m > 1_000:
            continue
        plan = cr.cr_plan_ex(2, 3, 1, m, d, model=logistic, x_dtype=bf16)
        if split:
            cr.cr_plan_set_split(plan, *split)
        begin, end, _, _ = cr.cr_plan_get_segments(plan)
        ws = cr.Workspace(plan)
        ws.slab_grads().fill_(float("nan"))
        cr.cr_partial_grads(plan, X, y, w)
        cr.cr_synchronize(plan)
        got = ws.slab_grads()
        for q, (b, e) in enumerate(zip(begin, end)):
            want, allowed = torch.zeros(d, dtype=torch.float64, device="cuda"), torch.zeros(d, dtype=torch.float64, device="cuda")
            for lo in range(int(b), int(e), step):
                hi = min(lo + step, int(e))
                x = X[lo:hi].double()
                want += (x * residual[lo:hi, None]).sum(dim=0)
                allowed += (x.abs() * (error[lo:hi] + 68 * U * residual[lo:hi].abs())[:, None]).sum(dim=0)
            assert bool(((got[q].double() - want).abs() <= allowed * 1.001).all()), (split, q)
        cr.cr_plan_destroy(plan)
