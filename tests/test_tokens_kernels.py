"""Every kernel that the sizes of log probabilities and of the distillation loss pick, on both sides of each border, in both types: sizes by the rules of the
planners, bounds and definitions those of test_tokens_log_probs.py and test_tokens_distill.py."""
import pytest

import paper_1902_01981_amd as cr
from test_tokens_distill import _check as check_distill
from test_tokens_distill import _inputs as distill_inputs
from test_tokens_distill import _run as run_distill
from test_tokens_log_probs import _check as check_log_probs
from test_tokens_log_probs import _check_gradient, _gradient, _logits, _tokens
from test_tokens_log_probs import _run as run_log_probs

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
TYPES = {"f32": (torch.float32, 4), "bf16": (torch.bfloat16, 8)}         # type, classes of a load


def _sizes(borders):
    """(type, classes): the last size of every kernel and the first of the next one."""
    return [(name, load * chunks + more) for name, (_, load) in TYPES.items() for chunks in borders for more in (0, 1)]


# chunks of a row: sixteen lanes with one chunk or two, a wavefront with one, two, four and eight a lane, a workgroup with one slice of the row and with several
@pytest.mark.parametrize("name,classes", _sizes([16, 32, 64, 128, 256, 512, 2048, 4096]))
def test_log_probs(name, classes):
    dtype, _ = TYPES[name]
    x, tokens = _logits(9, classes, dtype, classes), _tokens(9, classes, 2)
    x[3, classes // 2:] = -INF
    x[4, :] = -INF
    x[5, classes - 1] = NAN
    x[6] = torch.where(x[6] > 0, 1.0, -1.0)              # two values: the lists overflow
    x[7] = (x[7].double() / 64 + 1000).to(dtype)         # a large offset beside the spread: few numbers of 16 bits
    tokens[8] = classes - 1
    for top in (0, 1, 20, 128):
        out = run_log_probs(x, tokens, top)
        check_log_probs(x, tokens, top, out)
    gen = torch.Generator().manual_seed(3)
    dlogp, dentropy = torch.randn(9, generator=gen).cuda(), torch.randn(9, generator=gen).cuda()
    _check_gradient(x, tokens, dlogp, dentropy, _gradient(x, tokens, out, dlogp, dentropy))


# the gradient: rows beside each other in a workgroup, a workgroup and more per row
@pytest.mark.parametrize("name,classes", [(name, load * whole + more) for name, (_, load) in TYPES.items() for whole in (255, 256, 1024, 1025) for more in (0, load - 1)])
def test_log_probs_gradient(name, classes):
    dtype, _ = TYPES[name]
    x, tokens = _logits(70, classes, dtype, classes), _tokens(70, classes, 4)
    tokens[69] = classes - 1
    gen = torch.Generator().manual_seed(5)
    dlogp, dentropy = torch.randn(70, generator=gen).cuda(), torch.randn(70, generator=gen).cuda()
    out = run_log_probs(x, tokens, 0)
    dx = _gradient(x, tokens, out, dlogp, dentropy)
    _check_gradient(x, tokens, dlogp, dentropy, dx)
    over = x.clone()
    assert torch.equal(_gradient(over, tokens, out, dlogp, dentropy, over), dx)


# chunks of a row: sixteen lanes; a wavefront with one to eight chunks a lane; a workgroup with eight and eighteen a lane of 960, and behind them slices of one, two and
# more steps
@pytest.mark.parametrize("name,classes", _sizes([16] + [64 * k for k in range(1, 9)]) + [(name, load * whole + more) for name, (_, load) in TYPES.items()
                                                                                      for whole, more in ((960 * 8, 1), (960 * 8 + 1, 0), (960 * 18, load - 1), (960 * 18 + 1, 0))])
@pytest.mark.parametrize("top", [5, 128])
def test_distill(top, name, classes):
    dtype, _ = TYPES[name]
    x, index, z, weights = distill_inputs(8, classes, top, dtype, classes + top)
    index[0, 1], index[0, 2], index[0, 3] = classes - 1, 0, classes - 1
    index[3] = index[3].clamp(min=0) % (classes // 2)
    x[3, classes // 2:] = -INF
    x[4, :] = -INF
    x[5, classes - 1] = NAN
    index[5, 0] = 0
    index[6] = index[6].clamp(min=0) % 3                 # few classes, many times each
    index[7, 0] = classes                                # no class
    loss, dlogits = run_distill(x, index, z, 1.5, weights)
    check_distill(x, index, z, 1.5, weights, loss, dlogits)
    assert bool(loss[[5, 7]].isnan().all()) and bool(dlogits[[5, 7]].isnan().all())
    only_loss, _ = run_distill(x, index, z, 1.5, weights, gradient=False)
    assert torch.equal(only_loss.nan_to_num(nan=7.0), loss.nan_to_num(nan=7.0))
    over = x.clone()
    in_place = run_distill(over, index, z, 1.5, weights, dlogits=over)
    assert torch.equal(in_place[0].nan_to_num(nan=7.0), loss.nan_to_num(nan=7.0)) and torch.equal(over.nan_to_num(nan=7.0), dlogits.nan_to_num(nan=7.0))


def test_workspaces_say_which_rows_are_cut():
    """The borders above, as far as the workspaces show them: rows that one team holds need none."""
    for dtype, load in ((cr.CR_F32, 4), (cr.CR_BF16, 8)):
        assert cr.cr_log_probs_workspace_bytes(9, 2048 * load, dtype, 20) == 0 < cr.cr_log_probs_workspace_bytes(9, 2048 * load + 1, dtype, 20)
        assert cr.cr_distill_loss_workspace_bytes(9, 960 * 18 * load + load - 1, dtype, 20) == 0 < cr.cr_distill_loss_workspace_bytes(9, (960 * 18 + 1) * load, dtype, 20)
