"""The layers in a network under coded aggregation: its gradient against torch's automatic one, every holder's against every other's, the decoded one
against the uncoded one."""
import numpy as np
import pytest

from _layers import kept as kept_mask

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _network(rate=0.25):
    from examples import coded_network as net

    x, targets = net.data(60, 9, 13, 5, 3)
    return net, net.Network(13, 40, 5, 2, 8, rate, 11), x, targets


def test_the_gradient_is_torchs():
    """The same network in 64 bits out of torch's operations, differentiated by torch; the mask from its definition."""
    module, net, x, targets = _network()
    _, kept = net.forward(x, targets, step=4, first_point=1000)
    bounds = np.array([0, 7, 7, 31, 60])
    got = net.gradients(kept, bounds)
    w = net.w.double().cpu().requires_grad_()
    p, N, P = net.parameters(w), 60, 9
    u = x.double().cpu() @ p["embed"]
    for b in range(2):
        v = u.reshape(N, P, 8, 5)
        mean = v.mean(dim=(1, 3), keepdim=True)
        h = ((v - mean) * ((v - mean).square().mean(dim=(1, 3), keepdim=True) + 1e-5).rsqrt()).reshape(N, P, 40)
        z = torch.nn.functional.silu(h * p[f"gamma{b}"] + p[f"beta{b}"]) @ p[f"dense{b}"] + p[f"bias{b}"]
        mask, scale = kept_mask(range(1000, 1060), P, 40, 0.25, 11, 4 * 2 + b)
        u = u + z * mask * scale
    loss = torch.nn.functional.cross_entropy(u.mean(dim=1) @ p["out"], targets.cpu(), reduction="none")
    for r in range(4):
        if bounds[r] == bounds[r + 1]:
            assert bool((got[r] == 0).all())
            continue
        want, = torch.autograd.grad(loss[bounds[r]:bounds[r + 1]].sum(), w, retain_graph=True)
        for name, a in net.parameters(got[r].double().cpu()).items():
            b = net.parameters(want)[name]
            assert float((a - b).norm()) <= 1e-5 * float(b.norm()), name


def test_every_holder_forms_the_same():
    """A worker with some of the points, in a call of its own: the same losses and gradients up to rounding (torch's products go by the size)."""
    module, net, x, targets = _network()
    loss, kept = net.forward(x, targets, step=2, first_point=500)
    runs = net.gradients(kept, np.array([0, 20, 45, 60]))
    own, own_kept = net.forward(x[20:45], targets[20:45], step=2, first_point=520)
    for b in range(2):
        for name in ("mean", "rstd"):
            assert (own_kept[name][b] - kept[name][b][20:45]).abs().max() <= 1e-5 * kept[name][b].abs().max()
    assert (own - loss[20:45]).abs().max() <= 1e-5
    g = net.gradients(own_kept, np.array([0, 25]))
    assert float((g[0] - runs[1]).norm()) <= 1e-5 * float(runs[1].norm())


@pytest.mark.parametrize("tree", [(2, 3, 1), (1, 4, 2)])
def test_training(tree):
    """Decoded gradients are the uncoded ones under every mask; the loss falls."""
    from examples import coded_network as net

    losses, worst = net.train(points=300, steps=12, tree=tree, say=None)
    assert worst <= 1e-5 and losses[-1] < 0.8 * losses[0]
