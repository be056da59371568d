"""The layers over tokens together, in a network under coded aggregation: its gradient against torch's automatic one, every holder's against every other's, the
decoded one against the uncoded one."""
import numpy as np
import pytest

from _layers import kept as kept_mask

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
SIZES = dict(vocabulary=70, channels=40, blocks=2, groups=8, rate=0.25)


def _network(points=50, positions=9, top=6):
    from examples import coded_tokens as module

    tokens = module.data(points, positions, 70, 3)
    tokens[7] = -1                                       # a point of no tokens
    teacher, net = module.Network(seed=12, **SIZES), module.Network(seed=11, **SIZES)
    return net, tokens, teacher.answers(tokens, top)


def _in_64_bits(net, w, tokens, answers, T, masks):
    """The loss of every position out of torch's operations."""
    p, (N, P) = net.parameters(w), tokens.shape
    there = (tokens >= 0).double()[..., None]
    u = p["table"][tokens.clamp(min=0)] * net.scale * there
    for b in range(net.blocks):
        v = u.reshape(N, P, 8, 5)
        mean = v.mean(dim=(1, 3), keepdim=True)
        h = ((v - mean) * ((v - mean).square().mean(dim=(1, 3), keepdim=True) + 1e-5).rsqrt()).reshape(N, P, 40)
        z = torch.nn.functional.silu(h * p[f"gamma{b}"] + p[f"beta{b}"]) @ p[f"dense{b}"] + p[f"bias{b}"]
        u = u + (z if masks is None else z * masks[b])
    logits = u.reshape(N * P, 40) @ p["out"]
    if answers is None:
        return logits
    index, values = answers
    q = torch.softmax(values.double() / T, dim=1)
    log_p = torch.log_softmax(logits / T, dim=1).gather(1, index.clamp(min=0))
    return (T * T * (q * (q.log() - log_p)).sum(dim=1) * (index[:, 0] >= 0)).view(N, P)


def test_the_teachers_answers():
    net, tokens, answers = _network()
    from examples import coded_tokens as module

    teacher = module.Network(seed=12, **SIZES)
    logits = _in_64_bits(teacher, teacher.w.double().cpu(), tokens.cpu(), None, 1.0, None)
    here = tokens.reshape(-1).cpu() >= 0
    index, values = (t.cpu() for t in answers)
    assert bool((index[~here] == -1).all())
    want = torch.log_softmax(logits, dim=1)
    assert (want.gather(1, index.clamp(min=0)) - values)[here].abs().max() <= 1e-4
    assert (torch.topk(want, 6, dim=1).values - values)[here].abs().max() <= 1e-4            # as large as any others


def test_the_gradient_is_torchs():
    net, tokens, answers = _network()
    loss, kept = net.forward(tokens, answers, 2.0, step=4, first_point=1000)
    bounds = np.array([0, 7, 8, 8, 31, 50])              # the second run is the point of no tokens, the third has none
    got = net.gradients(kept, bounds)
    w = net.w.double().cpu().requires_grad_()
    masks = []
    for b in range(2):
        mask, scale = kept_mask(range(1000, 1050), 9, 40, 0.25, 11, 4 * 2 + b)
        masks.append(mask * scale)
    want_loss = _in_64_bits(net, w, tokens.cpu(), [t.cpu() for t in answers], 2.0, masks)
    assert (loss.cpu() - want_loss.detach()).abs().max() <= 1e-4
    for r in range(5):
        if r in (1, 2):
            assert bool((got[r] == 0).all())
            continue
        want, = torch.autograd.grad(want_loss[bounds[r]:bounds[r + 1]].sum(), w, retain_graph=True)
        for name, a in net.parameters(got[r].double().cpu()).items():
            b = net.parameters(want)[name]
            assert float((a - b).norm()) <= 2e-5 * float(b.norm()), name


def test_every_holder_forms_the_same():
    """A worker with some of the points, in a call of its own: the same losses and gradients up to rounding (torch's products go by the size)."""
    net, tokens, answers = _network()
    loss, kept = net.forward(tokens, answers, 2.0, step=2, first_point=500)
    runs = net.gradients(kept, np.array([0, 20, 45, 50]))
    rows = slice(20 * 9, 45 * 9)
    own, own_kept = net.forward(tokens[20:45], [t[rows] for t in answers], 2.0, step=2, first_point=520)
    assert (own - loss[20:45]).abs().max() <= 1e-4
    g = net.gradients(own_kept, np.array([0, 25]))
    assert float((g[0] - runs[1]).norm()) <= 2e-5 * float(runs[1].norm())


@pytest.mark.parametrize("tree", [(2, 3, 1), (1, 4, 2)])
def test_the_decoded_gradient(tree):
    """Decoded gradients are the uncoded ones under every mask, and the example runs."""
    from examples import coded_tokens as module

    losses, worst = module.train(points=120, steps=6, tree=tree, say=None)
    assert worst <= 1e-5 and all(np.isfinite(losses))
