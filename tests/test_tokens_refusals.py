"""What the layers over tokens refuse, at the C boundary (no launch follows, so no GPU is needed) and in the binding."""
import ctypes

import pytest

import paper_1902_01981_amd as cr
from paper_1902_01981_amd import layers

torch = pytest.importorskip("torch")
HERE = 0x10000                                           # an address nobody reads
F32, BF16 = cr.CR_F32, cr.CR_BF16
NAN, INF = float("nan"), float("inf")


def _shape(points=4, positions=6, channels=20, dtype=F32):
    return layers.cr_layer_shape_t(points, positions, channels, dtype)


def _view(dev=HERE, point=120, position=20):
    return layers.cr_layer_view_t(dev, point, position)


TOKENS = (HERE, 6, 1)


def _refused(status, text):
    assert status == cr.CR_E_INVAL and text in cr.cr_layers_last_error(), (status, cr.cr_layers_last_error())


def _lookup(shape=None, tokens=TOKENS, table=HERE, dtype=F32, vocabulary=30, scale=1.0, y=None):
    return cr.load_layers_library().cr_embedding_forward(_shape() if shape is None else shape, _view(*tokens), table, dtype, vocabulary, scale, _view() if y is None else y, 0)


def _gradient(shape=None, dy=None, tokens=TOKENS, vocabulary=30, scale=1.0, bounds=None, runs=1, dtable=HERE, ws=HERE, nbytes=1 << 40):
    b = None if bounds is None else (ctypes.c_int64 * len(bounds))(*bounds)
    return cr.load_layers_library().cr_embedding_backward(_shape() if shape is None else shape, _view() if dy is None else dy, _view(*tokens), vocabulary, scale, b, runs, dtable, ws,
                                                          nbytes, 0)


def _embedding_bytes(shape, vocabulary=30, bounds=None, runs=1):
    n = ctypes.c_size_t()
    b = None if bounds is None else (ctypes.c_int64 * len(bounds))(*bounds)
    status = cr.load_layers_library().cr_embedding_workspace_bytes(shape, vocabulary, b, runs, ctypes.byref(n))
    return status, n.value


BAD_SHAPES = [(dict(points=-1), "points"), (dict(points=1 << 31), "points"), (dict(positions=0), "positions"), (dict(channels=0), "channels"),
              (dict(channels=(1 << 24) + 1), "channels"), (dict(dtype=2), "dtype"), (dict(points=1 << 16, positions=1 << 15), "points, positions"),
              (dict(points=(1 << 31) - 1, positions=(1 << 31) - 1), "points, positions")]


@pytest.mark.parametrize("bad,text", BAD_SHAPES, ids=lambda b: str(b))
def test_shapes(bad, text):
    _refused(_lookup(_shape(**bad)), text)
    _refused(_gradient(_shape(**bad)), text)
    _refused(_embedding_bytes(_shape(**bad))[0], text)


def test_lookup_arguments():
    for vocabulary in (0, -1, (1 << 28) + 1):
        _refused(_lookup(vocabulary=vocabulary), "vocabulary")
    for scale in (NAN, INF, -INF):
        _refused(_lookup(scale=scale), "scale")
    _refused(_lookup(dtype=2), "table_dtype")
    _refused(_lookup(tokens=(0, 6, 1)), "tokens")
    _refused(_lookup(tokens=(HERE + 4, 6, 1)), "tokens")
    _refused(_lookup(tokens=(HERE, -6, 1)), "tokens")
    _refused(_lookup(tokens=(HERE, (1 << 40) + 1, 1)), "tokens")
    _refused(_lookup(table=0), "table")
    _refused(_lookup(table=HERE + 2), "table")
    _refused(_lookup(table=HERE + 1, dtype=BF16), "table")
    _refused(_lookup(y=_view(0)), "y")
    _refused(_lookup(y=_view(HERE + 2)), "y")
    _refused(_lookup(y=_view(HERE, 119, 20)), "overlap")
    _refused(_lookup(y=_view(HERE, 0, 20)), "overlap")


def test_gradient_arguments():
    for vocabulary in (0, (1 << 28) + 1):
        _refused(_gradient(vocabulary=vocabulary), "vocabulary")
    for scale in (NAN, INF):
        _refused(_gradient(scale=scale), "scale")
    _refused(_gradient(dy=_view(0)), "dy")
    _refused(_gradient(tokens=(0, 6, 1)), "tokens")
    _refused(_gradient(tokens=(HERE + 4, 6, 1)), "tokens")
    _refused(_gradient(dtable=0), "dtable")
    _refused(_gradient(dtable=HERE + 2), "dtable")
    _refused(_gradient(runs=2), "bounds")
    _refused(_gradient(bounds=[0, 4], runs=0), "runs")
    for bounds in ([1, 4], [0, 3], [0, 5], [0, 3, 2, 4], [0, -1, 4]):
        _refused(_gradient(bounds=bounds, runs=len(bounds) - 1), "bounds")
        _refused(_embedding_bytes(_shape(), bounds=bounds, runs=len(bounds) - 1)[0], "bounds")
    status, need = _embedding_bytes(_shape())
    assert status == cr.CR_OK and need > 0
    for at, have in ((0, need), (HERE, need - 1), (HERE + 128, need)):
        _refused(_gradient(ws=at, nbytes=have), "workspace")
    _refused(cr.load_layers_library().cr_embedding_workspace_bytes(_shape(), 30, None, 1, None), "backward_bytes")


def test_the_workspace_of_a_gradient():
    """No points need none; what is said of its size."""
    assert _embedding_bytes(_shape(points=0)) == (cr.CR_OK, 0)
    for points, positions, channels, vocabulary, runs in ((4, 6, 20, 30, 1), (3000, 100, 64, 50_000, 7), (1, 1 << 30, 1, 1 << 28, 1), (400, 3, 8, 1000, 400)):
        bounds = [points * r // runs for r in range(runs + 1)]
        status, need = _embedding_bytes(_shape(points, positions, channels, BF16), vocabulary, bounds, runs)
        n = points * positions
        most = 17 * n + (n // 16 + 1) * 8 * channels + min(runs, 128) * vocabulary + 512 * 1024 + 8 * 256
        assert status == cr.CR_OK and 16 * (n // runs) <= need <= most


def test_the_workspace_of_batches_of_runs_without_points():
    """Runs are taken 128 at a time: a batch of them may have no points at all."""
    for bounds in ([0] * 300 + [211], [0] + [211] * 300, [0] * 150 + [100] * 150 + [211]):
        status, need = _embedding_bytes(_shape(211, 6, 20, BF16), 70, bounds, len(bounds) - 1)
        assert status == cr.CR_OK and need >= 17 * 100 * 6


def _scores(rows=3, classes=10, dtype=F32, logits=HERE, stride=10, tokens=HERE, logp=HERE, entropy=0, top=0, index=0, values=0, largest=0, log_sum=0, ws=0, nbytes=0):
    return cr.load_layers_library().cr_log_probs(rows, classes, dtype, logits, stride, tokens, logp, entropy, top, index, values, largest, log_sum, ws, nbytes, 0)


def _score_gradient(rows=3, classes=10, dtype=F32, logits=HERE, stride=10, tokens=HERE, largest=HERE, log_sum=HERE, entropy=HERE, dlogp=HERE, dentropy=HERE, dlogits=HERE, dstride=10):
    return cr.load_layers_library().cr_log_probs_backward(rows, classes, dtype, logits, stride, tokens, largest, log_sum, entropy, dlogp, dentropy, dlogits, dstride, 0)


def _distil(rows=3, classes=10, dtype=F32, logits=HERE, stride=10, top=2, index=HERE, values=HERE, top_stride=2, T=1.0, weights=0, loss=HERE, dlogits=0, dstride=10):
    return cr.load_layers_library().cr_distill_loss(rows, classes, dtype, logits, stride, top, index, values, top_stride, T, weights, loss, dlogits, dstride, 0, 0, 0)


@pytest.mark.parametrize("call", [_scores, _score_gradient, _distil])
def test_rows_of_logits(call):
    _refused(call(rows=-1), "rows")
    _refused(call(rows=1 << 31), "rows")
    _refused(call(classes=0), "classes")
    _refused(call(classes=(1 << 28) + 1), "classes")
    _refused(call(dtype=5), "dtype")
    _refused(call(logits=0), "logits")
    _refused(call(logits=HERE + 2), "logits")
    _refused(call(logits=HERE + 1, dtype=BF16), "logits")
    _refused(call(stride=-1), "strides")
    _refused(call(rows=(1 << 31) - 1, stride=1 << 40), "logits")
    assert call(rows=0, logits=0) == cr.CR_OK


def test_log_probs_arguments():
    for top in (-1, 129):
        _refused(_scores(top=top), "top")
    _refused(_scores(tokens=0), "tokens, logp")
    _refused(_scores(logp=0), "tokens, logp")
    _refused(_scores(tokens=HERE + 4), "tokens")
    _refused(_scores(logp=HERE + 2), "logp")
    _refused(_scores(entropy=HERE + 1), "entropy")
    _refused(_scores(top=3, values=HERE), "top_index")
    _refused(_scores(top=3, index=HERE + 4, values=HERE), "top_index")
    _refused(_scores(top=3, index=HERE), "top_logp")
    _refused(_scores(top=3, index=HERE, values=HERE + 2), "top_logp")
    _refused(_scores(largest=HERE), "largest, log_sum")
    _refused(_scores(log_sum=HERE), "largest, log_sum")
    _refused(_scores(largest=HERE, log_sum=HERE + 2), "log_sum")
    lib, n = cr.load_layers_library(), ctypes.c_size_t()
    assert lib.cr_log_probs_workspace_bytes(2, 1 << 22, F32, 5, ctypes.byref(n)) == cr.CR_OK and n.value > 0
    for at, have in ((0, n.value), (HERE, n.value - 1), (HERE + 128, n.value)):
        _refused(_scores(rows=2, classes=1 << 22, stride=1 << 22, top=5, index=HERE, values=HERE, ws=at, nbytes=have), "workspace")
    _refused(lib.cr_log_probs_workspace_bytes(2, 100, F32, 5, None), "bytes")
    _refused(lib.cr_log_probs_workspace_bytes(2, 100, F32, 129, ctypes.byref(n)), "top")


def test_log_probs_gradient_arguments():
    for name, text in (("tokens", "tokens, dlogp"), ("dlogp", "tokens, dlogp"), ("entropy", "entropy, dentropy"), ("dentropy", "entropy, dentropy"), ("largest", "largest"),
                       ("log_sum", "log_sum"), ("dlogits", "dlogits")):
        _refused(_score_gradient(**{name: 0}), text)
        _refused(_score_gradient(**{name: HERE + 2}), name)
    _refused(_score_gradient(dstride=9), "overlap")


def test_distill_arguments():
    for top in (0, -1, 129):
        _refused(_distil(top=top), "top")
    _refused(_distil(index=0), "top_index")
    _refused(_distil(index=HERE + 4), "top_index")
    _refused(_distil(values=0), "top_logits")
    _refused(_distil(values=HERE + 2), "top_logits")
    _refused(_distil(top_stride=-1), "top_logits")
    for T in (0.0, -1.0, NAN, INF, 2.0 ** -41, 2.0 ** 41):
        _refused(_distil(T=T), "temperature")
    _refused(_distil(weights=HERE + 1), "weights")
    _refused(_distil(loss=0), "loss")
    _refused(_distil(loss=HERE + 2), "loss")
    _refused(_distil(dlogits=HERE + 2), "dlogits")
    _refused(_distil(dlogits=HERE, dstride=9), "overlap")
    lib, n = cr.load_layers_library(), ctypes.c_size_t()
    assert lib.cr_distill_loss_workspace_bytes(2, 1 << 22, F32, 5, ctypes.byref(n)) == cr.CR_OK
    if n.value:
        for at, have in ((0, n.value), (HERE, n.value - 1), (HERE + 128, n.value)):
            _refused(lib.cr_distill_loss(2, 1 << 22, F32, HERE, 1 << 22, 5, HERE, HERE, 5, 1.0, 0, HERE, 0, 0, at, have, 0), "workspace")
    _refused(lib.cr_distill_loss_workspace_bytes(2, 100, F32, 5, None), "bytes")
    _refused(lib.cr_distill_loss_workspace_bytes(2, 100, F32, 0, ctypes.byref(n)), "top")


def test_names_of_the_package():
    for name in layers.LAYERS_EXPORTS:
        assert getattr(cr, name) is getattr(layers, name)


def test_the_binding_wants_tensors_on_the_gpu():
    x, t = torch.zeros(4, 20), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError):
        cr.cr_embedding_forward(t, x, x)
    with pytest.raises(ValueError):
        cr.cr_embedding_backward(x, t, x)
    with pytest.raises(ValueError):
        cr.cr_log_probs(x, t, torch.zeros(4))
    with pytest.raises(ValueError):
        cr.cr_log_probs_backward(x, t, *(torch.zeros(4) for _ in range(5)), x)
    with pytest.raises(ValueError):
        cr.cr_distill_loss(x, t[:, None], x[:, :1], torch.zeros(4))


@pytest.mark.gpu
def test_the_binding_checks_shapes_types_and_strides():
    def f(*shape, dtype=torch.float32):
        return torch.zeros(*shape, dtype=dtype, device="cuda")

    def refused(call, *args, **more):
        with pytest.raises((ValueError, cr.CodedReduceError)):
            call(*args, **more)

    i64 = torch.int64
    y, table, tokens = f(4, 6, 20), f(30, 20), f(4, 6, dtype=i64)
    cr.cr_embedding_forward(tokens, table, y)
    for bad in (tokens.int(), tokens[:3], tokens[:, :5], tokens.cpu(), f(4, 6, 1, dtype=i64), f(24, dtype=i64)):
        refused(cr.cr_embedding_forward, bad, table, y)
        refused(cr.cr_embedding_backward, y, bad, table)
    for bad in (f(30, 21), f(20, 30).t(), table.half(), f(30, 20, 1), table.cpu()):
        refused(cr.cr_embedding_forward, tokens, bad, y)
    refused(cr.cr_embedding_forward, tokens, table, y[:, :1].expand(4, 6, 20))
    refused(cr.cr_embedding_forward, tokens, table, y.half())
    refused(cr.cr_embedding_forward, tokens, table, y, scale=INF)
    refused(cr.cr_embedding_forward, tokens, f(0, 20), y)
    for bad in (f(30, 21), f(2, 30, 20), f(30, 20, dtype=torch.bfloat16), f(20, 30).t(), f(20)):
        refused(cr.cr_embedding_backward, y, tokens, bad)
    refused(cr.cr_embedding_backward, y, tokens, f(2, 30, 20), bounds=[0, 3])
    refused(cr.cr_embedding_backward, y, tokens, f(2, 30, 20), bounds=[0, 3, 2])
    refused(cr.cr_embedding_backward, y, tokens, table, workspace=f(4))
    x, t, v = f(5, 12), f(5, dtype=i64), f(5)
    cr.cr_log_probs(x, t, v)
    refused(cr.cr_log_probs, x, t)
    refused(cr.cr_log_probs, x, None, v)
    refused(cr.cr_log_probs, x, t.int(), v)
    refused(cr.cr_log_probs, x, t[:4], v)
    refused(cr.cr_log_probs, x.half(), t, v)
    refused(cr.cr_log_probs, f(5, 2, 6), t, v)
    refused(cr.cr_log_probs, f(12, 5).t(), t, v)
    refused(cr.cr_log_probs, x, t, v, entropy=f(4))
    refused(cr.cr_log_probs, x, top_index=f(5, 3, dtype=i64))
    refused(cr.cr_log_probs, x, top_index=f(5, 3, dtype=i64), top_logp=f(5, 4))
    refused(cr.cr_log_probs, x, top_index=f(5, 129, dtype=i64), top_logp=f(5, 129))
    refused(cr.cr_log_probs, x, top_index=f(4, 3, dtype=i64), top_logp=f(4, 3))
    refused(cr.cr_log_probs, x, top_index=f(3, 5, dtype=i64).t(), top_logp=f(5, 3))
    refused(cr.cr_log_probs, x, top_index=f(5, 3), top_logp=f(5, 3))
    refused(cr.cr_log_probs, x, largest=v)
    refused(cr.cr_log_probs_backward, x, t, v, v, v, v, v, x[:4])
    refused(cr.cr_log_probs_backward, x, t, v, v, v, v, v, x.bfloat16())
    refused(cr.cr_log_probs_backward, x, t, v, v, v, None, v, x)
    refused(cr.cr_log_probs_backward, x, t, v, None, v, v, v, x)
    refused(cr.cr_log_probs_backward, x, t, v, v, None, v, v, x)
    j, z = f(5, 3, dtype=i64), f(5, 3)
    cr.cr_distill_loss(x, j, z, v)
    refused(cr.cr_distill_loss, x, j.int(), z, v)
    refused(cr.cr_distill_loss, x, j, z.bfloat16(), v)
    refused(cr.cr_distill_loss, x, j[:4], z[:4], v)
    refused(cr.cr_distill_loss, x, j[:, :2], z, v)
    refused(cr.cr_distill_loss, x, f(5, 6, dtype=i64)[:, ::2], f(5, 6)[:, ::2], v)
    refused(cr.cr_distill_loss, x, f(5, 6, dtype=i64)[:, :3], z, v)
    refused(cr.cr_distill_loss, x, f(5, 0, dtype=i64), f(5, 0), v)
    refused(cr.cr_distill_loss, x, f(5, 129, dtype=i64), f(5, 129), v)
    refused(cr.cr_distill_loss, x, j, z, v, temperature=0.0)
    refused(cr.cr_distill_loss, x, j, z, v[:4])
    refused(cr.cr_distill_loss, x, j, z, v, weights=f(4))
    refused(cr.cr_distill_loss, x, j, z, v, dlogits=f(5, 11))
