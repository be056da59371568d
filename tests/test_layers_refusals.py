"""What the network layers refuse, at the C boundary (no launch follows, so no GPU is needed) and in the binding; and what the library exports."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

import paper_1902_01981_amd as cr
from paper_1902_01981_amd import layers

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HERE = 0x10000                                           # an address nobody reads
ref = ctypes.byref


@pytest.mark.skipif(shutil.which("nm") is None, reason="needs nm")
def test_the_library_exports_what_its_header_declares():
    with open(os.path.join(ROOT, "include", "codedreduce_layers.h")) as f:
        declared = set(re.findall(r"^(?:int|void|const char \*)\s*\**(cr_\w+)\(", f.read(), flags=re.M))
    listed = subprocess.run(["nm", "-D", "--defined-only", cr.LAYERS_LIB_PATH], check=True, capture_output=True, text=True).stdout
    assert {line.split()[-1] for line in listed.splitlines()} == declared == set(cr.LAYERS_EXPORTS)
    cr.load_layers_library()


def _shape(points=4, positions=6, channels=20, dtype=cr.CR_F32):
    return layers.cr_layer_shape_t(points, positions, channels, dtype)


def _view(dev=HERE, point=120, position=20):
    return layers.cr_layer_view_t(dev, point, position)


def _refused(status, text):
    assert status == cr.CR_E_INVAL and text in cr.cr_layers_last_error(), cr.cr_layers_last_error()


def _forward(shape=None, x=None, gamma=0, beta=0, groups=4, eps=1e-5, activation=0, y=None, mean=0, rstd=0):
    return cr.load_layers_library().cr_group_norm_forward(_shape() if shape is None else shape, _view() if x is None else x, gamma, beta, groups, eps, activation,
                                                          _view() if y is None else y, mean, rstd, 0, 0, 0)


BAD_SHAPES = [(dict(points=-1), "points"), (dict(points=1 << 31), "points"), (dict(positions=0), "positions"), (dict(positions=1 << 31), "positions"),
              (dict(channels=0), "channels"), (dict(channels=(1 << 24) + 1), "channels"), (dict(dtype=2), "dtype"), (dict(dtype=-1), "dtype")]


@pytest.mark.parametrize("bad,text", BAD_SHAPES, ids=lambda b: str(b))
def test_shapes(bad, text):
    _refused(_forward(_shape(**bad), groups=1), text)
    drop = layers.cr_dropout_t(0.1, 0, 0, 0, 0, 0)
    _refused(cr.load_layers_library().cr_dropout_forward(_shape(**bad), _view(), 0, None, drop, _view(), 0), text)
    n, m = ctypes.c_size_t(), ctypes.c_size_t()
    _refused(cr.load_layers_library().cr_group_norm_workspace_bytes(_shape(**bad), 1, 0, 1, ref(n), ref(m)), text)
    _refused(cr.load_layers_library().cr_dropout_workspace_bytes(_shape(**bad), 0, 1, ref(n)), text)


def test_norm_arguments():
    _refused(_forward(groups=0), "groups")
    _refused(_forward(groups=3), "groups")
    _refused(_forward(groups=40), "groups")
    for eps in (-1e-5, float("nan"), float("inf")):
        _refused(_forward(eps=eps), "eps")
    _refused(_forward(activation=3), "activation")
    _refused(_forward(activation=-1), "activation")
    _refused(_forward(gamma=HERE + 2), "gamma")
    _refused(_forward(mean=HERE), "mean, rstd")
    _refused(_forward(rstd=HERE), "mean, rstd")
    _refused(_forward(x=_view(0)), "x")
    _refused(_forward(y=_view(0)), "y")
    _refused(_forward(x=_view(HERE + 1)), "x")
    _refused(_forward(x=_view(HERE, -120, 20)), "strides")
    _refused(_forward(x=_view(HERE, 120, 1 << 41)), "strides")
    lib = cr.load_layers_library()
    n, m = ctypes.c_size_t(), ctypes.c_size_t()
    _refused(lib.cr_group_norm_workspace_bytes(_shape(), 4, 0, 1, None, ref(m)), "forward_bytes")
    _refused(lib.cr_group_norm_workspace_bytes(None, 4, 0, 1, ref(n), ref(m)), "shape")


@pytest.mark.parametrize("point,position", [(120, 19), (119, 20), (20, 79), (19, 80), (0, 20), (120, 0), (20, 20)])
def test_outputs_whose_rows_overlap(point, position):
    _refused(_forward(y=_view(HERE, point, position)), "overlap")


def test_norm_backward_arguments():
    lib = cr.load_layers_library()

    def call(shape=None, dy=None, x=None, mean=HERE, rstd=HERE, groups=4, activation=0, bounds=None, runs=1, dx=None, dgamma=0, dbeta=0, ws=0, nbytes=0):
        b = None if bounds is None else (ctypes.c_int64 * len(bounds))(*bounds)
        return lib.cr_group_norm_backward(_shape() if shape is None else shape, _view() if dy is None else dy, _view() if x is None else x, mean, rstd, 0, 0, groups,
                                          activation, b, runs, dx, dgamma, dbeta, ws, nbytes, 0)

    _refused(call(mean=0), "mean")
    _refused(call(rstd=0), "rstd")
    _refused(call(dy=_view(0)), "dy")
    _refused(call(x=_view(0)), "x")
    _refused(call(dx=_view(HERE, 10, 20)), "overlap")
    _refused(call(groups=7), "groups")
    _refused(call(activation=9), "activation")
    _refused(call(runs=2), "bounds")
    _refused(call(bounds=[0, 4], runs=0), "runs")
    for bounds in ([1, 4], [0, 3], [0, 5], [0, 3, 2, 4], [0, -1, 4], [0, 5, 4]):
        _refused(call(bounds=bounds, runs=len(bounds) - 1), "bounds")
    _refused(call(dgamma=HERE + 1), "dgamma")
    _refused(call(dbeta=HERE + 2), "dbeta")


def test_workspaces():
    """Too small, missing or misaligned where one is needed."""
    lib = cr.load_layers_library()
    shape, view = _shape(200, 300, 64, cr.CR_BF16), _view(HERE, 300 * 64, 64)
    f, b = ctypes.c_size_t(), ctypes.c_size_t()
    assert lib.cr_group_norm_workspace_bytes(shape, 4, 0, 1, ref(f), ref(b)) == cr.CR_OK
    if b.value:
        for at, have in ((0, b.value), (HERE, b.value - 1), (HERE + 128, b.value)):
            _refused(lib.cr_group_norm_backward(shape, view, view, HERE, HERE, 0, 0, 4, 0, None, 1, view, HERE, HERE, at, have, 0), "workspace")
    assert lib.cr_dropout_workspace_bytes(shape, 0, 1, ref(b)) == cr.CR_OK
    if b.value:
        drop = layers.cr_dropout_t(0.1, 0, 0, 0, 0, 0)
        for at, have in ((0, b.value), (HERE, b.value - 1), (HERE + 128, b.value)):
            _refused(lib.cr_dropout_backward(shape, view, drop, view, None, 1, HERE, at, have, 0), "workspace")
    assert lib.cr_softmax_loss_workspace_bytes(1, 1 << 22, cr.CR_F32, ref(b)) == cr.CR_OK
    if b.value:
        for at, have in ((0, b.value), (HERE, b.value - 1), (HERE + 128, b.value)):
            _refused(lib.cr_softmax_loss(1, 1 << 22, cr.CR_F32, HERE, 1 << 22, HERE, 0, HERE, 0, HERE, 1 << 22, at, have, 0), "workspace")


def test_dropout_arguments():
    lib = cr.load_layers_library()

    def call(rate=0.1, dev=0, first=0, points=0, **kw):
        drop = layers.cr_dropout_t(rate, 0, 0, dev, first, points)
        return lib.cr_dropout_forward(_shape(), kw.get("x", _view()), kw.get("bias", 0), kw.get("residual"), drop, kw.get("y", _view()), 0)

    for rate in (-0.1, 1.0, 1.5, float("nan"), 1 - 2.0 ** -18):
        _refused(call(rate=rate), "rate")
    _refused(call(dev=HERE + 4), "draw_dev")
    _refused(call(points=HERE + 4), "point_dev")
    _refused(call(points=HERE, first=3), "first_point")
    _refused(call(bias=HERE + 1), "bias")
    _refused(call(x=_view(0)), "x")
    _refused(call(y=_view(HERE, 0, 20)), "overlap")
    _refused(call(residual=_view(HERE + 2)), "residual")
    _refused(lib.cr_dropout_forward(_shape(), _view(), 0, None, None, _view(), 0), "dropout")
    _refused(lib.cr_dropout_workspace_bytes(_shape(), 0, 1, None), "backward_bytes")


def test_loss_arguments():
    lib = cr.load_layers_library()

    def call(rows=3, classes=10, dtype=cr.CR_F32, logits=HERE, stride=10, targets=HERE, weights=0, loss=HERE, lse=0, dlogits=0, dstride=10):
        return lib.cr_softmax_loss(rows, classes, dtype, logits, stride, targets, weights, loss, lse, dlogits, dstride, 0, 0, 0)

    _refused(call(rows=-1), "rows")
    _refused(call(rows=1 << 31), "rows")
    _refused(call(classes=0), "classes")
    _refused(call(classes=(1 << 28) + 1), "classes")
    _refused(call(dtype=5), "dtype")
    _refused(call(logits=0), "logits")
    _refused(call(logits=HERE + 2), "logits")
    _refused(call(stride=-1), "strides")
    _refused(call(targets=0), "targets")
    _refused(call(targets=HERE + 4), "targets")
    _refused(call(loss=0), "loss")
    _refused(call(weights=HERE + 1), "weights")
    _refused(call(lse=HERE + 1), "lse")
    _refused(call(dlogits=HERE, dstride=9), "overlap")


def test_the_binding_wants_tensors_on_the_gpu():
    x = torch.zeros(4, 6, 20)
    with pytest.raises(ValueError):
        cr.cr_group_norm_forward(x, None, None, 4, x)
    with pytest.raises(ValueError):
        cr.cr_dropout_forward(x, x, 0.1, 1)
    with pytest.raises(ValueError):
        cr.cr_softmax_loss(x[0], torch.zeros(6, dtype=torch.int64), torch.zeros(6))
    with pytest.raises(TypeError):
        cr.cr_dropout_forward(HERE, x, 0.1, 1)


@pytest.mark.gpu
def test_the_binding_checks_shapes_types_and_strides():
    x = torch.zeros(4, 6, 20, device="cuda")
    ok = torch.zeros(20, device="cuda")
    stats = torch.zeros(4, 4, device="cuda")
    for bad in (x.half(), x[0, 0], x.cpu()):
        with pytest.raises(ValueError):
            cr.cr_group_norm_forward(bad, ok, ok, 4, bad)
    for y in (x.bfloat16(), x[:3], x.transpose(1, 2), torch.zeros(4, 6, 40, device="cuda")[:, :, ::2]):
        with pytest.raises(ValueError):
            cr.cr_group_norm_forward(x, ok, ok, 4, y)
    with pytest.raises(ValueError):
        cr.cr_group_norm_forward(x, ok[:10], ok, 4, x)
    with pytest.raises(ValueError):
        cr.cr_group_norm_forward(x, ok.double(), ok, 4, x)
    with pytest.raises(ValueError):
        cr.cr_group_norm_forward(x, ok, ok, 4, x, stats[:2], stats)
    with pytest.raises(ValueError):
        cr.cr_group_norm_backward(x, x, stats, None, ok, ok, 4)
    with pytest.raises(ValueError):
        cr.cr_group_norm_backward(x, x, stats, stats, ok, ok, 4, dgamma=ok, bounds=[0, 2, 4])
    with pytest.raises(cr.CodedReduceError):
        cr.cr_group_norm_backward(x, x, stats, stats, ok, ok, 4, dgamma=torch.zeros(2, 20, device="cuda"), bounds=[0, 3, 2])
    with pytest.raises(cr.CodedReduceError):
        cr.cr_group_norm_forward(x, ok, ok, 3, x)
    with pytest.raises(cr.CodedReduceError):
        cr.cr_dropout_forward(x, x[:1].expand(4, 6, 20), 0.1, 1)
    with pytest.raises(ValueError):
        cr.cr_dropout_forward(x, x, 0.1, 1, point_index=torch.zeros(3, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        cr.cr_dropout_forward(x, x, 0.1, 1, point_index=torch.zeros(4, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        cr.cr_softmax_loss(x[0], torch.zeros(6, dtype=torch.int32, device="cuda"), torch.zeros(6, device="cuda"))
    with pytest.raises(ValueError):
        cr.cr_softmax_loss(x, torch.zeros(24, dtype=torch.int64, device="cuda"), torch.zeros(24, device="cuda"))
    crossed = torch.zeros(4, 6, 5, 20, device="cuda").transpose(1, 2)
    with pytest.raises(ValueError):
        cr.cr_group_norm_forward(crossed, ok, ok, 4, torch.empty(4, 5, 6, 20, device="cuda"))
