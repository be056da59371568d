"""Views whose strides are allowed one by one, but together reach past what an offset of 64 bits can say: refused, not wrapped around.  (No launch follows.)"""
import ctypes

import pytest

import paper_1902_01981_amd as cr
from paper_1902_01981_amd import layers

HERE = 0x10000                                           # an address nobody reads
MOST = 1 << 40                                           # of a stride


def _refused(status, text):
    assert status == cr.CR_E_INVAL and text in cr.cr_layers_last_error(), (status, cr.cr_layers_last_error())


def _dropout(points, positions, x, y):
    shape = layers.cr_layer_shape_t(points, positions, 4, cr.CR_BF16)
    return cr.load_layers_library().cr_dropout_forward(shape, layers.cr_layer_view_t(HERE, *x), 0, None, layers.cr_dropout_t(0.1, 0, 0, 0, 0, 0),
                                                       layers.cr_layer_view_t(HERE, *y), 0)


@pytest.mark.parametrize("points,positions", [(2, (1 << 23) + 1), (2, 1 << 24), (2, (1 << 31) - 1), ((1 << 23) + 1, 2), ((1 << 31) - 1, 3), (1, (1 << 31) - 1)])
def test_outputs(points, positions):
    """Both strides the largest: where there are two dimensions, rows overlap, however far the product of a stride and a count has wrapped."""
    _refused(_dropout(points, positions, (4, 0), (MOST, MOST)), "y")


@pytest.mark.parametrize("points,positions,point,position", [((1 << 31) - 1, 1, MOST, 0), (1, (1 << 31) - 1, 0, MOST), (1 << 30, 1 << 30, 1 << 29, MOST),
                                                             (1 << 24, 1 << 24, 1 << 39, 1 << 39)])
def test_inputs(points, positions, point, position):
    _refused(_dropout(points, positions, (point, position), (4 * positions, 4)), "x")


def test_rows_of_logits():
    _refused(cr.load_layers_library().cr_softmax_loss((1 << 31) - 1, 4, cr.CR_F32, HERE, MOST, HERE, 0, HERE, 0, 0, 0, 0, 0, 0), "logits")


def test_what_overlaps_by_one_element_at_the_border():
    """The largest extents that a device could hold are judged exactly."""
    shape, n, p, c = layers.cr_layer_shape_t, 1 << 10, 1 << 16, 1 << 12
    block = (p - 1) * (1 << 12) + c
    drop = layers.cr_dropout_t(0.1, 0, 0, 0, 0, 0)
    for point, text in ((block - 1, "overlap"), (block, None)):
        status = cr.load_layers_library().cr_dropout_forward(shape(n, p, c, cr.CR_BF16), layers.cr_layer_view_t(0, 0, 0), 0, None, drop,
                                                             layers.cr_layer_view_t(HERE, point, 1 << 12), 0)
        _refused(status, "x is required")                # inputs are looked at first: no launch follows
        status = cr.load_layers_library().cr_group_norm_backward(shape(n, p, c, cr.CR_BF16), layers.cr_layer_view_t(HERE, 0, 0), layers.cr_layer_view_t(HERE, 0, 0), HERE,
                                                                 HERE, 0, 0, 1, 0, None, 1, layers.cr_layer_view_t(HERE, point, 1 << 12), 0, 0, 0, 0, 0)
        _refused(status, text or "workspace")            # what is right comes to a missing workspace


def _gradient_bytes(points, positions, channels=1, dtype=cr.CR_BF16):
    f, b = ctypes.c_size_t(), ctypes.c_size_t()
    status = cr.load_layers_library().cr_group_norm_workspace_bytes(layers.cr_layer_shape_t(points, positions, channels, dtype), 1, 0, 1, ctypes.byref(f), ctypes.byref(b))
    return status, b.value


def test_pieces_of_points():
    """Points cut into pieces leave a row of sums per piece.  Below 2^31 of them the workspace holds them all, above the gradient is refused (inputs that are
    broadcast can be so large)."""
    for points, positions in ((1 << 10, 1 << 16), (1 << 20, 1 << 20), (1 << 24, 1 << 19)):
        status, nbytes = _gradient_bytes(points, positions)
        pieces = points * positions // (256 * 64)        # threads of a workgroup, most positions of a thread
        assert status == cr.CR_OK and nbytes >= 2 * 4 * pieces
    _refused(_gradient_bytes(1 << 24, 1 << 24)[0], "points")
    _refused(_gradient_bytes((1 << 31) - 1, (1 << 31) - 1)[0], "points")
    view, lib = layers.cr_layer_view_t(HERE, 0, 0), cr.load_layers_library()
    _refused(lib.cr_group_norm_backward(layers.cr_layer_shape_t(1 << 24, 1 << 24, 1, cr.CR_BF16), view, view, HERE, HERE, 0, 0, 1, 0, None, 1, None, HERE, HERE, 0, 0, 0),
             "points")
