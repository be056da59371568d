"""The package's names without torch, which the layers' binding needs and nothing else does."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = """
import sys
sys.modules["torch"] = None                              # an import of it fails
import paper_1902_01981_amd as cr
assert not hasattr(cr, "cr_no_such_call") and not hasattr(cr, "cr_plan_no_such") and not hasattr(cr, "anything")
assert "paper_1902_01981_amd.layers" not in sys.modules
for name in ("cr_group_norm_forward", "cr_dropout_t", "cr_softmax_loss", "cr_layer_shape_t", "cr_layers_last_error", "CR_ACT_SILU", "LAYERS_EXPORTS", "load_layers_library"):
    try:
        getattr(cr, name)
    except ImportError:
        continue
    raise AssertionError(name)
print("done")
"""


def test_names_without_torch():
    done = subprocess.run([sys.executable, "-c", PROGRAM], cwd=ROOT, capture_output=True, text=True)
    assert done.stdout == "done\n", done.stderr


def test_names_with_torch():
    import paper_1902_01981_amd as cr
    from paper_1902_01981_amd import layers

    for name in layers.LAYERS_EXPORTS + ["cr_layer_shape_t", "cr_layer_view_t", "cr_dropout_t", "CR_ACT_NONE", "CR_ACT_RELU", "CR_ACT_SILU", "LAYERS_LIB_PATH", "LAYERS_EXPORTS",
                                         "load_layers_library"]:
        assert getattr(cr, name) is getattr(layers, name)
