"""MI355X-native CodedReduce hot path and network layers: thin ctypes bindings over libcodedreduce.so and libcodedreduce_layers.so (argument
marshalling only).  The layers' binding, which needs torch, is imported when one of its names is first asked for."""
from .api import *  # noqa: F401,F403


def __getattr__(name):
    if name.startswith(("cr_layer", "cr_group_norm_", "cr_dropout_", "cr_softmax_loss", "cr_embedding_", "cr_log_probs", "cr_distill_loss", "CR_ACT_", "LAYERS_", "load_layers")):
        from . import layers

        if hasattr(layers, name):
            value = globals()[name] = getattr(layers, name)              # asked for once
            return value
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
