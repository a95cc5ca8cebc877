"""MI355X-native PAHQ / ACDC edge-ablation path: thin Python binding over libpahq.so."""
import importlib as _importlib
import importlib.util as _importlib_util

from .binding import (lib, PahqError, Config, Model, n_senders, n_receivers, n_upstream, edge_count, edge_id,
                      node_of_receiver, workspace_bytes, measure_ceilings, quantize_rows_noalloc, tau_grid, rotary_entries, TraceRec,
                      ALL_FP32, ALL_FP8, PAHQ, MMA_FP8, MMA_F16_EXACT, METRIC_KL, METRIC_LOGIT_DIFF, W_Q, W_K, W_V, W_O, W_IN, W_GATE, W_OUT, W_U)

_OF_TENSORS = ("Mx4", "mx4_quantize", "mx4_dequantize", "mx4_gemm", "rotary_table", "rotary")
__all__ = [_n for _n in globals() if not _n.startswith("_")] + (list(_OF_TENSORS) if _importlib_util.find_spec("torch") else [])


def __getattr__(name):
    """The operators on device tensors, at their first use: they need torch, which takes seconds to import and which no other part
    of the package needs before it meets a GPU."""
    if name == "tensors" or name in _OF_TENSORS:
        tensors = _importlib.import_module(".tensors", __name__)
        globals().update({n: getattr(tensors, n) for n in _OF_TENSORS})
        return globals()[name]
    raise AttributeError("module %r has no attribute %r" % (__name__, name))


def __dir__():
    return sorted({*globals(), *_OF_TENSORS})
