"""MI355X-native sparsity-aware LDA sampler (hot path of SaberLDA) behind a C ABI.

``Saber`` wraps the ``saber_*`` calls of ``include/saber.h``; the work is done by
the HIP kernels in ``csrc/``.  ``ops`` holds the operators of a head that is trained on a
model's features (layer norm, softmax cross entropy over the vocabulary, 8-bit checkpoints);
it works on torch tensors and is imported when it is first asked for (torch before the sampler's
first use, so that both are on one HIP runtime).
"""
from .binding import (EXPORTS, Options, Saber, SaberError, Stats, bandwidth_probe, clear_hooks, library_path,
                      load_library, options_default, set_hooks, set_torch_hooks)

__all__ = ["EXPORTS", "Options", "Saber", "SaberError", "Stats", "bandwidth_probe", "clear_hooks", "library_path",
           "load_library", "options_default", "set_hooks", "set_torch_hooks"]


def __getattr__(name):
    if name == "ops":
        import importlib
        return importlib.import_module(".ops", __name__)
    raise AttributeError("module %r has no attribute %r" % (__name__, name))
