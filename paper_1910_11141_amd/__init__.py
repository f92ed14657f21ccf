"""Lock-step NUTS on MI355X: Python face of the C-ABI library (see include/nuts.h)."""
import importlib

from . import workloads  # noqa: F401  (pure numpy: safe without the HIP library)

# what categorical.py has, which imports PyTorch: not for who asks for something else
_CATEGORICAL = ("nuts_lookup", "nuts_lookup_grad", "nuts_logprobs", "nuts_logprobs_grad", "nuts_score", "nuts_score_grad", "Logprobs", "Scores",
                "nuts_penalties", "nuts_penalties_grad")
# and learning.py, which does, too
_LEARNING = ("nuts_norm", "nuts_adamw", "nuts_adamw_values", "Moments", "Norm")


def __getattr__(name):
    # The binding is loaded on first use so that `workloads` stays importable on a
    # machine where the library has not been built; using the sampler without the
    # library raises (there is no CPU path).
    if name.startswith("__"):
        raise AttributeError(name)
    if name in _CATEGORICAL:  # (calls of a few microseconds: found here from now on)
        return globals().setdefault(name, getattr(importlib.import_module(__name__ + ".categorical"), name))
    if name in _LEARNING:
        return globals().setdefault(name, getattr(importlib.import_module(__name__ + ".learning"), name))
    return getattr(importlib.import_module(__name__ + ".binding"), name)
