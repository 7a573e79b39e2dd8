"""n-softsync parameter-server update (arXiv 1511.05950) as sm_100a CUDA kernels behind a C ABI.

`binding` loads libsoftsync_ps.so and mirrors its entry points; `learn` holds the operators for language-model learners and
their server (losses from logits and without them, a norm and activations in 8 bits, gradient norm, AdamW).  Everything the two export is reachable
from this package (`paper_1511_05950_b200.ParameterServer`, `.AdamW`, `.ps_create`, ...).  The binding is
loaded on first use, so that `paper_1511_05950_b200.build` can be imported to build the library
first; using anything else without the built library raises (there is no CPU fallback).  The server needs the library
alone; what `learn` exports needs the _marshal extension too.
"""
import importlib

_LEARN = frozenset(("AdamW", "AdamWServer", "HeadCrossEntropy", "HeadGrad", "HeadLogprob", "INPLACE", "Packed8", "PolicyLoss", "PreferenceLoss",
                    "RmsNorm", "RmsNormGrad", "TensorList", "TokenLogprob", "head_cross_entropy", "head_logprob", "head_logprob_grad", "norm_linear",
                    "pack8", "packed_weight_grad", "policy_loss", "preference_loss", "rms_norm", "rms_norm_grad", "token_logprob", "unpack8"))


def __getattr__(name):
    if name.startswith("__"):
        raise AttributeError(name)
    if name == "build":                      # importable before the library exists
        return importlib.import_module(".build", __name__)
    if name == "learn" or name in _LEARN:
        learn = importlib.import_module(".learn", __name__)
        if name == "learn":
            return learn
        globals()[name] = getattr(learn, name)               # found once: later uses do not come here
        return globals()[name]
    binding = importlib.import_module(".binding", __name__)
    if name == "binding":
        return binding
    try:
        return getattr(binding, name)
    except AttributeError:
        raise AttributeError("module %r has no attribute %r" % (__name__, name)) from None
