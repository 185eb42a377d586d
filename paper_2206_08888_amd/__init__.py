"""MI355X-native population TD3 update engine (C-ABI HIP library + thin binding).

The computation lives entirely in libpop.so (hand-written gfx950 kernels);
this package only marshals arguments.  PyTorch is used by callers to allocate
the device workspace and to supply a stream.
"""
from importlib import import_module as _import_module
from importlib.util import find_spec as _find_spec

from .binding import (  # noqa: F401
    POP_ALGO_SAC, POP_ALGO_TD3, POP_ALGO_TD3_SHARED, POP_LAUNCH_AUTO, POP_LAUNCH_PER_PART, POP_LAUNCH_SINGLE, POP_LAUNCH_TAIL,
    POP_LAUNCH_TARGET_CRITIC, POP_OPT_WAIT_LIMIT_TICKS, POP_EEMPTY, POP_EHIP, POP_EINVAL, POP_ENOMEM, POP_EUNSUPPORTED, POP_OK,
    PARAM_CODES, DEBUG_CODES, PopError, Population, lib_path, load_library, make_config, make_hparams,
    pop_act, pop_act_explore, pop_act_explore_noalloc, pop_buffer_count, pop_create, pop_debug_get, pop_debug_indices, pop_destroy, pop_get_params,
    pop_insert, pop_last_error, pop_net_size, pop_copy_agent, pop_set_debug, pop_set_hparams, pop_set_option, pop_get_tuning, pop_set_params, pop_step_count, pop_sync, pop_update, pop_update_timed, KERNEL_NAMES,
    pop_workspace_bytes, pop_config, pop_hparams, pop_tuning,
    NS_COEF, POP_BF16, POP_F16, POP_F32, make_ns_config, pop_matrices, pop_muon_layer, pop_ns_config, pop_recurrence_config,
    pop_recurrence_grads, pop_recurrence_io, pop_sequence,
    pop_gradient, pop_heads, pop_linear_config, pop_linear_grads, pop_linear_io,
)

_ON_TENSORS = ("GradientClip", "LinearAttention", "Muon", "Orthogonalizer", "Recurrence", "operators")
__all__ = [name for name in globals() if not name.startswith("_")] + list(_ON_TENSORS if _find_spec("torch") else ())


def __getattr__(name):
    """The operators on tensors, which need PyTorch, when they are first asked for: the rest does without it."""
    if name not in _ON_TENSORS:
        raise AttributeError("module %r has no attribute %r" % (__name__, name))
    module = _import_module(".operators", __name__)
    return module if name == "operators" else getattr(module, name)


def __dir__():
    return sorted(set(globals()) | set(_ON_TENSORS))
