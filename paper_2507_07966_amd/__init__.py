"""Prefix-shared GRPO prefill attention for MI355X (gfx950), and the attention over a paged cache that samples the rollouts.

`workloads` (seeded synthetic inputs) is plain numpy.  Everything else is the thin
ctypes binding over the C-ABI library built from csrc/; it is imported on first
use and raises if the library has not been built.
"""
from . import workloads  # noqa: F401

_BINDING_NAMES = ("PrefixAttnPlan", "PrefixAttnError", "prefix_attn_plan", "prefix_attn_forward", "prefix_attn_forward_static",
                  "prefix_attn_forward_timed", "STATIC_SCRATCH_BYTES",
                  "prefix_attn_lse", "prefix_attn_destroy", "prefix_attn_status_string",
                  "prefix_attn_backward", "prefix_attn_backward_timed", "prefix_attn_forward_partial",
                  "prefix_attn_merge_partials", "token_logprob_workspace", "token_logprob_forward",
                  "grpo_group_advantages",
                  "library_path", "load_library")


_SAMPLING_NAMES = ("RopeAxes", "rope_axes", "rope_axes_forward", "rope_axes_backward", "PagedAttnPlan", "paged_attn_plan",
                   "paged_kv_append", "paged_kv_append_rope", "paged_attn_forward")


def __getattr__(name):
    if name == "sampling" or name in _SAMPLING_NAMES:
        import importlib
        mod = importlib.import_module(".sampling", __name__)
        return mod if name == "sampling" else getattr(mod, name)
    if name == "binding" or name in _BINDING_NAMES:
        import importlib
        mod = importlib.import_module(".binding", __name__)
        return mod if name == "binding" else getattr(mod, name)
    raise AttributeError(name)
