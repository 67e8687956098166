"""B200-native GDN tree verification and commit (Section 3.4 of "Trees from Marginals").

``gdn_tree_verify`` and ``gdn_tree_commit`` are thin bindings over the C-ABI CUDA library built from ``csrc/``;
``gdn_kv_append``, ``gdn_kv_commit``, ``gdn_attn_decode``, ``gdn_attn_tree_verify`` and ``gdn_sample``
serve the full-attention layers and the output layer of the same model; ``synth`` holds the seeded synthetic workload generators.  There is no CPU fallback: every call raises if the CUDA
library has not been built.
"""
from . import synth  # noqa: F401
from .binding import (  # noqa: F401
    GdnAttnShape,
    GdnSampleShape,
    GdnShape,
    gdn_attn_decode,
    gdn_attn_tree_verify,
    gdn_attn_workspace_bytes,
    gdn_kv_append,
    gdn_kv_commit,
    gdn_sample,
    gdn_status_string,
    gdn_tree_commit,
    gdn_tree_commit_host,
    gdn_tree_commit_padded,
    gdn_tree_commit_verify,
    gdn_tree_commit_verify_padded,
    gdn_tree_commit_verify_host,
    gdn_tree_commit_verify_host_arena_bytes,
    gdn_tree_host_arena_bytes,
    gdn_tree_plan,
    gdn_tree_plan_bytes,
    gdn_tree_validate_host,
    gdn_tree_verify,
    gdn_tree_verify_host,
    gdn_tree_verify_padded,
    gdn_tree_verify_planned,
    gdn_tree_verify_recurrent,
    gdn_tree_verify_static,
    gdn_tree_workspace_bytes,
    library_path,
    load_library,
)
