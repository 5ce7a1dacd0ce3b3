"""SENSE retrieval + soft-gated evaluation hot path for one AMD MI355X (gfx950).

The kernels live in ``libsense.so`` (HIP, built from ``csrc/``); ``sense``
is its Python binding and ``synth`` the seeded workload generator.
"""
from .sense import (  # noqa: F401
    Index,
    SenseError,
    load_library,
    sense_build_index,
    sense_build_kv_cache,
    sense_kv_attention,
    sense_kv_compact,
    sense_kv_fork,
    sense_kv_read,
    sense_kv_reserve,
    sense_kv_truncate,
    sense_kv_write,
    sense_retrieve,
    sense_retrieve_workspace_size,
    sense_soft_gate_verify,
    sense_soft_gate_verify_workspace_size,
)
