"""MI355X (gfx950) implementation of NaCl's one-shot encoding-phase KV-cache
eviction (arXiv 2408.03675): HIP kernels behind the C ABI of include/nacl.h,
with a thin ctypes binding."""

from .nacl import (  # noqa: F401
    NaclError, Problem, SAMPLE_PROPORTIONAL, SAMPLE_SOFTMAX, SAMPLE_UNIFORM, EXPORTED,
    LIB_PATH, load_library, workspace_bytes, workspace, score, select, compact, compact_slots, evict,
    evict_slots, attention, Step, Rotation, Prefix, rotate_append, prefix_workspace, prefix_attention,
    sample_workspace, sample, Pages, pages_assign, paged_append, paged_workspace, paged_attention,
    beam_workspace, beam_select, beam_reorder,
)
