"""SAKI coupling-and-routing path on AMD MI355X (gfx950).

The compute lives in libsaki.so (HIP kernels behind the C ABI of
include/saki.h, saki_kv.h and saki_distill.h); this package is its thin Python binding.
"""
from .binding import (  # noqa: F401
    COUPLE_FIELDS, EXPORTED, EXPORTED_DISTILL, EXPORTED_KV, KV_BAD, KV_NO_PAGES, KV_OK, KV_TOO_LONG, SAKI_BF16, SAKI_CHUNK, SAKI_F32,
    SAKI_KL_FORWARD, SAKI_KL_REVERSE, SAKI_MAX_TOP_K, SAKI_MAX_VOCAB, SAKI_OP_COUPLE, SAKI_OP_DISTILL_TOP,
    SAKI_OP_KV_ATTENTION, SAKI_OP_KV_COMPACT, SAKI_OP_KV_RESERVE, SAKI_OP_ROUTE,
    SAKI_OP_SELECT, SAKI_OP_TOP_LOGITS, SAKI_OP_VERIFY, SAKI_SELECT_RANDOM, SAKI_SELECT_TV_WEIGHTED, SAKI_STATIC_MAX_ROWS,
    SAKI_TARGET_MODE, SAKI_TARGET_SAMPLE, SEQ_FINISHED, SEQ_RUNNING, SEQ_STOPPED, SakiError,
    alloc_couple_out, alloc_rows, alloc_traj, couple,
    distill_top, linear_ce, linear_ce_workspace_bytes, load, probe_metrics, route_loss, sample, saki_commit, saki_couple, saki_couple_static,
    saki_distill_top, saki_linear_ce, saki_probe_metrics, saki_route_loss, saki_sample, saki_select_positions, saki_spec_verify, saki_top_logits,
    select_positions, spec_verify, top_logits, workspace_bytes)
from .cache import PagedKV, rope  # noqa: F401
from .speculative import rollout  # noqa: F401
