"""Rift hot path on AMD Instinct MI355X: query-conditioned tile scoring and
pruning, elastic per-tile token selection, varlen compaction and LLaMA-7B-shaped
prefill, as hand-written HIP kernels behind the C ABI of include/rift.h."""
from ._lib import (EXPORTS, LIB_PATH, RIFT_BF16, RIFT_F32, LayerWeights, ModelCfg,  # noqa: F401
                   RiftError, lib_available, load, model_cfg, rift_assign_budgets,
                   rift_assign_budgets_utility, rift_check_finite, rift_compact, rift_decode_step,
                   rift_decode_workspace_size,
                   rift_merge_context, rift_merge_workspace_size, rift_prefill,
                   rift_prefill_workspace_size, rift_score_tiles, rift_score_tiles_noalloc,
                   rift_score_workspace_size,
                   rift_select_tokens, rift_set_debug, rift_split_budgets)
from .kv import (KV_EXPORTS, RIFTKV_BF16, RIFTKV_F32, RIFTKV_FP8, RIFTKV_INT8, KvCache, riftkv_attention,  # noqa: F401
                 riftkv_attention_pages, riftkv_attention_pages_workspace_size, riftkv_attention_shared,
                 riftkv_attention_shared_workspace_size,
                 riftkv_attention_workspace_size, riftkv_cache, riftkv_decode_step, riftkv_decode_workspace_size,
                 riftkv_page_bounds, riftkv_read, riftkv_rope, riftkv_rope_axes, riftkv_rope_freqs, riftkv_select_pages,
                 riftkv_select_pages_workspace_size, riftkv_write)
