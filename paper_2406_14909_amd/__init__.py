"""MI355X (gfx950) Mixture-of-Attention-Spans attention: HIP kernels behind a C ABI.

The binding lives in :mod:`paper_2406_14909_amd.moa`; the library is built by
:mod:`paper_2406_14909_amd.build`.
"""
from .moa import (MOA_BAND_BLOCK, MOA_BLOCK_BAND, MOA_SPAN_INCLUDES_SINKS, MoaError, Plan,
                  load_library, moa_decode, moa_decode_ragged, moa_influence, moa_rule_loss,
                  moa_decode_workspace_bytes, moa_kv_append, moa_kv_append_ragged, moa_plan,
                  moa_paged_append, moa_paged_decode, moa_paged_decode_shared, moa_paged_prefill,
                  moa_paged_assign, moa_paged_workspace_bytes, moa_prefill, moa_quant_append,
                  moa_quant_decode, moa_quant_decode_shared, moa_quant_prefill, new_cache,
                  new_page_tables, new_paged_cache, new_paged_workspace, new_quant_cache,
                  new_workspace)

__all__ = [
    "MOA_BAND_BLOCK", "MOA_BLOCK_BAND", "MOA_SPAN_INCLUDES_SINKS", "MoaError", "Plan", "load_library", "moa_decode", "moa_decode_ragged", "moa_influence", "moa_rule_loss",
    "moa_decode_workspace_bytes", "moa_kv_append", "moa_kv_append_ragged", "moa_plan",
    "moa_paged_append", "moa_paged_decode", "moa_paged_decode_shared", "moa_paged_prefill",
    "moa_paged_workspace_bytes", "moa_prefill", "new_cache", "new_paged_cache",
    "new_paged_workspace", "new_workspace",
    "moa_paged_assign", "moa_quant_append", "moa_quant_decode", "moa_quant_decode_shared", "moa_quant_prefill",
    "new_page_tables", "new_quant_cache",
]
