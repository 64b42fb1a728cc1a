"""cfpp: MI355X-native single-token decode of GPT-NeoX / Pythia decoder blocks.

The product is the C-ABI HIP library `libcfpp.so` (see include/cfpp.h); this
package is its thin ctypes binding.  Every step of the decode path runs in the
library's kernels; PyTorch is used by callers only for device memory and streams.
"""
from .binding import (  # noqa: F401
    CfppError, Config, lib, library_path, profile_build,
    cfpp_validate_config, cfpp_packed_layer_bytes, cfpp_kv_layer_bytes, cfpp_workspace_bytes,
    cfpp_algorithmic_bytes, cfpp_pack_layer, cfpp_kv_import, cfpp_kv_export,
    cfpp_create, cfpp_destroy, cfpp_set_option, cfpp_get_option,
    cfpp_block_decode, cfpp_stack_decode, cfpp_stack_prefill, cfpp_prefill_scratch_bytes, cfpp_stack_prefill_gemm, cfpp_stack_capture, cfpp_stack_replay,
    cfpp_block_decode_static, cfpp_device_error, cfpp_debug_read, cfpp_debug_prefill_plan, cfpp_debug_prefill_narrow, cfpp_debug_prefill_beside, cfpp_debug_attention_plan, cfpp_debug_prefill_tiles, cfpp_debug_prefill_long, cfpp_debug_prefill_scratch, cfpp_debug_gelu, cfpp_stream_read, cfpp_stream_copy,
    Pages, TreeBatch, cfpp_validate_pages, cfpp_page_pool_bytes, cfpp_tree_plan_bytes, cfpp_page_tables, cfpp_tree_plan, cfpp_page_append,
    cfpp_tree_attention, cfpp_tree_accept, cfpp_tree_scratch_bytes, cfpp_stack_tree,
    cfpp_page8_pool_bytes, cfpp_page8_append, cfpp_page8_read, cfpp_page8_attention, Sampling, cfpp_sample, cfpp_lm_sample, cfpp_generate_sample_capture,
    TYPE_F16, TYPE_F32, TYPE_INT8, TYPE_E4M3,
    Lm, cfpp_lm_embed, cfpp_lm_next, cfpp_generate_capture,
    OPT_MODE, OPT_GRID, OPT_THREADS, OPT_PROFILE_SKIP, OPT_EPOCH_LIMIT, MODE_AUTO,
)
