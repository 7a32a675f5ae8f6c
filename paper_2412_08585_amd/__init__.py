"""MI355X (gfx950) TurboAttention hot path: FlashQ + SAS quantized attention.

The computation lives in libturboattn.so (hand-written HIP for gfx950 behind
the C ABI of include/turbo_attn.h); this package only marshals arguments.
"""
from .binding import (KVTail, PagedKVCache, TurboKVCacheStruct, TurboKVTailStruct, decode_auto_split,
                      decode_split, decode_workspace, lib, page_bytes, select_workspace,
                      selected_workspace, tree_workspace, turbo_append_kv, turbo_append_path,
                      turbo_attn_decode, turbo_attn_decode_noalloc, turbo_attn_decode_trace,
                      turbo_attn_prefill, turbo_attn_prefill_q8, turbo_attn_prefill_trace,
                      turbo_attn_selected, turbo_attn_tree, turbo_head_priority, turbo_int2_heads,
                      turbo_qkv_project, turbo_quantize_kv, turbo_sas_softmax, turbo_select_groups,
                      turbo_tail_init, turbo_tree_mask)

__all__ = ["KVTail", "PagedKVCache", "TurboKVCacheStruct", "TurboKVTailStruct", "decode_auto_split",
           "decode_split", "decode_workspace", "lib", "page_bytes", "select_workspace",
           "selected_workspace", "tree_workspace", "turbo_append_kv", "turbo_append_path",
           "turbo_attn_decode", "turbo_attn_decode_noalloc", "turbo_attn_decode_trace",
           "turbo_attn_prefill", "turbo_attn_prefill_q8", "turbo_attn_prefill_trace",
           "turbo_attn_selected", "turbo_attn_tree", "turbo_head_priority", "turbo_int2_heads",
           "turbo_qkv_project", "turbo_quantize_kv", "turbo_sas_softmax", "turbo_select_groups",
           "turbo_tail_init", "turbo_tree_mask"]
