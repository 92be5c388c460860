"""MI355X-native budgeted-KV decode + evict path (ForesightKV generation loop).

`binding` exposes the C ABI of libfk.so (fk_append, fk_decode_attn, fk_score_kv,
fk_select_keep, fk_compact); `build` compiles it in-tree with hipcc for gfx950.
"""
from .binding import (CacheDesc, FkError, fk_append, fk_compact, fk_decode_attn, fk_decode_attn_workspace,  # noqa: F401
                      fk_decode_step, fk_decode_window, fk_decode_step_static, new_attn_workspace, fk_decode_step_feat, fk_decode_window_feat, fk_score_kv_feat, fk_compact_feat,
                      feat_heads, new_feat, new_feat_workspace, fk_golden_steps, fk_golden_scores, fk_golden_trace,
                      PagedDesc, fk_paged_append, fk_paged_attn_workspace, new_paged_attn_workspace, fk_paged_attn, fk_paged_weights_workspace,
                      new_paged_weights_workspace, fk_paged_weights, fk_paged_compress, new_acc, fk_decode_step_acc_workspace, new_acc_workspace,
                      fk_decode_step_acc, fk_compact_acc, RopeDesc, rope_frequencies, fk_rope, fk_tree_attn_workspace, new_tree_attn_workspace, fk_tree_attn,
                      fk_paged_tree_attn_workspace, new_paged_tree_attn_workspace, fk_paged_tree_attn, fk_verify_drafts_workspace, new_verify_workspace,
                      fk_verify_drafts, fk_commit_drafts, fk_paged_commit_drafts,
                      fk_score_kv, fk_select_keep, fk_select_keep_workspace, fk_select_keep_ws, fk_select_keep_sampled, fk_stream_read, lib, prepare, status_string, version)
