"""B200 delta-transfer hot path: fused AdamW-inversion / BF16-compare / compaction /
remap extract kernel, sparse apply kernel and the storage path's chunk codec behind a C ABI
(include/dte.h), and operators of the training step whose weights it moves: embedding lookup, layer / RMS norm, rotary
positions, causal attention over packed sequences and the linear head's cross entropy, with their gradients, and the
global gradient norm with clipping."""
from .binding import (CHUNK_REF_DTYPE, DTE_CHUNK_BYTE_PLANES, DTE_CHUNK_DELTA_PLANES, DTE_CHUNK_PLAIN, DTE_DEV_BOUNDS,
                      DTE_DEV_CORRUPT, DTE_DEV_OVERFLOW, DTE_DEV_TIMEOUT, SYMBOLS, ChunkStream, Delta,
                      DteError, HostResult, Layout, PushTarget, dte_extract_delta_push, dte_push_wait, dte_apply, dte_apply_canonical, dte_derive_constants, dte_extract_delta,
                      dte_extract_delta_groups, dte_extract_delta_host, dte_extract_delta_static,
                      dte_op_counts, dte_pack_chunks, dte_unpack_chunks, lib,
                      library_path)
from .operators import (DTE_ROPE_BASE, DTE_ROPE_LINEAR, DTE_ROPE_PLAIN, DTE_ROPE_RAMP, dte_attention_backward,
                        dte_attention_backward_workspace_bytes, dte_attention_forward, dte_attention_plan, dte_attention_plan_bytes,
                        dte_embedding_backward, dte_embedding_backward_workspace_bytes, dte_embedding_forward,
                        dte_grad_clip, dte_grad_sum_squares, dte_grad_sum_squares_workspace_bytes,
                        dte_linear_ce_backward, dte_linear_ce_backward_workspace_bytes,
                        dte_linear_ce_backward_workspace_min_bytes, dte_linear_ce_forward,
                        dte_linear_ce_forward_workspace_bytes, dte_norm_backward, dte_norm_backward_workspace_bytes,
                        dte_norm_forward, dte_rope, dte_rope_frequencies)

__all__ = ["CHUNK_REF_DTYPE", "DTE_CHUNK_BYTE_PLANES", "DTE_CHUNK_DELTA_PLANES", "DTE_CHUNK_PLAIN", "DTE_DEV_BOUNDS",
           "DTE_DEV_CORRUPT", "DTE_DEV_OVERFLOW", "DTE_DEV_TIMEOUT", "SYMBOLS", "ChunkStream", "Delta",
           "DteError", "HostResult", "Layout", "PushTarget", "dte_extract_delta_push", "dte_push_wait", "dte_apply", "dte_apply_canonical", "dte_derive_constants", "dte_extract_delta",
           "dte_extract_delta_groups", "dte_extract_delta_host", "dte_extract_delta_static",
           "dte_op_counts", "dte_pack_chunks", "dte_unpack_chunks", "lib",
           "library_path",
           "DTE_ROPE_BASE", "DTE_ROPE_LINEAR", "DTE_ROPE_PLAIN", "DTE_ROPE_RAMP", "dte_attention_backward",
           "dte_attention_backward_workspace_bytes", "dte_attention_forward", "dte_attention_plan", "dte_attention_plan_bytes",
           "dte_grad_clip", "dte_grad_sum_squares", "dte_grad_sum_squares_workspace_bytes", "dte_rope", "dte_rope_frequencies",
           "dte_embedding_backward", "dte_embedding_backward_workspace_bytes", "dte_embedding_forward",
           "dte_linear_ce_backward", "dte_linear_ce_backward_workspace_bytes",
           "dte_linear_ce_backward_workspace_min_bytes", "dte_linear_ce_forward",
           "dte_linear_ce_forward_workspace_bytes", "dte_norm_backward", "dte_norm_backward_workspace_bytes",
           "dte_norm_forward"]
