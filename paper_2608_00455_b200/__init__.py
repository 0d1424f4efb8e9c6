"""B200 delta-transfer hot path: fused AdamW-inversion / BF16-compare / compaction /
remap extract kernel, sparse apply kernel and the storage path's chunk codec behind a C ABI
(include/dte.h), and the operators at the two ends of the model whose weights it moves: embedding lookup,
layer / RMS norm and the linear head's cross entropy, with their gradients."""
from .binding import (CHUNK_REF_DTYPE, DTE_CHUNK_BYTE_PLANES, DTE_CHUNK_DELTA_PLANES, DTE_CHUNK_PLAIN, DTE_DEV_BOUNDS,
                      DTE_DEV_CORRUPT, DTE_DEV_OVERFLOW, DTE_DEV_TIMEOUT, SYMBOLS, ChunkStream, Delta,
                      DteError, HostResult, Layout, PushTarget, dte_extract_delta_push, dte_push_wait, dte_apply, dte_apply_canonical, dte_derive_constants, dte_extract_delta,
                      dte_extract_delta_groups, dte_extract_delta_host, dte_extract_delta_static,
                      dte_op_counts, dte_pack_chunks, dte_unpack_chunks, lib,
                      library_path)
from .operators import (dte_embedding_backward, dte_embedding_backward_workspace_bytes, dte_embedding_forward,
                        dte_linear_ce_backward, dte_linear_ce_backward_workspace_bytes,
                        dte_linear_ce_backward_workspace_min_bytes, dte_linear_ce_forward,
                        dte_linear_ce_forward_workspace_bytes, dte_norm_backward, dte_norm_backward_workspace_bytes,
                        dte_norm_forward)

__all__ = ["CHUNK_REF_DTYPE", "DTE_CHUNK_BYTE_PLANES", "DTE_CHUNK_DELTA_PLANES", "DTE_CHUNK_PLAIN", "DTE_DEV_BOUNDS",
           "DTE_DEV_CORRUPT", "DTE_DEV_OVERFLOW", "DTE_DEV_TIMEOUT", "SYMBOLS", "ChunkStream", "Delta",
           "DteError", "HostResult", "Layout", "PushTarget", "dte_extract_delta_push", "dte_push_wait", "dte_apply", "dte_apply_canonical", "dte_derive_constants", "dte_extract_delta",
           "dte_extract_delta_groups", "dte_extract_delta_host", "dte_extract_delta_static",
           "dte_op_counts", "dte_pack_chunks", "dte_unpack_chunks", "lib",
           "library_path",
           "dte_embedding_backward", "dte_embedding_backward_workspace_bytes", "dte_embedding_forward",
           "dte_linear_ce_backward", "dte_linear_ce_backward_workspace_bytes",
           "dte_linear_ce_backward_workspace_min_bytes", "dte_linear_ce_forward",
           "dte_linear_ce_forward_workspace_bytes", "dte_norm_backward", "dte_norm_backward_workspace_bytes",
           "dte_norm_forward"]
