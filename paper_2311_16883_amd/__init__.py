"""Structured activation pruning hot path for AMD MI355X (gfx950).

Forward side: block l2 scoring, exact top-k block selection, Block Sparse Row
packing.  Backward side: weight gradient dW = Xhat^T dY straight from the BSR
tensor.  Token operators (``include/bsr_token_step.h``): the token table, the sort by
expert and the distillation loss of a token model, with their gradients.  Layer operators (``include/bsr_layer_ops.h``): layer norm and
the gated feed-forward block with their gradients, AdamW over many tensors.  All compute lives in ``libbsr_actprune.so`` (hand-written HIP); this
package is the thin ctypes binding (``binding``), the in-tree build (``build``)
and the seeded synthetic workloads (``synth``).
"""
from .binding import (  # noqa: F401
    BSR_BF16, BSR_F32, BSR_OP_COMPRESS, BSR_OP_DECOMPRESS, BSR_OP_SCORE_SELECT,
    BSR_OP_T_DENSE_MATMUL, BsrError, bsr_compress, bsr_decompress, bsr_keep_count,
    bsr_score_select, bsr_storage_bytes, bsr_t_dense_matmul, bsr_version, bsr_workspace_bytes,
    bsr_distill_grad, bsr_distill_loss, bsr_distill_loss_grad, bsr_embedding_grad, bsr_embedding_lookup,
    bsr_expert_capacity, bsr_expert_combine, bsr_expert_combine_grad, bsr_expert_gather, bsr_expert_sort,
    AdamWBatch, bsr_adamw_batched, bsr_adamw_blocks, bsr_adamw_state_values, bsr_gated_ff, bsr_gated_ff_grad, bsr_layer_norm,
    bsr_layer_norm_grad,
)
