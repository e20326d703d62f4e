"""MI355X-native mask-only logits for diffusion-LLM denoising steps (Mosaic, arXiv 2601.06562).

The product is the HIP library behind ``include/mosaic.h``, for the layer work on either side of the
logits ``include/mosaic_layer.h``, and for both ends of the model, tokens into rows and rows back onto
given tokens, ``include/mosaic_tokens.h``; ``binding`` marshals torch device tensors to it,
``workloads`` draws the seeded synthetic inputs, ``build`` compiles the library.
"""
from . import binding, workloads  # noqa: F401
from .binding import (MaskOnlyLogits, MosaicError, MosaicPlan, Q8Rows, mosaic_checkpoint_load,  # noqa: F401
                      mosaic_checkpoint_store, mosaic_compact_scratch_bytes, mosaic_dropout_backward,
                      mosaic_dropout_forward, mosaic_embedding_backward, mosaic_embedding_backward_workspace_bytes,
                      mosaic_embedding_forward, mosaic_gated_ffn_backward, mosaic_gated_ffn_backward_workspace_bytes,
                      mosaic_gated_ffn_forward, mosaic_mask_compact, mosaic_masked_logits_reduce,
                      mosaic_masked_logits_sample, mosaic_masked_logprobs, mosaic_masked_logprobs_backward,
                      mosaic_masked_logprobs_backward_workspace_bytes, mosaic_masked_logprobs_workspace_bytes,
                      mosaic_plan_workspace, mosaic_rmsnorm_backward, mosaic_rmsnorm_backward_workspace_bytes,
                      mosaic_rmsnorm_forward, mosaic_sample_workspace_bytes,
                      mosaic_shift_indices, mosaic_unmask_topn)
