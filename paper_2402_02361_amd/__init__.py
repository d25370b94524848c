"""MI355X-native hot path of Pruner's draft-then-verify schedule exploration (arXiv 2402.02361).

`binding` holds thin wrappers with the names of the C boundary (include/pruner.h):
draft_score, topk, topk_static, prior_filter, lse, random_init, moa_update, verify_score, pacm_score, and the operators of a trainable Transformer block: gated_norm, gated_norm_grad,
checkpoint_pack, checkpoint_restore, checkpoint_wgrad, rel_attention, rel_attention_grad (and the helper relative_edges); and those of a sequence read token by token: rotary, rotary_grad (rotary_frequencies), cache_append, cache_restore,
cache_attention (new_cache), weights_pack, weights_restore, weights_linear.  They only marshal arguments; every step runs in the HIP
kernels of libpruner_hip.so.  There is no CPU fallback: a missing library raises.
"""
from .binding import (  # noqa: F401
    PrunerError, draft_score, topk, topk_static, prior_filter, lse, random_init, moa_update, time_dominant_draft_launch, verify_score, pacm_score, workspace_bytes, strerror, load_library, library_path,
    NO_COMPUTE_PENALTY, NO_MEMORY_PENALTY, REFERENCE_ROUNDING, FUSED_ARITHMETIC, NSYM, SYMBOL_NAMES, WS_DRAFT, WS_TOPK, WS_VERIFY, WS_PRIOR_FILTER, WS_LSE, WS_PACM,
    CSubgraph, CMlp, CPacm, to_c_subgraphs,
    Checkpoint, checkpoint_pack, checkpoint_restore, checkpoint_wgrad, gated_norm, gated_norm_grad, relative_edges, rel_attention, rel_attention_grad,
    rotary_frequencies, rotary, rotary_grad, Cache, new_cache, cache_append, cache_restore, cache_attention, PackedWeights, weights_pack, weights_restore, weights_linear,
)
