"""SubZero+ hot path on AMD Instinct MI355X (gfx950).

The computation lives in libzo.so (hand-written HIP kernels behind the C ABI
of include/zo.h); this package only binds it.  Entry points:

    subspace_refresh       Haar factors of Gaussian panels (Eq. 11, Alg. 1);
                           subspace_refresh_noalloc the same for callers that cannot
                           allocate (the library's static per-GPU scratch)
    perturbed_linear       X_b (W +- eps U Z_j V^T)^T for all query blocks (Eq. 4);
                           PerturbedLinear.apply takes a fused ReLU or residual epilogue;
                           prepare_group prepares a layer's q, k, v in one pass over X
    lora_perturbed_linear  the same for a LoRA-adapted layer: both adapter factors
                           perturbed in their own subspaces
    layernorm, causal_attention, DecoderLayer
                           the network a query evaluates (the forward of Eq. 5): a
                           pre-LN decoder layer with all six matrices perturbed
    rmsnorm, rope, LlamaLayer
                           the same for a LLaMA-family layer (RMS norms, rotary
                           positions, SwiGLU MLP) with all seven matrices perturbed
    LlamaLoraLayer         the LoRA scheme's layer (grouped key/value heads, frozen
                           base, perturbed adapters on q and v)
    kv_append, paged_attention
                           answering with a tuned model: a layer's paged key/value cache
                           (16-bit, or e4m3 with a scale per page and head), appended to with
                           the rotation on the way, and the causal attention that reads it
    embedding, embedding_backward
                           a model's first step, rows of a table by token, and the table's gradient
                           by sorted tokens
    token_logprob, token_logprob_backward
                           its last: the labels' log-probabilities over the vocabulary for all query
                           blocks, and the logits' gradient
    preference_loss, policy_loss
                           losses over sequences of token log-probabilities, one per query block
                           (float64, for the estimates below), with their gradients
    subspace_adam_update   subspace Adam and W <- W - lr U S V^T (Eqs. 6-10)
    subspace_sgd_update    plain subspace SGD, W <- W - lr U Zbar V^T
    sq_loss, combine_central, combine_forward   loss and estimate helpers (central
                           difference, or forward difference against a baseline block)
"""
from ._lib import (ZO_BF16, ZO_E4M3, ZO_EPI_NONE, ZO_EPI_RELU, ZO_EPI_RESIDUAL, ZO_EPI_SILU_MUL, ZO_F16,
                   ZO_F32, ZO_MAX_BLOCKS, ZO_MAX_QR_RANK, ZO_MAX_RANK, ZO_NOALLOC_SCRATCH_BYTES, ABI_SYMBOLS,
                   LIB_PATH, DecoderLayer, LlamaLayer, LlamaLoraLayer, LoraPerturbedLinear, PerturbedLinear,
                   Workspace, ZoError, abi_version, causal_attention, combine_central, combine_forward,
                   embedding, embedding_backward, kv_append, layernorm, lib, lora_perturbed_linear,
                   paged_attention, perturbed_linear, policy_loss, preference_loss, prepare_group, rmsnorm,
                   rope, sq_loss, subspace_adam_update, subspace_refresh, subspace_refresh_noalloc,
                   subspace_sgd_update, token_logprob, token_logprob_backward)

__all__ = ["ZO_BF16", "ZO_E4M3", "ZO_EPI_NONE", "ZO_EPI_RELU", "ZO_EPI_RESIDUAL", "ZO_EPI_SILU_MUL", "ZO_F16",
           "ZO_F32", "ZO_MAX_BLOCKS", "ZO_MAX_QR_RANK", "ZO_MAX_RANK", "ZO_NOALLOC_SCRATCH_BYTES",
           "ABI_SYMBOLS", "LIB_PATH", "DecoderLayer", "LlamaLayer", "LlamaLoraLayer", "LoraPerturbedLinear",
           "PerturbedLinear", "Workspace", "ZoError", "abi_version", "causal_attention", "combine_central",
           "combine_forward", "embedding", "embedding_backward", "kv_append", "layernorm", "lib",
           "lora_perturbed_linear", "paged_attention", "perturbed_linear", "policy_loss", "preference_loss",
           "prepare_group", "rmsnorm", "rope", "sq_loss", "subspace_adam_update", "subspace_refresh",
           "subspace_refresh_noalloc", "subspace_sgd_update", "token_logprob", "token_logprob_backward"]
