"""K-Forcing batched joint next-k-token decode on MI355X (gfx950).

The compute path lives in libkforcing.so (hand-written HIP kernels behind the
C ABI of include/kforcing.h).  This package is its thin Python binding:
argument marshalling only.  PyTorch supplies device memory and the stream.
"""
from .binding import (  # noqa: F401
    GradClip, KF_BF16, KF_EHIP, KF_ECTX, KF_EINVAL, KF_ENOMEM, KF_ESTATE, KF_FLAG_DEBUG_LOGITS, KF_FP16, KF_FP32,
    KF_KC_NAMES, KF_MASK_DOUBLE, KF_MASK_SINGLE, KF_OK, KfConfig, KfError, KForcing, lib,
    PolicyLoss, dropout, dropout_backward, dropout_norm, dropout_norm_backward, policy_loss, qkv_heads,
    qkv_heads_backward, rope_table, TokenLogprobs, layer_norm, layer_norm_backward, lib_path, token_logprobs,
    token_logprobs_backward, training_attention, training_attention_backward,
    training_attention_lse, training_attention_shapes,
)
