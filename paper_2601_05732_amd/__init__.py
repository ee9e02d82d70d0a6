"""mHC-lite hyper-connection hot path for AMD MI355X (gfx950).

The work is done by ``libmhcl.so`` (hand-written HIP, C ABI in
``include/mhcl.h``); :mod:`paper_2601_05732_amd.binding` only marshals torch
tensors into its arguments.  There is no CPU or eager fallback: if the
library is missing, loading it raises.
"""
from .binding import (  # noqa: F401
    BF16, F32, RES_LITE, RES_SK, RES_SUBSET, OP_COEFFS, OP_COEFFS_BWD, OP_FWD_COEFFS_PRE, OP_BWD_FUSED, OP_COEFFS_LAYERS,
    MhclError, Desc, lib, lib_path, exported_symbols, logit_count, workspace_bytes, perm_table,
    mhcl_coeffs, mhcl_pre, mhcl_post, mhcl_fwd_coeffs_pre, mhcl_post_bwd, mhcl_pre_bwd,
    mhcl_coeffs_bwd, mhcl_bwd_fused, mhcl_logits, mhcl_coeffs_logits, mhcl_coeffs_logits_layers, mhcl_ds_chain, mhcl_fwd_coeffs_pre_static,
    STATIC_SCRATCH_BYTES,
    I64, I32, OP_EMBED_BWD, OP_STREAMS_NORM_BWD, OP_HEAD_LOSS, OP_HEAD_LOSS_GRAD, EndsDesc, ends_workspace_bytes,
    mhcl_embed, mhcl_embed_bwd, mhcl_streams_norm, mhcl_streams_norm_bwd, mhcl_head_loss, mhcl_head_loss_grad,
    mhcl_head_total, mhcl_scale, mhcl_scale_to,
    mhcl_head_distill, head_distill_workspace_bytes, mhcl_head_preference, head_preference_workspace_bytes,
    OP_FFN, OP_FFN_GRAD, FfnDesc, ffn_workspace_bytes, mhcl_ffn, mhcl_ffn_grad, mhcl_ffn_grad_of,
)
from .layer import GpuLayer, desc_for, empty_stream, place_stream  # noqa: F401,E402
from .autograd import HyperConnection, HyperConnectionStack, init_params  # noqa: F401,E402
from .ends import (  # noqa: F401,E402
    embed_tokens, embed_tokens_grad, streams_norm, streams_norm_grad, head_loss, head_loss_grad,
    head_distill, head_distill_grad, head_preference, head_preference_grad,
    TokenEmbedding, StreamsNorm, Head,
)
from .ffn import gated_ffn, gated_ffn_grad, GatedFeedForward  # noqa: F401,E402


def __getattr__(name):
    if name == "LanguageModel":     # imported when it is asked for: the module is also run by itself (python -m)
        from .lm import LanguageModel
        return LanguageModel
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
