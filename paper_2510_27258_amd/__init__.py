"""MI355X-native Higher-order Linear Attention (arXiv 2510.27258).

The computation lives in libhla.so (HIP for gfx950, C ABI in include/hla.h).
`capi` mirrors the C entry points one to one; `hla` wraps them for torch
tensors (torch provides device memory and the current stream only).
"""
from . import capi  # noqa: F401
from .block import (GatedLinearRecurrence, GatedNorm, GatedProjections, ResidualNorm, gated_norm,  # noqa: F401
                    gated_norm_backward, gated_norm_forward, glr_backward, glr_forward, glr_prefill, glr_scan,
                    glr_step, glu, glu_backward, glu_forward, residual_norm, residual_norm_backward,
                    residual_norm_forward)
from .hla import (HLA2, State, ahla_forward, backward, chunk_summaries, forward, forward_decay,  # noqa: F401
                  hla2_attention, hla3_forward, prefill, scan, split_state, state_floats, step, workspace_bytes)
from .mixer import (QKNormRope, ShortConv, SSMScan, conv_backward, conv_forward, conv_prefill,  # noqa: F401
                    conv_step, qk_norm_rope, qk_norm_rope_backward, qk_norm_rope_forward, short_conv, ssm_backward,
                    ssm_forward, ssm_prefill, ssm_scan, ssm_step)
