"""SMAT's per-step Scale/Mask/Perturb parameter transform on MI355X (gfx950).

`libsmat.so` (C ABI in include/smat.h) holds the HIP kernels; this package binds it with
ctypes.  Build it with `python -m paper_2609_33437_amd.build`.
"""
from ._lib import (EXPORTS, OP_PARAMS_DTYPE, SMAT_BF16, SMAT_EXPERT, SMAT_F32, SMAT_NOISE_GAUSSIAN,
                   SMAT_NOISE_LAPLACE, SMAT_NOISE_UNIFORM, SMAT_SIMULATED, AdamStepState, MergePlan, Plan, SmatError,
                   StepState, adamw_params, lib, load_library, merge_term, op_params, op_params_array, rng_key,
                   scale_draw, smat_adamw_fused, smat_backward_accum, smat_debug_draws, smat_merge, smat_simulate,
                   smat_stream_copy)
from ._linear import (SMAT_ACT_GELU, SMAT_ACT_GELU_TANH, SMAT_ACT_NONE, SMAT_ACT_SILU, ActCheckpoint, smat_ckpt_read,
                      smat_ckpt_write, smat_linear, smat_linear_dgrad, smat_linear_wgrad)
from ._decoder import (SMAT_NORM_LAYER, SMAT_NORM_RMS, smat_embed, smat_embed_grad, smat_linear_xent,
                       smat_linear_xent_grad, smat_norm, smat_norm_grad)

__all__ = ["SMAT_ACT_GELU", "SMAT_ACT_GELU_TANH", "SMAT_ACT_NONE", "SMAT_ACT_SILU", "ActCheckpoint", "smat_ckpt_read",
           "smat_ckpt_write", "smat_linear", "smat_linear_dgrad", "smat_linear_wgrad",
           "SMAT_NORM_LAYER", "SMAT_NORM_RMS", "smat_embed", "smat_embed_grad", "smat_linear_xent",
           "smat_linear_xent_grad", "smat_norm", "smat_norm_grad",
           "EXPORTS", "OP_PARAMS_DTYPE", "op_params_array", "SMAT_BF16", "SMAT_EXPERT", "SMAT_F32", "SMAT_NOISE_GAUSSIAN", "SMAT_NOISE_LAPLACE", "SMAT_NOISE_UNIFORM",
           "SMAT_SIMULATED", "MergePlan", "Plan", "SmatError", "StepState", "AdamStepState", "adamw_params", "lib", "load_library", "merge_term",
           "op_params", "rng_key", "scale_draw", "smat_adamw_fused", "smat_backward_accum", "smat_debug_draws", "smat_merge",
           "smat_simulate", "smat_stream_copy"]
