"""MI355X-native JARQ refinement sweep.

The per-layer hot path of JARQ (joint alternating refinement of a group-wise
quantized weight matrix against a calibration Hessian) as hand-written HIP for
gfx950 behind the C ABI of include/jarq.h, with a thin ctypes binding; and the
operators that run, train and evaluate refined layers: the gated feed-forward block with its
gradients, linear layers in 8-bit integers, token log probabilities, the norm in front of a
block, log probabilities straight from hidden states, and the AdamW step.
"""

from .binding import (AdamWState, DEC_ACCEPT, DEC_REJECT, DEC_SKIP,
                      DEC_STOPPED, EXPORTED, JARQ_EHIP, JARQ_EINVAL,
                      JARQ_ENOT_SPD, JARQ_ESCALE_SOLVE, JARQ_EWORKSPACE,
                      JARQ_OK, JarqError, LIB_PATH, LinearLogprobs,
                      MAX_RECORDED_SWEEPS, Params, Stats, abi_version,
                      adamw_moments, adamw_state, adamw_step, alloc_workspace,
                      code_step, codes_i8, gated_backward, gated_forward,
                      linear_i8, linear_logprobs, linear_logprobs_backward,
                      load_library, make_params, matmul_i8, objective,
                      prepare, quant_rows_i8, refine, rms_norm,
                      rms_norm_backward, rms_norm_i8, scale_step,
                      status_string, stop_sweeps, sweeps, token_logprobs,
                      token_logprobs_backward, workspace_bytes)

__all__ = [
    "AdamWState", "DEC_ACCEPT", "DEC_REJECT", "DEC_SKIP", "DEC_STOPPED", "EXPORTED",
    "JARQ_EHIP", "JARQ_EINVAL", "JARQ_ENOT_SPD", "JARQ_ESCALE_SOLVE", "JARQ_EWORKSPACE",
    "JARQ_OK", "JarqError", "LIB_PATH", "LinearLogprobs", "MAX_RECORDED_SWEEPS", "Params",
    "Stats", "abi_version", "adamw_moments", "adamw_state", "adamw_step", "alloc_workspace",
    "code_step", "codes_i8", "gated_backward", "gated_forward", "linear_i8", "linear_logprobs",
    "linear_logprobs_backward", "load_library", "make_params", "matmul_i8", "objective",
    "prepare", "quant_rows_i8", "refine", "rms_norm", "rms_norm_backward", "rms_norm_i8",
    "scale_step", "status_string", "stop_sweeps", "sweeps", "token_logprobs",
    "token_logprobs_backward", "workspace_bytes",
]
