"""FlipFlop Hessian estimation on AMD MI355X (gfx950).

Estimates the Kronecker-factored Hessian A (x) B of a linear layer from
gradient samples G_i with the flip-flop iteration (WaterKron and FlipFlop
Hessian, Section 5), and quantises its weights with WaterKron (two-sided
GPTQ with waterfilling scales, Section 3), entirely in the HIP library
``libff.so`` whose C ABI is ``include/ff.h``.  Around the layer are its
operators (layer.py): the norm, the layer in bf16 or from the quantiser's codes, their
gradients, the orthogonalisation of an update.  This package is the thin
binding (ctypes + torch memory).
"""
from .binding import (FF_APPLY, FF_APPLY_INV, FF_BF16, FF_ERR_HIP, FF_ERR_INVALID_ARG,
                      FF_ERR_NOT_SPD, FF_ERR_STATE, FF_ERR_WORKSPACE, FF_F32, FF_OK,
                      FF_ORDER_A_FIRST, FF_ORDER_B_FIRST, FF_SAMPLES_DENSE, FF_SAMPLES_RANK1,
                      FF_SCALES_GIVEN, FF_SCALES_WATERFILL, FF_EST_FLIPFLOP, FF_EST_FROBENIUS,
                      FF_EST_MARGINAL, FF_EST_INPUT, ESTIMATORS, FlipFlop, FlipFlopError, ff_config,
                      ff_destroy, ff_factors, ff_fit_noalloc, ff_half_step, ff_init, ff_iterate,
                      ff_iterate_tol, ff_kernel_timing, FF_HALF_A, FF_HALF_B, FF_NOALLOC_SCRATCH_BYTES,
                      ff_kron_apply, ff_last_error, ff_objective, ff_quantize,
                      ff_quantize_workspace_size, ff_set_timing, ff_status_string,
                      ff_whiten_split_state,
                      ff_workspace_size, header_functions, load_library, LIB_PATH)

# The layer operators are torch functions: imported with the first use of one,
# so that the rest of the package does not need torch to be imported.
_LAYER = ("ACTIVATIONS", "ff_linear_args", "ff_linear_grad_args", "ff_norm_args", "ff_norm_grad_args",
          "ff_ortho_args", "linear", "linear_backward", "linear_q8", "orthogonalize", "quantize_rows",
          "rms_norm", "rms_norm_backward", "rms_norm_q8")


def __getattr__(name):
    if name not in _LAYER:
        raise AttributeError(f"module {__name__!r} has no attribute {name!r}")
    from . import layer
    globals().update({n: getattr(layer, n) for n in _LAYER})
    return globals()[name]


__all__ = [n for n in dir() if not n.startswith("_")] + list(_LAYER)
