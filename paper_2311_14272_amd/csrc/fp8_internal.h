// Launchers of the 8-bit layers (not installed).  Arguments have been checked.
#pragma once
#include <hip/hip_runtime.h>

#include "crisp_fp8.h"
#include "fp8_ways.h"

namespace crisp {

hipError_t launch_fp8_quant(const void* X, int in_type, int64_t rows, int64_t cols, int64_t ldx, const uint32_t* mask,
                            const crisp_fp8_mat* Q, const crisp_fp8_mat* Qt, hipStream_t st);
hipError_t launch_fp8_product(const crisp_fp8_mat& X, const crisp_fp8_mat& W, void* Y, int64_t ldy, int y_type,
                              const crisp_epilogue* ep, hipStream_t st);

// Both gradients of a layer: dX = G Wt^T and dW = Gt Xt^T (ep: dW's).
hipError_t launch_fp8_gradients(const crisp_fp8_mat& G, const crisp_fp8_mat& Wt, void* dX, int64_t lddx, int dx_type, const crisp_fp8_mat& Gt,
                                const crisp_fp8_mat& Xt, void* dW, int64_t lddw, int dw_type, const crisp_epilogue* ep, hipStream_t st);

// The layer from X as it is, in one launch, for sizes that fp8_takes_raw takes.
hipError_t launch_fp8_raw(const void* X, int in_type, int64_t T, int64_t ldx, const crisp_fp8_mat& W, void* Y, int64_t ldy, int y_type,
                          const crisp_epilogue* ep, hipStream_t st);

}  // namespace crisp
