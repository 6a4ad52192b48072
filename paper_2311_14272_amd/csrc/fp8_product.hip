// The 8-bit product's launcher, and its kernel for sizes that the others do not take.
#include "fp8_product.h"

namespace crisp {

// 16 x 16 outputs, 128 products each, from zero.  Lane l holds 32 columns of row l % 16 of either operand, the same ones of
// both, so that their order does not matter; output register i of lane l is (W row 4 (l / 16) + i, X row l % 16).
__device__ __forceinline__ f32x4 block_product(i32x8 w, i32x8 x) {
    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, zero, 0, 0, 0, 0, 0, 0);
}

__device__ __forceinline__ f32x4 block_product_exact(i32x8 w, i32x8 x) {
    f32x4 c = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < 4; ++k)
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(w[2 * k], w[2 * k + 1]), widen(x[2 * k], x[2 * k + 1]), c, 0, 0, 0);
    return c;
}

// A wave computes 16 W rows x 16 X rows straight from memory.
template <bool EXACT>
__global__ __launch_bounds__(256) void fp8_product_kernel(ProductArgs a) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int n16 = (a.S + 15) / 16;
    const int64_t tile = (int64_t)blockIdx.x * 4 + wave;
    const int t0 = (int)(tile / n16) * 16, s0 = (int)(tile % n16) * 16;
    if (t0 >= a.T) return;
    const int i = lane % 16, h = lane / 16;
    const int t = min(t0 + i, a.T - 1), s = min(s0 + i, a.S - 1);      // rows behind the last one repeat it and are not stored
    const uint8_t* x = a.x + t * a.ldx + h * 32;
    const uint8_t* w = a.w + s * a.ldw + h * 32;
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int b = 0; b < a.kb; ++b) {
        i32x8 wv, xv;
        const i32x4 w0 = *reinterpret_cast<const i32x4*>(w + b * 128), w1 = *reinterpret_cast<const i32x4*>(w + b * 128 + 16);
        const i32x4 x0 = *reinterpret_cast<const i32x4*>(x + b * 128), x1 = *reinterpret_cast<const i32x4*>(x + b * 128 + 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) { wv[j] = w0[j]; wv[4 + j] = w1[j]; xv[j] = x0[j]; xv[4 + j] = x1[j]; }
        const f32x4 p = EXACT ? block_product_exact(wv, xv) : block_product(wv, xv);
        const float xs = a.xs[b * a.ldxs + t];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int row = min(s0 + 4 * h + j, a.S - 1);
            const float ws = a.w_tiles ? a.ws[row / 128 * a.ldws + b] : a.ws[b * a.ldws + row];
            sum[j] += p[j] * (xs * ws);
        }
    }
    if (t0 + i >= a.T) return;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (s0 + 4 * h + j < a.S) store_y(a, t0 + i, s0 + 4 * h + j, sum[j]);
}

hipError_t launch_fp8_product(const crisp_fp8_mat& X, const crisp_fp8_mat& W, void* Y, int64_t ldy, int y_type,
                              const crisp_epilogue* ep, hipStream_t st) {
    ProductArgs a = {};
    a.x = X.q; a.w = W.q; a.xs = X.scale; a.ws = W.scale;
    a.ldx = X.ld; a.ldw = W.ld; a.ldxs = X.lds; a.ldws = W.lds;
    a.T = (int)X.rows; a.S = (int)W.rows; a.kb = (int)((X.cols + FP8_BLOCK - 1) / FP8_BLOCK);
    a.w_tiles = W.kind == CRISP_FP8_TILES;
    a.y = Y; a.ldy = ldy; a.y_bf16 = y_type == CRISP_Y_BF16;
    if (ep) { a.scale = ep->scale; a.bias = ep->bias; a.residual = ep->residual; a.ldr = ep->ldr; a.relu = ep->relu; }
    // (the tiled kernel's offsets inside a tile are 32 bits)
    if (a.T > 64 && a.S > 64 && a.ldx < 1 << 24 && a.ldw < 1 << 24) return launch_fp8_tiled(a, st);
    const int64_t tiles = (int64_t)((a.T + 15) / 16) * ((a.S + 15) / 16);
    auto kernel = a.y_bf16 ? fp8_product_kernel<false> : fp8_product_kernel<true>;
    kernel<<<(unsigned)((tiles + 3) / 4), 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace crisp
