// The product of two matrices in 8 bits with a scale for each block of 128 columns.  Block by block the matrix cores add up
// 128 products from zero; the sum enters the fp32 accumulator times the two scales.
//
// Two ways to the sum of a block, by the type of the result:
//   bf16  the 8-bit matrix instruction (4.1 PFLOP/s measured with independent operands).  Inside it groups of eight products
//         are aligned to the largest one's exponent and keep 13 bits below it before they enter an fp32 sum (probed with
//         single products: one that is 2^-13 of its neighbour arrives, one of 2^-14 does not; across groups all do).  On normal
//         operands that is 1.5e-5 of the result, a hundredth of the rounding to bf16 that follows.
//   fp32  the operands widened to bf16, which holds every e4m3 value, and the bf16 instruction, at half the rate: a gradient
//         that is accumulated over many steps keeps fp32's precision.
#include "fp8_common.h"
#include "fp8_internal.h"

namespace crisp {

struct ProductArgs {
    const uint8_t *x, *w;
    const float *xs, *ws;
    int64_t ldx, ldw, ldxs, ldws;
    int T, S, kb;                       // rows of X, rows of W, blocks of 128 columns
    int w_tiles;
    void* y;
    int64_t ldy, ldr;
    const float *scale, *bias;
    const void* residual;
    int relu, y_bf16;
};

// 16 x 16 outputs, 128 products each, from zero.  Lane l holds 32 columns of row l % 16 of either operand, the same ones of
// both, so that their order does not matter; output register i of lane l is (W row 4 (l / 16) + i, X row l % 16).
__device__ __forceinline__ f32x4 block_product(i32x8 w, i32x8 x) {
    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, zero, 0, 0, 0, 0, 0, 0);
}

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;

// Eight e4m3 values to bf16, exactly.
__device__ __forceinline__ bf16x8 widen(int lo, int hi) {
    float x[8];
    from_fp8x8(make_uint2((uint32_t)lo, (uint32_t)hi), x);
    bf16x8 y;
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = (__bf16)x[j];
    return y;
}

__device__ __forceinline__ f32x4 block_product_exact(i32x8 w, i32x8 x) {
    f32x4 c = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < 4; ++k)
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(w[2 * k], w[2 * k + 1]), widen(x[2 * k], x[2 * k + 1]), c, 0, 0, 0);
    return c;
}

__device__ __forceinline__ void store_y(const ProductArgs& a, int64_t t, int s, float y) {
    if (a.scale) y *= a.scale[s];
    if (a.bias) y += a.bias[s];
    if (a.y_bf16) {
        if (a.residual) y += __uint_as_float((uint32_t)static_cast<const uint16_t*>(a.residual)[t * a.ldr + s] << 16);
        if (a.relu) y = fmaxf(y, 0.0f);
        static_cast<uint16_t*>(a.y)[t * a.ldy + s] = to_bf16(y);
    } else {
        if (a.residual) y += static_cast<const float*>(a.residual)[t * a.ldr + s];
        if (a.relu) y = fmaxf(y, 0.0f);
        static_cast<float*>(a.y)[t * a.ldy + s] = y;
    }
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
    const int64_t tiles = (int64_t)((a.T + 15) / 16) * ((a.S + 15) / 16);
    auto kernel = a.y_bf16 ? fp8_product_kernel<false> : fp8_product_kernel<true>;
    kernel<<<(unsigned)((tiles + 3) / 4), 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace crisp
