// Quantisation to e4m3 with one scale for each block of 128 columns of a row, or of 128 x 128 elements: read once, largest
// magnitude per block, multiply by the scale's inverse, round, write one or both directions.  Bound by memory.
#include "fp8_common.h"
#include "fp8_internal.h"

namespace crisp {

// ROWS, one direction, no mask: 16 lanes take a block of 128 columns, a workgroup 16 consecutive blocks of the matrix in
// row order.
template <bool BF16>
__global__ __launch_bounds__(256) void fp8_rows_kernel(const void* __restrict__ X, int64_t rows, int cols, int64_t ldx, bool vec,
                                                       uint8_t* __restrict__ q, int64_t ld, float* __restrict__ scale, int64_t lds) {
    const int kb = (cols + FP8_BLOCK - 1) / FP8_BLOCK;
    const int64_t id = (int64_t)blockIdx.x * 16 + threadIdx.x / 16;
    const int64_t r = id / kb;
    const int b = (int)(id - r * kb), lane = threadIdx.x % 16;
    if (r >= rows) return;      // all 16 lanes of a group leave together
    const int c = b * FP8_BLOCK + lane * 8;
    float x[8], s;
    load8<BF16>(X, r * ldx + c, cols - c, vec, x);
    *reinterpret_cast<uint2*>(q + r * ld + c) = quantize_block(x, s);
    if (lane == 0) scale[b * lds + r] = s;
}

// A 128 x 128 tile per workgroup, for everything else.  Thread (g, l): rows 8g .. 8g+7, columns 8l .. 8l+7, held in registers:
// 16 bytes a load of bf16 (with four columns and twice the threads, 24 waves a CU instead of 12, 8192 x 4096 bf16 in both
// directions took 38.8 us against 35.2).  Largest magnitudes meet in LDS, where one thread each makes the scale of a row or
// column.  The transpose is eight bytes per column and thread, gathered in LDS so that it leaves in whole rows.
template <bool BF16>
__global__ __launch_bounds__(256) void fp8_tile_kernel(const void* __restrict__ X, int64_t rows, int64_t cols, int64_t ldx, bool vec,
                                                       const uint32_t* __restrict__ mask, int kind, int tiles_c,
                                                       uint8_t* __restrict__ q, int64_t ld, float* __restrict__ scale, int64_t lds,
                                                       uint8_t* __restrict__ qt, int64_t ldt, float* __restrict__ scale_t,
                                                       int64_t ldst) {
    __shared__ uint32_t row_top[FP8_BLOCK], col_top[4][FP8_BLOCK];
    __shared__ float row_inv[FP8_BLOCK], col_inv[FP8_BLOCK];
    constexpr int PITCH = FP8_BLOCK + 8;
    __shared__ __align__(16) uint8_t turned[FP8_BLOCK * PITCH];
    const int64_t tr = blockIdx.x / tiles_c, tc = blockIdx.x % tiles_c;
    const int tid = threadIdx.x, l = tid % 16, g = tid / 16, wave = tid / 64, lane = tid % 64;
    const int64_t c = tc * FP8_BLOCK + l * 8, r0 = tr * FP8_BLOCK + g * 8;
    float x[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) load8<BF16>(X, (r0 + i) * ldx + c, r0 + i < rows ? cols - c : 0, vec, x[i]);
    if (mask) {
        const int64_t words = (cols + 31) / 32;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t bits = r0 + i < rows && c < cols ? mask[(r0 + i) * words + c / 32] >> (c % 32) : 0u;
#pragma unroll
            for (int j = 0; j < 8; ++j) x[i][j] = (bits >> j) & 1u ? x[i][j] : 0.0f;
        }
    }
    const bool tiles = kind == CRISP_FP8_TILES;
    uint32_t top[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        uint32_t t = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t b = abs_bits(x[i][j]);
            t = umax(t, b);
            top[j] = umax(top[j], b);
        }
        t = max16(t);
        if (l == i) row_top[g * 8 + i] = t;
    }
    if (!tiles && qt) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            top[j] = umax(top[j], (uint32_t)__shfl_xor((int)top[j], 16));
            top[j] = umax(top[j], (uint32_t)__shfl_xor((int)top[j], 32));
            if (lane < 16) col_top[wave][l * 8 + j] = top[j];
        }
    }
    __syncthreads();
    if (tiles) {
        uint32_t t = max16(umax(row_top[lane], row_top[lane + 64]));
        t = umax(t, (uint32_t)__shfl_xor((int)t, 16));
        t = umax(t, (uint32_t)__shfl_xor((int)t, 32));
        const float s = fp8_scale(__uint_as_float(t)), inv = 1.0f / s;
        if (tid == 0) {
            if (q) scale[tr * lds + tc] = s;
            if (qt) scale_t[tc * ldst + tr] = s;
        }
        if (tid < FP8_BLOCK) row_inv[tid] = col_inv[tid] = inv;
    } else if (tid < FP8_BLOCK) {
        if (q) {
            const float s = fp8_scale(__uint_as_float(row_top[tid]));
            row_inv[tid] = 1.0f / s;
            if (tr * FP8_BLOCK + tid < rows) scale[tc * lds + tr * FP8_BLOCK + tid] = s;
        }
    } else if (qt) {
        const int k = tid - FP8_BLOCK;
        const uint32_t t = umax(umax(col_top[0][k], col_top[1][k]), umax(col_top[2][k], col_top[3][k]));
        const float s = fp8_scale(__uint_as_float(t));
        col_inv[k] = 1.0f / s;
        if (tc * FP8_BLOCK + k < cols) scale_t[tr * ldst + tc * FP8_BLOCK + k] = s;
    }
    __syncthreads();
    if (q) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float inv = row_inv[g * 8 + i];
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = x[i][j] * inv;
            if (r0 + i < rows) *reinterpret_cast<uint2*>(q + (r0 + i) * ld + c) = to_fp8x8(y);
        }
    }
    if (!qt) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float inv = col_inv[l * 8 + j];
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[i][j] * inv;
        *reinterpret_cast<uint2*>(turned + (l * 8 + j) * PITCH + g * 8) = to_fp8x8(y);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int row = tid / 8 + 32 * k;
        const uint8_t* from = turned + row * PITCH + tid % 8 * 16;
        const uint2 a = *reinterpret_cast<const uint2*>(from), b = *reinterpret_cast<const uint2*>(from + 8);
        if (tc * FP8_BLOCK + row < cols)
            *reinterpret_cast<uint4*>(qt + (tc * FP8_BLOCK + row) * ldt + tr * FP8_BLOCK + tid % 8 * 16) = make_uint4(a.x, a.y, b.x, b.y);
    }
}

hipError_t launch_fp8_quant(const void* X, int in_type, int64_t rows, int64_t cols, int64_t ldx, const uint32_t* mask,
                            const crisp_fp8_mat* Q, const crisp_fp8_mat* Qt, hipStream_t st) {
    const bool bf16 = in_type == CRISP_IN_BF16;
    const bool vec = fp8_whole_vectors(X, in_type, ldx);
    const int64_t rb = (rows + FP8_BLOCK - 1) / FP8_BLOCK, cb = (cols + FP8_BLOCK - 1) / FP8_BLOCK;
    const int kind = Q ? Q->kind : Qt->kind;
    if (kind == CRISP_FP8_ROWS && !Qt && !mask) {
        const unsigned grid = (unsigned)((rows * cb + 15) / 16);
        if (bf16) fp8_rows_kernel<true><<<grid, 256, 0, st>>>(X, rows, (int)cols, ldx, vec, Q->q, Q->ld, Q->scale, Q->lds);
        else fp8_rows_kernel<false><<<grid, 256, 0, st>>>(X, rows, (int)cols, ldx, vec, Q->q, Q->ld, Q->scale, Q->lds);
        return hipGetLastError();
    }
    const crisp_fp8_mat none = {};
    const crisp_fp8_mat &a = Q ? *Q : none, &b = Qt ? *Qt : none;
    const unsigned grid = (unsigned)(rb * cb);
    auto kernel = bf16 ? fp8_tile_kernel<true> : fp8_tile_kernel<false>;
    kernel<<<grid, 256, 0, st>>>(X, rows, cols, ldx, vec, mask, kind, (int)cb, a.q, a.ld, a.scale, a.lds, b.q, b.ld, b.scale, b.lds);
    return hipGetLastError();
}

}  // namespace crisp
