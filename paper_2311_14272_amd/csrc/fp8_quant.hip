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

// C elements of a row from column c on; what lies at or behind `cols` counts as zero.  vec: as in load8.
template <bool BF16, int C>
__device__ __forceinline__ void load_some(const void* X, int64_t at, int64_t left, bool vec, float (&x)[C]) {
    if constexpr (C == 8) {
        load8<BF16>(X, at, left, vec, x);
    } else {
        typedef uint32_t words __attribute__((ext_vector_type(BF16 ? C / 2 : C)));
        if (vec && left >= C) {
            if constexpr (BF16) {
                const words v = *reinterpret_cast<const words*>(static_cast<const uint16_t*>(X) + at);
#pragma unroll
                for (int j = 0; j < C / 2; ++j) { x[2 * j] = __uint_as_float(v[j] << 16); x[2 * j + 1] = __uint_as_float(v[j] & 0xffff0000u); }
            } else {
                const words v = *reinterpret_cast<const words*>(static_cast<const float*>(X) + at);
#pragma unroll
                for (int j = 0; j < C; ++j) x[j] = __uint_as_float(v[j]);
            }
            return;
        }
#pragma unroll
        for (int j = 0; j < C; ++j) {
            x[j] = 0.0f;
            if (j < left) {
                if constexpr (BF16) x[j] = __uint_as_float((uint32_t)static_cast<const uint16_t*>(X)[at + j] << 16);
                else x[j] = static_cast<const float*>(X)[at + j];
            }
        }
    }
}

// A 128 x 128 tile per workgroup, for everything else.  Thread (g, l): rows 8g .. 8g+7, columns Cl .. Cl+C-1, held in registers.
// Largest magnitudes meet in LDS, where one thread each makes the scale of a row or column.  The transpose is eight bytes per
// column and thread, gathered in LDS so that it leaves in whole rows.
// C = 8 reads 16 bytes of bf16 at a time: 8192 x 4096 in both directions 33.0 us, with C = 4 34.8.  C = 4 has the shorter way from a
// tile's first load to its last store, the time where CUs have a tile or two: 500 x 512 5.4 us against 7.4, 2048 x 2048 6.6
// against 7.4 (C = 2: 5.4 and 6.9).
template <bool BF16, int C>
__global__ __launch_bounds__(2048 / C) void fp8_tile_kernel(const void* __restrict__ X, int64_t rows, int64_t cols, int64_t ldx, bool vec,
                                                            const uint32_t* __restrict__ mask, int kind, int tiles_c,
                                                            uint8_t* __restrict__ q, int64_t ld, float* __restrict__ scale, int64_t lds,
                                                            uint8_t* __restrict__ qt, int64_t ldt, float* __restrict__ scale_t,
                                                            int64_t ldst) {
    constexpr int L = FP8_BLOCK / C, THREADS = 16 * L, WAVES = THREADS / 64;
    __shared__ uint32_t row_top[FP8_BLOCK], col_top[WAVES][FP8_BLOCK];
    __shared__ float row_inv[FP8_BLOCK], col_inv[FP8_BLOCK];
    constexpr int PITCH = FP8_BLOCK + 8;
    __shared__ __align__(16) uint8_t turned[FP8_BLOCK * PITCH];
    const int64_t tr = blockIdx.x / tiles_c, tc = blockIdx.x % tiles_c;
    const int tid = threadIdx.x, l = tid % L, g = tid / L, wave = tid / 64, lane = tid % 64;
    const int64_t c = tc * FP8_BLOCK + l * C, r0 = tr * FP8_BLOCK + g * 8;
    float x[8][C];
#pragma unroll
    for (int i = 0; i < 8; ++i) load_some<BF16, C>(X, (r0 + i) * ldx + c, r0 + i < rows ? cols - c : 0, vec, x[i]);
    if (mask) {
        const int64_t words = (cols + 31) / 32;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t bits = r0 + i < rows && c < cols ? mask[(r0 + i) * words + c / 32] >> (c % 32) : 0u;
#pragma unroll
            for (int j = 0; j < C; ++j) x[i][j] = (bits >> j) & 1u ? x[i][j] : 0.0f;
        }
    }
    const bool tiles = kind == CRISP_FP8_TILES;
    uint32_t top[C];
#pragma unroll
    for (int j = 0; j < C; ++j) top[j] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        uint32_t t = 0;
#pragma unroll
        for (int j = 0; j < C; ++j) {
            const uint32_t b = abs_bits(x[i][j]);
            t = umax(t, b);
            top[j] = umax(top[j], b);
        }
        t = max16(t);
        if constexpr (L > 16) t = umax(t, (uint32_t)__shfl_xor((int)t, 16));
        if (l == i) row_top[g * 8 + i] = t;
    }
    if (!tiles && qt) {
#pragma unroll
        for (int j = 0; j < C; ++j) {
            if constexpr (L < 32) top[j] = umax(top[j], (uint32_t)__shfl_xor((int)top[j], 16));
            top[j] = umax(top[j], (uint32_t)__shfl_xor((int)top[j], 32));
            if (lane < L) col_top[wave][l * C + j] = top[j];
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
    } else if (tid < 2 * FP8_BLOCK && qt) {
        const int k = tid - FP8_BLOCK;
        uint32_t t = 0;
#pragma unroll
        for (int v = 0; v < WAVES; ++v) t = umax(t, col_top[v][k]);
        const float s = fp8_scale(__uint_as_float(t));
        col_inv[k] = 1.0f / s;
        if (tc * FP8_BLOCK + k < cols) scale_t[tr * ldst + tc * FP8_BLOCK + k] = s;
    }
    __syncthreads();
    if (q) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float inv = row_inv[g * 8 + i];
            float y[C];
#pragma unroll
            for (int j = 0; j < C; ++j) y[j] = x[i][j] * inv;
            if (r0 + i < rows) {
                uint8_t* to = q + (r0 + i) * ld + c;
                if constexpr (C == 8) {
                    *reinterpret_cast<uint2*>(to) = to_fp8x8(y);
                } else {
                    static_assert(C == 4, "four bytes");
                    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
                    *reinterpret_cast<int*>(to) = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
                }
            }
        }
    }
    if (!qt) return;
#pragma unroll
    for (int j = 0; j < C; ++j) {
        const float inv = col_inv[l * C + j];
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[i][j] * inv;
        *reinterpret_cast<uint2*>(turned + (l * C + j) * PITCH + g * 8) = to_fp8x8(y);
    }
    __syncthreads();
    for (int row = tid / 8; row < FP8_BLOCK; row += THREADS / 8) {
        const uint8_t* from = turned + row * PITCH + tid % 8 * 16;
        const uint2 a = *reinterpret_cast<const uint2*>(from), b = *reinterpret_cast<const uint2*>(from + 8);
        if (tc * FP8_BLOCK + row < cols)
            *reinterpret_cast<uint4*>(qt + (tc * FP8_BLOCK + row) * ldt + tr * FP8_BLOCK + tid % 8 * 16) = make_uint4(a.x, a.y, b.x, b.y);
    }
}

constexpr unsigned FEW_TILES = 512;      // two a CU

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
    const bool few = grid <= FEW_TILES;
    auto kernel = few ? (bf16 ? fp8_tile_kernel<true, 4> : fp8_tile_kernel<false, 4>) : (bf16 ? fp8_tile_kernel<true, 8> : fp8_tile_kernel<false, 8>);
    kernel<<<grid, few ? 512 : 256, 0, st>>>(X, rows, cols, ldx, vec, mask, kind, (int)cb, a.q, a.ld, a.scale, a.lds, b.q, b.ld, b.scale, b.lds);
    return hipGetLastError();
}

}  // namespace crisp
