// Quantisation to e4m3 with one scale for each block of 128 columns of a row, or of 128 x 128 elements: read once, largest
// magnitude per block, multiply by the scale's inverse, round, write one or both directions.  Bound by memory.
#include "fp8_common.h"
#include "fp8_internal.h"

namespace crisp {

// ROWS, one direction, no mask: 16 lanes take a block of 128 columns, a workgroup 16 consecutive blocks of the matrix in
// row order.
template <bool BF16>
__global__ __launch_bounds__(256) void fp8_rows_kernel(const void* __restrict__ X, int64_t rows, int cols, int64_t ldx,
                                                       uint8_t* __restrict__ q, int64_t ld, float* __restrict__ scale, int64_t lds) {
    const int kb = (cols + FP8_BLOCK - 1) / FP8_BLOCK;
    const int64_t id = (int64_t)blockIdx.x * 16 + threadIdx.x / 16;
    const int64_t r = id / kb;
    const int b = (int)(id - r * kb), lane = threadIdx.x % 16;
    if (r >= rows) return;      // all 16 lanes of a group leave together
    const int c = b * FP8_BLOCK + lane * 8;
    Elements<BF16, 8> in[1];
    read_rows(in, X, c, cols, [&](int) { return r * ldx; });
    float x[8], s;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = in[0][j];
    *reinterpret_cast<uint2*>(q + r * ld + c) = quantize_block(x, s);
    if (lane == 0) scale[b * lds + r] = s;
}

// A 128 x 128 tile per workgroup, for everything else.  Thread (g, l): rows 8g .. 8g+7, columns 4l .. 4l+3, held in registers as
// they were read.  Largest magnitudes meet in LDS, where one thread each makes the scale of a row or column.  The transpose is
// eight bytes per column and thread, gathered in LDS so that it leaves in whole rows.
// bf16 in both directions: 8192 x 4096 26.6 us (128 MiB, 5.0 TB/s), 2048 x 2048 6.3, 500 x 512 4.7; with eight columns a thread, half as
// many of them, 26.1, 6.9 and 5.4.  With conditions around the reads, each waiting for the one before, 34.8, 6.6 and 5.4.
constexpr int C = 4;
template <bool BF16>
__global__ __launch_bounds__(512) void fp8_tile_kernel(const void* __restrict__ X, int64_t rows, int64_t cols, int64_t ldx,
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
    auto row = [&](int i) { return r0 + i < rows ? r0 + i : rows - 1; };      // (rows behind the last one repeat it, and are zeros below)
    uint32_t bits[8];
    if (mask) {
        const int64_t words = (cols + 31) / 32, word = c < cols ? c / 32 : 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) bits[i] = mask[row(i) * words + word];
    }
    Elements<BF16, C> x[8];
    read_rows(x, X, c, cols, [&](int i) { return row(i) * ldx; });
    if (mask) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i].keep(bits[i] >> (c % 32));
    }
    if (r0 + 8 > rows) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i].keep(r0 + i < rows ? ~0u : 0u);
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
        t = umax(t, (uint32_t)__shfl_xor((int)t, 16));
        if (l == i) row_top[g * 8 + i] = t;
    }
    if (!tiles && qt) {
#pragma unroll
        for (int j = 0; j < C; ++j) {
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
                const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
                *reinterpret_cast<int*>(q + (r0 + i) * ld + c) = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
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

hipError_t launch_fp8_quant(const void* X, int in_type, int64_t rows, int64_t cols, int64_t ldx, const uint32_t* mask,
                            const crisp_fp8_mat* Q, const crisp_fp8_mat* Qt, hipStream_t st) {
    const bool bf16 = in_type == CRISP_IN_BF16;
    const int64_t rb = (rows + FP8_BLOCK - 1) / FP8_BLOCK, cb = (cols + FP8_BLOCK - 1) / FP8_BLOCK;
    const int kind = Q ? Q->kind : Qt->kind;
    if (kind == CRISP_FP8_ROWS && !Qt && !mask) {
        const unsigned grid = (unsigned)((rows * cb + 15) / 16);
        if (bf16) fp8_rows_kernel<true><<<grid, 256, 0, st>>>(X, rows, (int)cols, ldx, Q->q, Q->ld, Q->scale, Q->lds);
        else fp8_rows_kernel<false><<<grid, 256, 0, st>>>(X, rows, (int)cols, ldx, Q->q, Q->ld, Q->scale, Q->lds);
        return hipGetLastError();
    }
    const crisp_fp8_mat none = {};
    const crisp_fp8_mat &a = Q ? *Q : none, &b = Qt ? *Qt : none;
    auto kernel = bf16 ? fp8_tile_kernel<true> : fp8_tile_kernel<false>;
    kernel<<<(unsigned)(rb * cb), 512, 0, st>>>(X, rows, cols, ldx, mask, kind, (int)cb, a.q, a.ld, a.scale, a.lds, b.q, b.ld, b.scale, b.lds);
    return hipGetLastError();
}

}  // namespace crisp
