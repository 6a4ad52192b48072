// The 8-bit product for few rows of X: the weights are read once and bound it, so nothing is staged.  A workgroup computes
// 16 MS x 16 MT results (W rows x X rows); its waves take the blocks of 128 columns in turn, straight from memory into the
// matrix instruction's registers, and add their sums up in LDS, in the order of the waves.
//
// Lane l holds 32 columns of row l % 16 of either operand, the same ones of both, so that their order does not matter;
// register i of lane l is (W row 4 (l / 16) + i, X row l % 16).
#include "fp8_product.h"

namespace crisp {

template <bool BF16>
__device__ __forceinline__ f32x4 block_sum(const i32x4 (&w)[2], const i32x4 (&x)[2]) {
    f32x4 c = {0.0f, 0.0f, 0.0f, 0.0f};
    if constexpr (BF16) {
        const i32x8 wa = __builtin_shufflevector(w[0], w[1], 0, 1, 2, 3, 4, 5, 6, 7);
        const i32x8 xa = __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wa, xa, c, 0, 0, 0, 0, 0, 0);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(w[k / 2][k % 2 * 2], w[k / 2][k % 2 * 2 + 1]),
                                                        widen(x[k / 2][k % 2 * 2], x[k / 2][k % 2 * 2 + 1]), c, 0, 0, 0);
        return c;
    }
}

// U: blocks that a wave requests at a time.  RAW: X is not in 8 bits yet; the workgroup quantises it into LDS, all of it, while its
// first weights are on their way (16 rows at most, and FP8_OWN_BLOCKS blocks).
template <int MS, int MT, int U, int WAVES, bool BF16, bool TILES, bool RAW>
__global__ __launch_bounds__(64 * WAVES) void fp8_split_kernel(ProductArgs a, int tiles_s) {
    __shared__ f32x4 part[WAVES][MS * MT][64];
    __shared__ __align__(16) uint8_t own_q[RAW ? FP8_OWN_BLOCKS * 128 : 16];
    __shared__ float own_s[RAW ? FP8_OWN_BLOCKS : 1];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int i = lane % 16, h = lane / 16;
    const int s0 = (int)(blockIdx.x % tiles_s) * (16 * MS), t0 = (int)(blockIdx.x / tiles_s) * (16 * MT);
    // rows behind the last one repeat it, their results are not stored
    const uint8_t *w[MS], *x[MT] = {};
    const float* xs[MT] = {};
    const float* wsp[MS];
#pragma unroll
    for (int r = 0; r < MS; ++r) {
        w[r] = a.w + min(s0 + 16 * r + i, a.S - 1) * a.ldw + h * 32;
        wsp[r] = TILES ? a.ws + min(s0 + 16 * r, a.S - 1) / 128 * a.ldws : a.ws;
    }
#pragma unroll
    for (int q = 0; q < (RAW ? 0 : MT); ++q) {
        const int t = min(t0 + 16 * q + i, a.T - 1);
        x[q] = a.x + t * a.ldx + h * 32;
        xs[q] = a.xs + t;
    }
    f32x4 sum[MS][MT];
#pragma unroll
    for (int r = 0; r < MS; ++r)
#pragma unroll
        for (int q = 0; q < MT; ++q) sum[r][q] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    i32x4 wv[U][MS][2];
    float g[U][MS][TILES ? 1 : 4];
    auto weights = [&](int b0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int b = min(b0 + u * WAVES, a.kb - 1);       // (behind the last block it is fetched again and left out)
#pragma unroll
            for (int r = 0; r < MS; ++r) {
                wv[u][r][0] = *reinterpret_cast<const i32x4*>(w[r] + (int64_t)b * 128);
                wv[u][r][1] = *reinterpret_cast<const i32x4*>(w[r] + (int64_t)b * 128 + 16);
                if constexpr (TILES) {
                    g[u][r][0] = wsp[r][b];
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) g[u][r][j] = a.ws[b * a.ldws + min(s0 + 16 * r + 4 * h + j, a.S - 1)];
                }
            }
        }
    };
    if constexpr (RAW) {
        static_assert(MT == 1, "one tile of X rows");
        weights(wave);
        __builtin_amdgcn_sched_barrier(0);
        const int blocks = a.T * a.kb;
        for (int e0 = 0; e0 < blocks; e0 += 4 * WAVES) {
            const int e = e0 + threadIdx.x / 16;
            if (e < blocks) {
                const int t = e / a.kb, c = (e - t * a.kb) * 128 + threadIdx.x % 16 * 8;
                float v[8], scale;
                auto own = [&](auto in) {
                    read_rows(in.x, a.raw, c, a.K, [&](int) { return t * a.ldraw; });
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = in.x[0][j];
                };
                struct Half { Elements<true, 8> x[1]; };
                struct Whole { Elements<false, 8> x[1]; };
                if (a.raw_bf16) own(Half());
                else own(Whole());
                *reinterpret_cast<uint2*>(own_q + e * 128 + threadIdx.x % 16 * 8) = quantize_block(v, scale);
                if (threadIdx.x % 16 == 0) own_s[e] = scale;
            }
        }
        __syncthreads();
    }

    for (int b0 = wave; b0 < a.kb; b0 += U * WAVES) {
        i32x4 xv[U][MT][2];
        float f[U][MT];
        if (!RAW || b0 != wave) weights(b0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int b = min(b0 + u * WAVES, a.kb - 1);
#pragma unroll
            for (int q = 0; q < MT; ++q) {
                if constexpr (RAW) {
                    const int e = min(i, a.T - 1) * a.kb + b;
                    xv[u][q][0] = *reinterpret_cast<const i32x4*>(own_q + e * 128 + h * 32);
                    xv[u][q][1] = *reinterpret_cast<const i32x4*>(own_q + e * 128 + h * 32 + 16);
                    f[u][q] = own_s[e];
                } else {
                    xv[u][q][0] = *reinterpret_cast<const i32x4*>(x[q] + (int64_t)b * 128);
                    xv[u][q][1] = *reinterpret_cast<const i32x4*>(x[q] + (int64_t)b * 128 + 16);
                    f[u][q] = xs[q][b * a.ldxs];
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);       // all requests first
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool there = b0 + u * WAVES < a.kb;
#pragma unroll
            for (int r = 0; r < MS; ++r)
#pragma unroll
                for (int q = 0; q < MT; ++q) {
                    const f32x4 p = block_sum<BF16>(wv[u][r], xv[u][q]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float next = __builtin_fmaf(p[j], f[u][q] * g[u][r][TILES ? 0 : j], sum[r][q][j]);
                        sum[r][q][j] = there ? next : sum[r][q][j];
                    }
                }
        }
    }
#pragma unroll
    for (int r = 0; r < MS; ++r)
#pragma unroll
        for (int q = 0; q < MT; ++q) part[wave][r * MT + q][lane] = sum[r][q];
    __syncthreads();
    // thread (tile, lane): four consecutive results of a row
    for (int e = threadIdx.x; e < MS * MT * 64; e += 64 * WAVES) {
        const int tile = e / 64, l = e % 64;
        f32x4 y = part[0][tile][l];
        // (four at a time: 64 registers let two workgroups of 16 waves run on a CU, 8 x 11008 x 4096 13.1 us against 14.8 with one)
#pragma unroll 4
        for (int v = 1; v < WAVES; ++v) y += part[v][tile][l];
        float v[4] = {y[0], y[1], y[2], y[3]};
        store_row<4, BF16>(a, t0 + tile % MT * 16 + l % 16, s0 + tile / MT * 16 + l / 16 * 4, v);
    }
}

template <int MS, int MT, int U, int WAVES, bool RAW = false>
static void launch_split(const ProductArgs& a, hipStream_t st) {
    const int ts = (a.S + 16 * MS - 1) / (16 * MS), tt = (a.T + 16 * MT - 1) / (16 * MT);
    auto kernel = a.y_bf16 ? (a.w_tiles ? fp8_split_kernel<MS, MT, U, WAVES, true, true, RAW> : fp8_split_kernel<MS, MT, U, WAVES, true, false, RAW>)
                           : (a.w_tiles ? fp8_split_kernel<MS, MT, U, WAVES, false, true, RAW> : fp8_split_kernel<MS, MT, U, WAVES, false, false, RAW>);
    kernel<<<(unsigned)ts * (unsigned)tt, 64 * WAVES, 0, st>>>(a, ts);
}

// (the sums' order depends on the number of waves alone)
hipError_t launch_fp8_split(const ProductArgs& a, hipStream_t st) {
    const Fp8Size z = size_of(a);
    const bool many = fp8_split_waves(z.kb) == 16, two = fp8_split_estimate(z, 2) < fp8_split_estimate(z, 1);
    if (a.raw) many ? launch_split<1, 1, 2, 16, true>(a, st) : launch_split<1, 1, 2, 8, true>(a, st);
    else if (two) many ? launch_split<2, 1, 2, 16>(a, st) : launch_split<2, 1, 2, 8>(a, st);
    else many ? launch_split<1, 1, 2, 16>(a, st) : launch_split<1, 1, 2, 8>(a, st);
    return hipGetLastError();
}

}  // namespace crisp
