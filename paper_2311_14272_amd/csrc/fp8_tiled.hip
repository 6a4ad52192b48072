// The 8-bit product for many rows: a workgroup computes BS x BT results (W rows x X rows) block by block.  Both operands' next
// block travels from memory into LDS, sixteen bytes a lane and without passing through registers, while the matrix cores work
// on the present one.
//
// LDS holds rows of 128 bytes; the 16-byte chunks of a row are permuted by its number so that the lanes of a read fall on
// different banks.  Within a row the lanes of either half of a wave take four chunks each; the order of the columns does not
// matter as long as both operands have the same one.  Row 8q + 4h + e of the matrix instruction is W row 16h + 4q + e of its 32:
// a lane's 16 sums, rows 8q + 4h + e for its h, are then consecutive in Y.
//
// Workgroups go round the XCDs by their number: consecutive tiles of one XCD are a patch of GROUP X tiles by all W tiles, so
// that its L2 sees each operand's blocks several times.
#include "fp8_product.h"

namespace crisp {

typedef const __attribute__((address_space(1))) void* global_ptr;
typedef __attribute__((address_space(3))) void* lds_ptr;

constexpr int GROUP = 4;
constexpr int XCDS = 8;

__device__ __forceinline__ int w_swizzle(int r) { return (r & 3) | ((r >> 2) & 4); }

// Sixteen consecutive results of row t from column s on.
template <bool BF16>
__device__ __forceinline__ void store_y16(const ProductArgs& a, int t, int s, const f32x16& v, bool plain) {
    if (t >= a.T) return;
    if (plain && s + 16 <= a.S) {
        if constexpr (BF16) {
            uint4* p = reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.y) + t * a.ldy + s);
            p[0] = make_uint4(to_bf16x2(v[0], v[1]), to_bf16x2(v[2], v[3]), to_bf16x2(v[4], v[5]), to_bf16x2(v[6], v[7]));
            p[1] = make_uint4(to_bf16x2(v[8], v[9]), to_bf16x2(v[10], v[11]), to_bf16x2(v[12], v[13]), to_bf16x2(v[14], v[15]));
        } else {
            f32x4* p = reinterpret_cast<f32x4*>(static_cast<float*>(a.y) + t * a.ldy + s);
#pragma unroll
            for (int j = 0; j < 4; ++j) p[j] = f32x4{v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]};
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 16; ++j)
        if (s + j < a.S) store_y(a, t, s + j, v[j]);
}

// NS x NT waves, each RS x RT tiles of 32 x 32.  BF16: the result's type, and with it the instruction.  TILES: W's scales.
template <int NS, int NT, int RS, int RT, bool BF16, bool TILES>
__global__ __launch_bounds__(64 * NS * NT, NS * NT == 8 ? 2 : 2) void fp8_tiled_kernel(ProductArgs a, int tiles_s, int tiles_t) {
    constexpr int NW = NS * NT, BS = NS * RS * 32, BT = NT * RT * 32;
    constexpr int LW = BS / 8 / NW, LX = BT / 8 / NW;            // loads of eight rows that a wave issues
    __shared__ __align__(16) uint8_t w_even[BS * 128], w_odd[BS * 128], x_even[BT * 128], x_odd[BT * 128];
    __shared__ __align__(16) float s_even[TILES ? 4 : BS], s_odd[TILES ? 4 : BS];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);

    int id = blockIdx.x;
    const int n = tiles_s * tiles_t, per = n / XCDS;
    if (id < per * XCDS) id = id % XCDS * per + id / XCDS;
    const int in_group = GROUP * tiles_s, group = id / in_group, first = group * GROUP;
    const int high = min(GROUP, tiles_t - first), rest = id - group * in_group;
    const int t0 = (first + rest % high) * BT, s0 = rest / high * BS;

    // what each lane fetches: rows behind the last one repeat it, their results are not stored
    uint32_t wo[LW], xo[LX];
#pragma unroll
    for (int j = 0; j < LW; ++j) {
        const int r = (wave + j * NW) * 8 + lane / 8;
        wo[j] = (uint32_t)min(r, a.S - 1 - s0) * (uint32_t)a.ldw + (lane % 8 ^ w_swizzle(r)) * 16;
    }
#pragma unroll
    for (int j = 0; j < LX; ++j) {
        const int r = (wave + j * NW) * 8 + lane / 8;
        xo[j] = (uint32_t)min(r, a.T - 1 - t0) * (uint32_t)a.ldx + (lane % 8 ^ r % 8) * 16;
    }
    const uint8_t *wb = a.w + s0 * a.ldw, *xb = a.x + t0 * a.ldx;

    const int i = lane % 32, h = lane / 32;
    const int ws = wave % NS, wt = wave / NS;
    const int si = 16 * (i >> 2 & 1) + 4 * (i >> 3) + (i & 3);
    int wr[4], xr[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        wr[c] = (ws * RS * 32 + si) * 128 + ((4 * h + c) ^ w_swizzle(si)) * 16;
        xr[c] = (wt * RT * 32 + i) * 128 + ((4 * h + c) ^ (i & 7)) * 16;
    }
    int tcol[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) tcol[r] = min(t0 + (wt * RT + r) * 32 + i, a.T - 1);
    const float* wscale = a.ws + (TILES ? (int64_t)min((s0 + ws * RS * 32) / 128, (a.S - 1) / 128) * a.ldws : 0);

    f32x16 acc[RS][RT];
#pragma unroll
    for (int r = 0; r < RS; ++r)
#pragma unroll
        for (int q = 0; q < RT; ++q)
#pragma unroll
            for (int j = 0; j < 16; ++j) acc[r][q][j] = 0.0f;
    float next[RT], wnext = 0.0f;

    auto fetch = [&](int b, uint8_t* wl, uint8_t* xl, float* sl) {
#pragma unroll
        for (int r = 0; r < RT; ++r) next[r] = a.xs[b * a.ldxs + tcol[r]];
        if constexpr (TILES) {
            wnext = wscale[b];
        } else {
            if (wave < BS / 64) {
                const int row = min(s0 + wave * 64 + lane, a.S - 1);
                __builtin_amdgcn_global_load_lds((global_ptr)(a.ws + b * a.ldws + row), (lds_ptr)(sl + wave * 64), 4, 0, 0);
            }
        }
        const uint8_t *wp = wb + (int64_t)b * 128, *xp = xb + (int64_t)b * 128;
#pragma unroll
        for (int j = 0; j < LW; ++j) __builtin_amdgcn_global_load_lds((global_ptr)(wp + wo[j]), (lds_ptr)(wl + (wave + j * NW) * 1024), 16, 0, 0);
#pragma unroll
        for (int j = 0; j < LX; ++j) __builtin_amdgcn_global_load_lds((global_ptr)(xp + xo[j]), (lds_ptr)(xl + (wave + j * NW) * 1024), 16, 0, 0);
    };

    auto compute = [&](const uint8_t* wl, const uint8_t* xl, const float* sl, const float (&f)[RT]) {
        i32x4 xv[RT][4];
#pragma unroll
        for (int q = 0; q < RT; ++q)
#pragma unroll
            for (int c = 0; c < 4; ++c) xv[q][c] = *reinterpret_cast<const i32x4*>(xl + xr[c] + q * 4096);
        bf16x8 xw[BF16 ? 1 : RT][8];
        if constexpr (!BF16) {
#pragma unroll
            for (int q = 0; q < RT; ++q)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    xw[q][2 * c] = widen(xv[q][c][0], xv[q][c][1]);
                    xw[q][2 * c + 1] = widen(xv[q][c][2], xv[q][c][3]);
                }
        }
#pragma unroll
        for (int r = 0; r < RS; ++r) {
            i32x4 wv[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) wv[c] = *reinterpret_cast<const i32x4*>(wl + wr[c] + r * 4096);
            f32x4 wsv[4];
            if constexpr (!TILES) {
#pragma unroll
                for (int c = 0; c < 4; ++c) wsv[c] = *reinterpret_cast<const f32x4*>(sl + (ws * RS + r) * 32 + 16 * h + 4 * c);
            }
            f32x16 p[RT];
            const f32x16 zero = {};
            if constexpr (BF16) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const i32x8 wa = __builtin_shufflevector(wv[2 * k], wv[2 * k + 1], 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
                    for (int q = 0; q < RT; ++q) {
                        const i32x8 xa = __builtin_shufflevector(xv[q][2 * k], xv[q][2 * k + 1], 0, 1, 2, 3, 4, 5, 6, 7);
                        p[q] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wa, xa, k ? p[q] : zero, 0, 0, 0, 0, 0, 0);
                    }
                }
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const bf16x8 wa = widen(wv[k / 2][k % 2 * 2], wv[k / 2][k % 2 * 2 + 1]);
#pragma unroll
                    for (int q = 0; q < RT; ++q) p[q] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wa, xw[q][k], k ? p[q] : zero, 0, 0, 0);
                }
            }
#pragma unroll
            for (int q = 0; q < RT; ++q)
#pragma unroll
                for (int j = 0; j < 16; ++j) acc[r][q][j] = __builtin_fmaf(p[q][j], TILES ? f[q] : f[q] * wsv[j / 4][j % 4], acc[r][q][j]);
        }
    };

    float f[RT];
    auto take = [&]() {
#pragma unroll
        for (int r = 0; r < RT; ++r) f[r] = TILES ? next[r] * wnext : next[r];
    };
    fetch(0, w_even, x_even, s_even);
    __syncthreads();
    for (int b = 0; b < a.kb; b += 2) {
        take();
        if (b + 1 < a.kb) fetch(b + 1, w_odd, x_odd, s_odd);
        compute(w_even, x_even, s_even, f);
        __syncthreads();
        if (b + 1 >= a.kb) break;
        take();
        if (b + 2 < a.kb) fetch(b + 2, w_even, x_even, s_even);
        compute(w_odd, x_odd, s_odd, f);
        __syncthreads();
    }

    const bool plain = !a.scale && !a.bias && !a.residual && !a.relu && ((uintptr_t)a.y & 15) == 0 && a.ldy % (BF16 ? 8 : 4) == 0;
#pragma unroll
    for (int r = 0; r < RS; ++r)
#pragma unroll
        for (int q = 0; q < RT; ++q)
            store_y16<BF16>(a, t0 + (wt * RT + q) * 32 + i, s0 + (ws * RS + r) * 32 + 16 * h, acc[r][q], plain);
}

template <int NS, int NT, int RS, int RT, bool BF16>
static void launch_tiles(const ProductArgs& a, hipStream_t st) {
    const int ts = (a.S + NS * RS * 32 - 1) / (NS * RS * 32), tt = (a.T + NT * RT * 32 - 1) / (NT * RT * 32);
    const unsigned grid = (unsigned)ts * (unsigned)tt;
    if (a.w_tiles) fp8_tiled_kernel<NS, NT, RS, RT, BF16, true><<<grid, 64 * NS * NT, 0, st>>>(a, ts, tt);
    else fp8_tiled_kernel<NS, NT, RS, RT, BF16, false><<<grid, 64 * NS * NT, 0, st>>>(a, ts, tt);
}

hipError_t launch_fp8_tiled(const ProductArgs& a, hipStream_t st) {
    const int64_t big = (int64_t)((a.S + 255) / 256) * ((a.T + 255) / 256);
    // 256 x 256 tiles where they fill three quarters of the CUs.  Widening to bf16 takes more registers than such a wave has
    // left: 128 x 128 for fp32 results (4096 x 4096 x 4096: 660 TFLOP/s with 256 x 256, 980 at half the rows with 128 x 128).
    if (a.y_bf16 && big >= 192) launch_tiles<2, 4, 4, 2, true>(a, st);
    else if (a.y_bf16) launch_tiles<2, 2, 2, 2, true>(a, st);
    else launch_tiles<2, 2, 2, 2, false>(a, st);
    return hipGetLastError();
}

}  // namespace crisp
