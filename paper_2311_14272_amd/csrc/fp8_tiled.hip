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

// Chunk c of row r lies at place c ^ swizzle(r).  A read serves 16 lanes a cycle from 64 banks of 4 bytes, two rows' worth: of
// the 16 rows that those lanes want, the eight of either parity have different values here.
__device__ __forceinline__ int x_swizzle(int r) { return (r >> 1) & 7; }                       // rows 16n .. 16n+15
__device__ __forceinline__ int w_swizzle(int r) { return ((r >> 1) & 3) | ((r >> 2) & 4); }    // 8m+{0..7}, 8m+16+{0..7}

// Waits until at most `left` of the wave's memory operations are outstanding, and for all its LDS reads.
template <int LEFT>
__device__ __forceinline__ void wait_loads() {
    static_assert(LEFT < 64, "six bits");
    __builtin_amdgcn_s_waitcnt((LEFT & 15) | 7 << 4 | 0 << 8 | (LEFT >> 4) << 14);
}

// That wait, and the barrier: behind it no wave of the workgroup still reads what it read before, and the requests that the wait
// covered have arrived for all of them.  (The compiler moves no access of memory across an empty asm; it emits nothing.)
template <int LEFT>
__device__ __forceinline__ void wait_and_meet() {
    asm volatile("" ::: "memory");
    wait_loads<LEFT>();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// A wave's 32 x 32 results, register j of lane (i, h) row t0 + i and column s0 + 16h + j, through the epilogue and out.  They change
// lanes in LDS (4 KiB of the wave's own) so that a request writes whole rows of the tile: as 16 bytes here and there they left at
// 2 TB/s.
template <bool BF16>
__device__ __forceinline__ void store_tile(const ProductArgs& a, int t0, int s0, const f32x16& sums, float* own, int lane) {
    constexpr int N = BF16 ? 8 : 4, LANES = 32 / N, ROWS = 64 / LANES;      // columns of a lane; lanes of a row; rows of a request
    const int i = lane % 32, h = lane / 32;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        *reinterpret_cast<f32x4*>(own + i * 32 + ((4 * h + j) ^ (i & 7)) * 4) = f32x4{sums[4 * j], sums[4 * j + 1], sums[4 * j + 2], sums[4 * j + 3]};
    const int c = lane % LANES * N;
#pragma unroll
    for (int k = 0; k < 32 / ROWS; ++k) {
        const int row = k * ROWS + lane / LANES;
        float v[N];
#pragma unroll
        for (int j = 0; j < N; j += 4) {
            const f32x4 p = *reinterpret_cast<const f32x4*>(own + row * 32 + (((c + j) / 4) ^ (row & 7)) * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[j + e] = p[e];
        }
        store_row<N, BF16>(a, t0 + row, s0 + c, v);
    }
}

// NS x NT waves, each RS x RT tiles of 32 x 32; STAGES blocks in LDS, all but one of them on their way.  BF16: the result's
// type, and with it the instruction.  TILES: W has a scale for 128 x 128.
//
// KG: groups of waves that take the blocks in turn, for sizes whose tiles leave most CUs with one workgroup or none: a step then
// costs its latencies (a barrier, LDS reads, two dependent matrix instructions: 0.5 us measured), whatever it computes.  Their
// sums are added up in LDS, in the order of the groups.
//
// A step begins when its block has arrived for every wave (each waits for its own share, then all meet) - by then everybody
// is done with the block before, whose place the next request takes.  All a wave's memory operations are requests to LDS,
// the same number each step, so that the wait can leave the later steps' ones outstanding.
//
// One object of LDS a stage: W's rows, X's rows, scales.  The compiler tells requests to LDS apart by the object that they write,
// no more than eight of them, and follows few address steps from an object: every address here is an object and one offset.  Where
// it cannot tell, a read of LDS waits for all requests.
template <int NS, int NT, int RS, int RT, int KG>
struct Tiles {
    static constexpr int NW = NS * NT, BS = NS * RS * 32, BT = NT * RT * 32;
    static constexpr int LS = ((BS + BT) / 64 + NW - 1) / NW;    // requests of 64 scales that a wave makes per step (some may be nobody's)
    static constexpr int SC = LS * NW * 64;
    static constexpr int W = KG * BS * 128, X = KG * BT * 128, STAGE = W + X + KG * SC * 4;
};

template <int NS, int NT, int RS, int RT, int STAGES, int KG, bool BF16, bool TILES>
__device__ __forceinline__ void tiled_product(const ProductArgs& a, int tiles_s, int tiles_t, int id, uint8_t* st0, uint8_t* st1, uint8_t* st2,
                                              uint8_t* st3) {
    typedef Tiles<NS, NT, RS, RT, KG> G;
    constexpr int NW = G::NW, BS = G::BS, BT = G::BT, LS = G::LS, SC = G::SC, W = G::W, X = G::X, STAGE = G::STAGE;
    constexpr int LW = BS / 8 / NW, LX = BT / 8 / NW;            // requests of eight rows that a wave makes per step
    static_assert(BS % (8 * NW) == 0 && BT % (8 * NW) == 0 && BS % 64 == 0, "whole requests");
    constexpr int PER = LW + LX + LS;
    constexpr bool DIRECT = BF16 && RS * RT >= 6;                // results leave without changing lanes
    const int lane = threadIdx.x % 64, all = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int wave = all % NW, kg = all / NW;                    // (kg is 0 where there is one group)

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
        xo[j] = (uint32_t)min(r, a.T - 1 - t0) * (uint32_t)a.ldx + (lane % 8 ^ x_swizzle(r)) * 16;
    }
    const uint8_t *wb = a.w + s0 * a.ldw, *xb = a.x + t0 * a.ldx;
    // scales: a wave's 64 rows are W's or X's
    const float* sp[LS];
    int64_t sstep[LS];
#pragma unroll
    for (int j = 0; j < LS; ++j) {
        const int r = (wave + j * NW) * 64 + lane;
        if ((wave + j * NW) * 64 < BS) {
            const int row = min(s0 + r, a.S - 1);
            sp[j] = a.ws + (a.w_tiles ? row / 128 * a.ldws : (int64_t)row);
            sstep[j] = a.w_tiles ? 1 : a.ldws;
        } else {
            sp[j] = a.xs + min(t0 + r - BS, a.T - 1);
            sstep[j] = a.ldxs;
        }
    }

    const int i = lane % 32, h = lane / 32;
    const int ws = wave % NS, wt = wave / NS;
    const int si = 16 * (i >> 2 & 1) + 4 * (i >> 3) + (i & 3);
    int wr[4], xr[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        wr[c] = (kg * BS + ws * RS * 32 + si) * 128 + ((4 * h + c) ^ w_swizzle(si)) * 16;
        xr[c] = W + (kg * BT + wt * RT * 32 + i) * 128 + ((4 * h + c) ^ x_swizzle(i)) * 16;
    }

    f32x16 acc[RS][RT];
#pragma unroll
    for (int r = 0; r < RS; ++r)
#pragma unroll
        for (int q = 0; q < RT; ++q)
#pragma unroll
            for (int j = 0; j < 16; ++j) acc[r][q][j] = 0.0f;

    // request n of a step's PER.  Rows of W and X through buffer descriptors of the tile: the lane's offset stays, the block's goes
    // into the scalar one.
    const __amdgpu_buffer_rsrc_t wd = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(wb), 0, -1, 0x00027000);
    const __amdgpu_buffer_rsrc_t xd = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(xb), 0, -1, 0x00027000);
    auto request = [&](int n, int b, uint8_t* to) {
        if (n < LW) {
            const int j = n;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(wd, (lds_ptr)(to + ((kg * (BS / 8) + wave + j * NW) * 1024)), 16, (int)wo[j], b * 128, 0, 0);
        } else if (n < LW + LX) {
            const int j = n - LW;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(xd, (lds_ptr)(to + (W + (kg * (BT / 8) + wave + j * NW) * 1024)), 16, (int)xo[j], b * 128, 0, 0);
        } else {
            const int j = n - LW - LX;
            __builtin_amdgcn_global_load_lds((global_ptr)(sp[j] + b * sstep[j]), (lds_ptr)(to + (W + X + (kg * SC + (wave + j * NW) * 64) * 4)), 4, 0, 0);
        }
    };
    auto fetch = [&](int b, uint8_t* to) {
#pragma unroll
        for (int n = 0; n < PER; ++n) request(n, b, to);
    };

    const int xscale = W + X + 4 * (kg * SC + BS + wt * RT * 32 + i), wscales = W + X + 4 * (kg * SC + ws * RS * 32 + (TILES ? 0 : 16 * h));
    // one scale for all of a wave's W rows (otherwise one for 32: those never lie in two blocks)
    constexpr bool ONE = TILES && 128 % (RS * 32) == 0;
    auto compute = [&](const uint8_t* st, auto part) {
        i32x4 xv[RT][4], wv[4];
        float f[RT];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            wv[c] = *reinterpret_cast<const i32x4*>(st + wr[c]);
            xv[0][c] = *reinterpret_cast<const i32x4*>(st + xr[c]);
        }
#pragma unroll
        for (int q = 1; q < RT; ++q)
#pragma unroll
            for (int c = 0; c < 4; ++c) xv[q][c] = *reinterpret_cast<const i32x4*>(st + (xr[c] + q * 4096));
#pragma unroll
        for (int q = 0; q < RT; ++q) f[q] = *reinterpret_cast<const float*>(st + (xscale + q * 128));
        float wscale = TILES ? *reinterpret_cast<const float*>(st + wscales) : 0.0f;
        __builtin_amdgcn_sched_barrier(0);
        f32x4 wsv[4];
        const f32x16 zero = {};
        if constexpr (BF16) {
            // the matrix cores are a tile ahead of the sums that enter the accumulators
            f32x16 p[2];
#pragma unroll
            for (int k = 0; k <= RS * RT; ++k) {
                if (k < RS * RT) {
                    const int r = k / RT, q = k % RT;
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const i32x8 wa = __builtin_shufflevector(wv[2 * u], wv[2 * u + 1], 0, 1, 2, 3, 4, 5, 6, 7);
                        const i32x8 xa = __builtin_shufflevector(xv[q][2 * u], xv[q][2 * u + 1], 0, 1, 2, 3, 4, 5, 6, 7);
                        p[k % 2] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wa, xa, u ? p[k % 2] : zero, 0, 0, 0, 0, 0, 0);
                        __builtin_amdgcn_sched_barrier(0);
                        if (q == RT - 1 && r + 1 < RS) {
#pragma unroll
                            for (int c = 2 * u; c < 2 * u + 2; ++c) wv[c] = *reinterpret_cast<const i32x4*>(st + (wr[c] + (r + 1) * 4096));
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    }
                    if (ONE && k == 0) {
#pragma unroll
                        for (int e = 0; e < RT; ++e) f[e] *= wscale;
                    }
                    part(k);
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (k > 0) {
                    const int r = (k - 1) / RT, q = (k - 1) % RT;
                    if (!TILES && q == 0) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) wsv[c] = *reinterpret_cast<const f32x4*>(st + (wscales + r * 128 + 16 * c));
                    }
                    const float both = TILES && !ONE ? f[q] * wscale : f[q];
#pragma unroll
                    for (int j = 0; j < 16; ++j) acc[r][q][j] = __builtin_fmaf(p[(k - 1) % 2][j], TILES ? both : f[q] * wsv[j / 4][j % 4], acc[r][q][j]);
                    if (TILES && !ONE && q == RT - 1 && r + 1 < RS) wscale = *reinterpret_cast<const float*>(st + (wscales + (r + 1) * 128));
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        } else {
            // a row of tiles ahead; an eighth of the widening and of the sums goes between any two steps of the instruction
            f32x16 p[2][RT];
            bf16x8 xw[RT][8];
#pragma unroll
            for (int r = 0; r <= RS; ++r) {
                if (!TILES && r > 0) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) wsv[c] = *reinterpret_cast<const f32x4*>(st + (wscales + (r - 1) * 128 + 16 * c));
                }
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    if (r < RS) {
                        const bf16x8 wa = widen(wv[u / 2][u % 2 * 2], wv[u / 2][u % 2 * 2 + 1]);
#pragma unroll
                        for (int q = 0; q < RT; ++q) {
                            if (r == 0) xw[q][u] = widen(xv[q][u / 2][u % 2 * 2], xv[q][u / 2][u % 2 * 2 + 1]);
                            p[r % 2][q] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wa, xw[q][u], u ? p[r % 2][q] : zero, 0, 0, 0);
                        }
                        if (u % 2 == 1 && r + 1 < RS) wv[u / 2] = *reinterpret_cast<const i32x4*>(st + (wr[u / 2] + (r + 1) * 4096));
                        if (u == 1 && r == 0 && ONE) {
#pragma unroll
                            for (int e = 0; e < RT; ++e) f[e] *= wscale;
                        }
                        if (u % (8 / RT) == 8 / RT - 1 && u / (8 / RT) < RT) part(r * RT + u / (8 / RT));
                    }
                    if (r > 0) {
#pragma unroll
                        for (int q = 0; q < RT; ++q)
#pragma unroll
                            for (int j = 2 * u; j < 2 * u + 2; ++j)
                                acc[r - 1][q][j] = __builtin_fmaf(p[(r - 1) % 2][q][j], ONE ? f[q] : TILES ? f[q] * wscale : f[q] * wsv[j / 4][j % 4], acc[r - 1][q][j]);
                    }
                    if (TILES && !ONE && u == 7 && r > 0 && r < RS) wscale = *reinterpret_cast<const float*>(st + (wscales + r * 128));
                    if (r < RS) __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
    };

    constexpr int AHEAD = STAGES - 1;
    // tiles of a step that its requests go between: with two stages they have to arrive by the next step (8192^3: 425 us for three
    // eighths of the step, 423 for six, 440 for all)
    constexpr int SPREAD = STAGES == 2 ? (RS * RT * 6 + 7) / 8 : RS * RT;
    // (behind the last block the requests repeat it, into places that nobody reads any more: a step is then free of branches)
#define CRISP_STEP(k, here, there)                                                                                \
    {                                                                                                             \
        const int step = step0 + k, b = step * KG + kg;                                                           \
        const int ahead = min(b + AHEAD * KG, a.kb - 1);                                                          \
        wait_and_meet<(AHEAD - 1) * PER>();                                                                       \
        if (KG > 1 && b >= a.kb) break;               /* the last step may have no block for the later groups */  \
        compute(st##here, [&](int tile) {                                                                         \
            _Pragma("unroll") for (int n = 0; n < PER; ++n)                                                       \
                if (n * SPREAD / PER == tile) request(n, ahead, st##there);                                       \
        });                                                                                                       \
        if (step + 1 >= steps) break;                                                                             \
    }
    if constexpr (STAGES == 1) {                     // other workgroups of the CU work while this one waits
        static_assert(KG == 1, "one group");
        for (int b = 0; b < a.kb; ++b) {
            if (b) wait_and_meet<0>();               // (the block's reads are done in every wave: its place may be written)
            fetch(b, st0);
            wait_and_meet<0>();
            compute(st0, [](int) {});
        }
    } else {
        const int steps = (a.kb + KG - 1) / KG;
        fetch(min(kg, a.kb - 1), st0);
        if constexpr (AHEAD > 1) fetch(min(KG + kg, a.kb - 1), st1);
        if constexpr (AHEAD > 2) fetch(min(2 * KG + kg, a.kb - 1), st2);
        // (with requests under way at the loop's head the compiler would wait for all of them in each of its rounds)
        wait_loads<0>();
        for (int step0 = 0;; step0 += STAGES) {
            if constexpr (STAGES == 2) {
                CRISP_STEP(0, 0, 1) CRISP_STEP(1, 1, 0)
            } else if constexpr (STAGES == 3) {
                CRISP_STEP(0, 0, 2) CRISP_STEP(1, 1, 0) CRISP_STEP(2, 2, 1)
            } else {
                CRISP_STEP(0, 0, 3) CRISP_STEP(1, 1, 0) CRISP_STEP(2, 2, 1) CRISP_STEP(3, 3, 2)
            }
        }
    }
#undef CRISP_STEP
    if constexpr (DIRECT) wait_loads<0>();
    else wait_and_meet<0>();
    if constexpr (KG > 1) {
        static_assert(STAGE >= BS * BT * 4, "a group's sums fit a stage");
        f32x16* part = reinterpret_cast<f32x16*>(st0);
#pragma unroll
        for (int g = 1; g < KG; ++g) {
            __syncthreads();
#pragma unroll
            for (int r = 0; r < RS; ++r)
#pragma unroll
                for (int q = 0; q < RT; ++q) {
                    f32x4* p = reinterpret_cast<f32x4*>(part + ((wave * RS + r) * RT + q) * 64);     // four registers of all lanes at a time
                    if (kg == g) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) p[j * 64 + lane] = f32x4{acc[r][q][4 * j], acc[r][q][4 * j + 1], acc[r][q][4 * j + 2], acc[r][q][4 * j + 3]};
                    }
                }
            __syncthreads();
            if (kg == 0) {
#pragma unroll
                for (int r = 0; r < RS; ++r)
#pragma unroll
                    for (int q = 0; q < RT; ++q) {
                        const f32x4* p = reinterpret_cast<const f32x4*>(part + ((wave * RS + r) * RT + q) * 64);
#pragma unroll
                        for (int j = 0; j < 16; ++j) acc[r][q][j] += p[j / 4 * 64 + lane][j % 4];
                    }
            }
        }
        if (kg > 0) return;
    }

    // With six tiles and more a wave the way round by LDS costs 1 to 3 % (4096 x 11008 x 4096, a scale for each W row: 212.5 us against 206).
    // (a group's sums lay in the stage too: every wave goes on in the place of its own)
    float* own = reinterpret_cast<float*>(st0 + wave * (KG > 1 ? RS * RT : 1) * 4096);
    static_assert(KG > 1 || STAGE >= NW * 4096, "a tile a wave");
#pragma unroll
    for (int r = 0; r < RS; ++r)
#pragma unroll
        for (int q = 0; q < RT; ++q) {
            if constexpr (DIRECT) {
                float v[16];
#pragma unroll
                for (int j = 0; j < 16; ++j) v[j] = acc[r][q][j];
                store_row<16, true>(a, t0 + (wt * RT + q) * 32 + i, s0 + (ws * RS + r) * 32 + 16 * h, v);
            } else {
                store_tile<BF16>(a, t0 + (wt * RT + q) * 32, s0 + (ws * RS + r) * 32, acc[r][q], own, lane);
            }
        }
}

template <int NS, int NT, int RS, int RT, int STAGES, int KG, bool BF16, bool TILES>
__global__ __launch_bounds__(64 * NS * NT * KG, 2) void fp8_tiled_kernel(ProductArgs a, int tiles_s, int tiles_t) {
    constexpr int STAGE = Tiles<NS, NT, RS, RT, KG>::STAGE;
    __shared__ __align__(16) uint8_t st0[STAGE], st1[STAGES > 1 ? STAGE : 16], st2[STAGES > 2 ? STAGE : 16], st3[STAGES > 3 ? STAGE : 16];
    tiled_product<NS, NT, RS, RT, STAGES, KG, BF16, TILES>(a, tiles_s, tiles_t, (int)blockIdx.x, st0, st1, st2, st3);
}

// A layer's two gradients in one launch, the input's (bf16, W with a scale for 128 x 128) in the first workgroups, the weight's
// (fp32, both operands with a scale for each row) in the others.
template <int STAGES, int KG>
__global__ __launch_bounds__(256 * KG, 2) void fp8_pair_kernel(ProductArgs a, ProductArgs b, int a_s, int a_t, int b_s, int b_t) {
    constexpr int STAGE = Tiles<2, 2, 1, 1, KG>::STAGE;
    __shared__ __align__(16) uint8_t st0[STAGE], st1[STAGE], st2[STAGES > 2 ? STAGE : 16];
    const int first = a_s * a_t;
    if ((int)blockIdx.x < first) tiled_product<2, 2, 1, 1, STAGES, KG, true, true>(a, a_s, a_t, (int)blockIdx.x, st0, st1, st2, nullptr);
    else tiled_product<2, 2, 1, 1, STAGES, KG, false, false>(b, b_s, b_t, (int)blockIdx.x - first, st0, st1, st2, nullptr);
}

// ALWAYS: W has a scale for 128 x 128, whatever calls.
template <int NS, int NT, int RS, int RT, int STAGES, int KG, bool BF16, bool ALWAYS = false>
static void launch_tiles(const ProductArgs& a, hipStream_t st) {
    const int ts = (a.S + NS * RS * 32 - 1) / (NS * RS * 32), tt = (a.T + NT * RT * 32 - 1) / (NT * RT * 32);
    auto kernel = a.w_tiles || ALWAYS ? fp8_tiled_kernel<NS, NT, RS, RT, STAGES, KG, BF16, true> : fp8_tiled_kernel<NS, NT, RS, RT, STAGES, KG, BF16, ALWAYS>;
    kernel<<<(unsigned)ts * (unsigned)tt, 64 * NS * NT * KG, 0, st>>>(a, ts, tt);
}

hipError_t launch_fp8_pair(int pairs, const ProductArgs& a, const ProductArgs& b, hipStream_t st) {
    const int as = (a.S + 63) / 64, at = (a.T + 63) / 64, bs = (b.S + 63) / 64, bt = (b.T + 63) / 64;
    const unsigned grid = (unsigned)(as * at + bs * bt);
    if (pairs == 1) fp8_pair_kernel<3, 2><<<grid, 512, 0, st>>>(a, b, as, at, bs, bt);
    else fp8_pair_kernel<2, 1><<<grid, 256, 0, st>>>(a, b, as, at, bs, bt);
    return hipGetLastError();
}

hipError_t launch_fp8_tiled(const ProductArgs& a, hipStream_t st) {
    switch (fp8_tile_shape(size_of(a)) * 2 + a.y_bf16) {
        case 0: launch_tiles<2, 2, 1, 1, 3, 2, false>(a, st); break;
        case 1: launch_tiles<2, 2, 1, 1, 3, 2, true>(a, st); break;
        case 2: launch_tiles<2, 2, 1, 1, 1, 1, false>(a, st); break;
        case 3: launch_tiles<2, 2, 1, 1, 1, 1, true>(a, st); break;
        case 4: launch_tiles<2, 2, 1, 1, 2, 1, false>(a, st); break;
        case 5: launch_tiles<2, 2, 1, 1, 2, 1, true>(a, st); break;
        case 7: launch_tiles<2, 2, 2, 1, 3, 2, true>(a, st); break;
        case 8: launch_tiles<2, 2, 2, 1, 2, 1, false>(a, st); break;
        case 11: launch_tiles<2, 4, 2, 1, 4, 1, true, true>(a, st); break;
        case 12: launch_tiles<2, 2, 2, 2, 2, 1, false>(a, st); break;
        case 13: launch_tiles<2, 4, 2, 1, 2, 1, true>(a, st); break;
        case 15: launch_tiles<2, 4, 3, 1, 3, 1, true>(a, st); break;
        case 17: launch_tiles<2, 4, 3, 2, 2, 1, true>(a, st); break;
        default: launch_tiles<2, 4, 4, 2, 2, 1, true, true>(a, st); break;
    }
    return hipGetLastError();
}

}  // namespace crisp
