// Which kernel of the 8-bit product takes which sizes.  Host arithmetic only, so that it also runs in a host test.
#pragma once
#include <stdint.h>

namespace crisp {

// A product: rows of X, rows of W, blocks of 128 columns, the result's type, whether W has a scale for 128 x 128.
struct Fp8Size { int T, S, kb; bool bf16, w_tiles; };

// The tile and its stages by estimated time.  Kernels of one workgroup a CU (their stages fill its LDS) take, for each round of 256 of
// them, a first request and a last store that nothing hides and a time for each block.  Of those with one or two small stages
// several run on a CU and hide these from each other: the work of a CU's tiles counts once a tile, or the way through the blocks
// once for as many as run together.  So small tiles win where the results' way out bounds the time (few blocks) or their number
// does not fill the last round, large ones where the matrix cores do.
//
// Constants in microseconds, fitted to the times of 266 sizes of 33 x 33 x 16 to 9000 x 12000 x 9000 for each type; the rule's choices take
// 2 % longer than the best of twelve to fourteen shapes, in the geometric mean.  A few sizes, us (the rule's choices marked; --: no registers
// for it; not built: 128 x 64 for bf16, 192 x 128 for fp32, 128 x 256, which gains 2.5 % at the last size for fp32 and is behind
// at the others):
//
//                          5632 x 2614 x 16   8192 x 5120 x 256    1280 x 3456 x 1840     4096 x 4096 x 4096
//                           fp32    bf16        fp32    bf16         fp32    bf16           fp32    bf16
//   64 x 64, two groups     51.3    41.4       135.6   112.4         47.1    32.0          236.3   158.2
//   64 x 64, one stage      17.3*   11.6*       48.1*   28.8*        30.1    21.2          169.1   109.8
//   64 x 64, two stages     18.6    14.2        50.4    36.6         31.5*   24.1          169.5   111.1
//   128 x 64, two stages    19.0    14.1        51.5    36.5         30.7    20.8          157.8    91.9
//   128 x 128, two stages   21.0    14.5        51.4    36.5         34.9    18.1          142.1*   73.9
//   the same, 8 waves       23.0    12.8        56.1    29.2         42.7    19.7          167.9    75.2
//   192 x 128               24.5    17.4        59.1    41.4         31.0    17.3*         163.6    87.8
//   128 x 256, 3 stages     22.8    15.2        53.3    36.4         36.2    19.9          138.6    75.6
//   256 x 256                 --    15.9          --    37.6           --    27.4             --    63.3*
struct Fp8Times { float base, tile, block, way; };          // a launch; a tile's ends; a tile's block; a block's way
struct Fp8Shape { int bs, bt, together; Fp8Times t[3]; };   // fp32; bf16: W tiles, W rows; 0: not built
constexpr int FP8_SHAPES = 10;
static const Fp8Shape fp8_shapes[FP8_SHAPES] = {
    {64, 64, 1, {{1.75f, 2.88f, 0.37f, 0}, {1.76f, 2.45f, 0.215f, 0}, {1.6f, 2.3f, 0.23f, 0}}},               // two groups
    {64, 64, 5, {{3.33f, 0.56f, 0.32f, 0.74f}, {3.4f, 0.24f, 0.20f, 0.49f}, {3.0f, 0.25f, 0.22f, 0.65f}}},    // one stage
    {64, 64, 4, {{3.54f, 0.66f, 0.31f, 0.49f}, {2.9f, 0.54f, 0.19f, 0.37f}, {2.93f, 0.47f, 0.205f, 0.38f}}},  // two stages
    {128, 64, 1, {{}, {1.62f, 3.67f, 0.31f, 0}, {1.44f, 3.78f, 0.35f, 0}}},                                   // two groups
    {128, 64, 3, {{3.52f, 1.43f, 0.54f, 0.73f}, {}, {}}},                                                     // two stages
    {128, 128, 1, {{}, {1.21f, 3.90f, 0.48f, 0}, {}}},                                                        // four stages
    {128, 128, 2, {{3.56f, 3.09f, 0.92f, 1.09f}, {3.12f, 1.77f, 0.49f, 0.52f}, {2.8f, 1.76f, 0.57f, 0.64f}}}, // two stages; bf16: 8 waves
    {192, 128, 1, {{}, {0.39f, 5.09f, 0.72f, 0}, {0.32f, 5.9f, 0.86f, 0}}},
    {192, 256, 1, {{}, {0.0f, 8.2f, 1.04f, 0}, {0.0f, 8.3f, 1.3f, 0}}},
    {256, 256, 1, {{}, {0.0f, 12.0f, 1.25f, 0}, {}}}};

inline int fp8_type(const Fp8Size& a) { return !a.bf16 ? 0 : a.w_tiles ? 1 : 2; }
inline int64_t fp8_tiles(const Fp8Shape& s, const Fp8Size& a) { return (int64_t)((a.S + s.bs - 1) / s.bs) * ((a.T + s.bt - 1) / s.bt); }

inline float fp8_estimate(const Fp8Shape& s, const Fp8Times& t, int64_t tiles, int kb) {
    const int64_t m = (tiles + 255) / 256;
    const float work = (float)m * t.block, way = (float)((m + s.together - 1) / s.together) * t.way;
    return t.base + (float)m * t.tile + (float)kb * (work > way ? work : way);
}

inline float fp8_estimate(int shape, const Fp8Size& a) {
    const Fp8Shape& s = fp8_shapes[shape];
    return fp8_estimate(s, s.t[fp8_type(a)], fp8_tiles(s, a), a.kb);
}

// Two groups add their sums in an order of their own; the other shapes have the same bits.
inline bool fp8_grouped(int shape) { return shape == 0 || shape == 3; }

// Two groups from twelve blocks on: at nine they gain 0.2 to 0.5 us (512 x 512 x 1152: 6.1 against 6.3, fp32 7.5 against 8.0), and a layer's two
// gradients, one of them of few blocks, then rarely have a launch in common (256 x 1024 x 1024 with the quantiser: 14.9 us apart, 12.3 together).
inline int fp8_tile_shape(const Fp8Size& a) {
    int best = -1;
    for (int k = 0; k < FP8_SHAPES; ++k) {
        if (fp8_shapes[k].t[fp8_type(a)].block == 0.0f || (fp8_grouped(k) && a.kb < 12)) continue;
        if (best < 0 || fp8_estimate(k, a) < fp8_estimate(best, a)) best = k;
    }
    return best;
}

// Two products in one launch of 64 x 64 tiles, of two groups or of two stages: where neither result changes by it and that takes less time
// than two launches.  0: not.
inline int fp8_pairs(const Fp8Size& a, const Fp8Size& b) {
    if (!a.bf16 || !a.w_tiles || b.bf16 || b.w_tiles) return 0;
    const int sa = fp8_tile_shape(a), sb = fp8_tile_shape(b);
    if (fp8_grouped(sa) != fp8_grouped(sb)) return 0;
    const Fp8Shape& s = fp8_shapes[fp8_grouped(sa) ? 0 : 2];
    const int64_t tiles = fp8_tiles(s, a) + fp8_tiles(s, b);
    const float ea = fp8_estimate(s, s.t[1], tiles, a.kb), eb = fp8_estimate(s, s.t[0], tiles, b.kb);
    return (ea > eb ? ea : eb) < fp8_estimate(sa, a) + fp8_estimate(sb, b) ? 2 - fp8_grouped(sa) : 0;
}

// Two blocks requested at a time: with four, 16 x 512 x 1152 takes 6.1 us instead of 4.4 (what is requested behind the last block is
// fetched for nothing) and 4 x 4096 x 11008 16.0 instead of 14.7.  16 waves where they get two blocks each: 1 x 4096 x 4096 6.3 us against
// 6.9, 2 x 11008 x 4096 12.0 against 12.7.  More rows of X in a workgroup never pay: 32 x 512 x 1152 5.3 us with 32 of them, 4.4 with 16.
inline int fp8_split_waves(int kb) { return kb >= 32 ? 16 : 8; }

// Microseconds with 16 ms rows of W in a workgroup, fitted to 23 sizes of 1 x 512 x 1152 to 32 x 28672 x 4096 and 64 x 8 x 4096 to 16384 x 32 x
// 11008 whose weights come from memory: what the workgroups read (10 TB/s, mostly out of caches; as if the last round of CUs were full), their
// number, and a wave's way through its blocks.  Two tiles of W share X's reads: 32 x 4096 x 4096 9.4 us against 11.2, 1 x 4096 x 4096 7.9
// against 6.3.
inline float fp8_split_estimate(const Fp8Size& a, int ms) {
    static const float c[2][5] = {{2.2f, 0.112f, 0.096f, 0.82f, 0.039f}, {2.9f, 0.010f, 0.120f, 0.36f, 0.071f}};
    const float* k = c[ms - 1];
    const int waves = fp8_split_waves(a.kb);
    const int64_t n = (int64_t)((a.S + 16 * ms - 1) / (16 * ms)) * ((a.T + 15) / 16);
    const float mb = (float)a.kb * 128e-6f * (float)((a.S < 16 * ms ? a.S : 16 * ms) + (a.T < 16 ? a.T : 16)), all = k[1] * (float)n * mb, rounds = k[2] * (float)((n + 255) / 256 * 256) * mb;
    return k[0] + (all > rounds ? all : rounds) + k[3] * (float)((a.kb + 2 * waves - 1) / (2 * waves)) + k[4] * (float)waves * (float)n / 256.0f;
}

inline float fp8_split_time(const Fp8Size& a) {
    const float one = fp8_split_estimate(a, 1), two = fp8_split_estimate(a, 2);
    return one < two ? one : two;
}

// Blocks of X that a workgroup of fp8_split_kernel quantises for itself.  Its 512 or 1024 threads take 32 or 64 of them in
// 0.2 us; a launch of the quantiser's own costs 2 us more on the GPU and 3 on the host.
constexpr int FP8_OWN_BLOCKS = 128;
inline bool fp8_takes_raw(int64_t T, int64_t kb) { return T <= 16 && T * kb <= FP8_OWN_BLOCKS; }

// Whether the product of T x K and S x K may run without staging; ld: the larger row stride.
inline bool fp8_may_split(int64_t T, int64_t S, int64_t ld) { return T <= 32 || S <= 32 || ld >= 1 << 24; }

// Few rows of X or of W: no staging, the waves split the contraction - but where many rows of the other one fill the CUs with tiles (32 x 28672 x
// 4096, us: 28 against 45; 32 x 4096 x 11008: 27 against 22; 16384 x 32 x 4096: 14 against 20).  The tiled kernel's estimate is for
// operands in the caches; from memory bf16 results take 1.1 times as long (fp32, bound by the widening, 0.95), and no less than the reads at
// 4.3 TB/s.  What one launch could have done
// together with the quantiser is summed in that launch's order.  The tiled kernels' offsets inside a tile are 32 bits.
inline bool fp8_takes_split(const Fp8Size& a, int64_t ld) {
    if (!fp8_may_split(a.T, a.S, ld)) return false;
    if (ld >= 1 << 24 || fp8_takes_raw(a.T, a.kb)) return true;
    const float tiled = (a.bf16 ? 1.1f : 0.95f) * fp8_estimate(fp8_tile_shape(a), a), read = 2.0f + ((float)a.T + (float)a.S) * (float)a.kb * (128e-6f / 4.3f);
    return fp8_split_time(a) < (tiled > read ? tiled : read);
}

}  // namespace crisp
