// What the 8-bit kernels share: a block's scale, conversions of eight values at a time, reductions over 16 lanes.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace crisp {

constexpr int FP8_BLOCK = 128;              // columns (or elements) that share a scale
constexpr float FP8_MAX = 448.0f;           // largest e4m3 value
constexpr float FP8_LEAST_SCALE = 0x1p-126f;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// Scale of a block whose largest magnitude is amax.  amax is compared as an integer everywhere, so that a NaN is larger than
// any number and reaches this place; the comparison below lets it through.
__device__ __forceinline__ float fp8_scale(float amax) {
    const float s = amax / FP8_MAX;
    return s < FP8_LEAST_SCALE ? FP8_LEAST_SCALE : s;
}

__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }

// Largest of a value over the 16 lanes of a DPP row, in every lane: four rotations inside the row.
__device__ __forceinline__ uint32_t max16(uint32_t x) {
    x = umax(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, false));  // row_ror:8
    x = umax(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x124, 0xf, 0xf, false));  // row_ror:4
    x = umax(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x122, 0xf, 0xf, false));  // row_ror:2
    x = umax(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x121, 0xf, 0xf, false));  // row_ror:1
    return x;
}

// Eight fp32 values to eight e4m3 codes, to nearest even; |x| <= 448 up to one rounding, or NaN.
__device__ __forceinline__ uint2 to_fp8x8(const float (&x)[8]) {
    int a = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    a = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], a, true);
    int b = __builtin_amdgcn_cvt_pk_fp8_f32(x[4], x[5], 0, false);
    b = __builtin_amdgcn_cvt_pk_fp8_f32(x[6], x[7], b, true);
    return make_uint2((uint32_t)a, (uint32_t)b);
}

__device__ __forceinline__ void from_fp8x8(uint2 q, float (&x)[8]) {
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)q.x, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)q.x, true);
    const auto c = __builtin_amdgcn_cvt_pk_f32_fp8((int)q.y, false), d = __builtin_amdgcn_cvt_pk_f32_fp8((int)q.y, true);
    x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1];
    x[4] = c[0]; x[5] = c[1]; x[6] = d[0]; x[7] = d[1];
}

__device__ __forceinline__ void from_bf16x8(uint4 q, float (&x)[8]) {
    x[0] = __uint_as_float(q.x << 16); x[1] = __uint_as_float(q.x & 0xffff0000u);
    x[2] = __uint_as_float(q.y << 16); x[3] = __uint_as_float(q.y & 0xffff0000u);
    x[4] = __uint_as_float(q.z << 16); x[5] = __uint_as_float(q.z & 0xffff0000u);
    x[6] = __uint_as_float(q.w << 16); x[7] = __uint_as_float(q.w & 0xffff0000u);
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Two fp32 values to bf16, to nearest even (one v_cvt_pk_bf16_f32).
__device__ __forceinline__ uint32_t to_bf16x2(float a, float b) {
    const bf16x2 p = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, p);
}
__device__ __forceinline__ uint16_t to_bf16(float a) { return __builtin_bit_cast(uint16_t, (__bf16)a); }

// Vectors at any address: the hardware takes them in one request also where they are not aligned.
typedef uint32_t loose_u32x2 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t loose_u32x4 __attribute__((ext_vector_type(4), aligned(2)));
typedef float loose_f32x4 __attribute__((ext_vector_type(4), aligned(2)));

// C (four or eight) elements of a row as they lie in memory, from column c on; columns at or behind `cols` are zeros.
template <bool BF16, int C>
struct Elements {
    static constexpr int WORDS = BF16 ? C / 2 : C;
    uint32_t w[WORDS];

    // cols >= C: of the row's last C elements where the wanted ones end behind it, so that every lane makes the same request and
    // those of several rows are under way together.  settle() then moves them to their places.
    __device__ __forceinline__ void request(const void* X, int64_t row_at, int64_t c, int64_t cols) {
        const int64_t at = row_at + (c < cols - C ? c : cols - C);
        const uint8_t* p = static_cast<const uint8_t*>(X) + at * (BF16 ? 2 : 4);
        if constexpr (WORDS == 2) {
            const loose_u32x2 v = *reinterpret_cast<const loose_u32x2*>(p);
            w[0] = v[0]; w[1] = v[1];
        } else {
#pragma unroll
            for (int k = 0; k < WORDS; k += 4) {
                const loose_u32x4 v = *reinterpret_cast<const loose_u32x4*>(p + k * 4);
#pragma unroll
                for (int j = 0; j < 4; ++j) w[k + j] = v[j];
            }
        }
    }

    __device__ __forceinline__ void settle(int64_t c, int64_t cols) {
        int64_t ahead = c - (cols - C);      // elements before the wanted ones
        for (ahead = ahead < C ? ahead : C; ahead > 0; --ahead) {
#pragma unroll
            for (int j = 0; j < WORDS; ++j) {
                const uint32_t next = j + 1 < WORDS ? w[j + 1] : 0;
                w[j] = BF16 ? w[j] >> 16 | next << 16 : next;
            }
        }
    }

    // cols < C: one by one.
    __device__ __forceinline__ void gather(const void* X, int64_t row_at, int64_t c, int64_t cols) {
#pragma unroll
        for (int j = 0; j < WORDS; ++j) w[j] = 0;
#pragma unroll
        for (int j = 0; j < C - 1; ++j)
            if (c + j < cols) {
                if constexpr (BF16) w[j / 2] |= (uint32_t)static_cast<const uint16_t*>(X)[row_at + c + j] << (j % 2 * 16);
                else w[j] = static_cast<const uint32_t*>(X)[row_at + c + j];
            }
    }

    // bit j of `bits`: whether element j stays, else zero
    __device__ __forceinline__ void keep(uint32_t bits) {
#pragma unroll
        for (int j = 0; j < WORDS; ++j) {
            if constexpr (BF16) w[j] &= ((bits >> (2 * j) & 1) ? 0xffffu : 0u) | ((bits >> (2 * j + 1) & 1) ? 0xffff0000u : 0u);
            else w[j] = bits >> j & 1 ? w[j] : 0u;
        }
    }

    __device__ __forceinline__ float operator[](int j) const {
        if constexpr (BF16) return __uint_as_float(j % 2 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
        else return __uint_as_float(w[j]);
    }
};

// Elements c, c + 1, ... of N rows, all requested before any is used; row_at: where a row starts.
template <int N, bool BF16, int C, typename At>
__device__ __forceinline__ void read_rows(Elements<BF16, C> (&x)[N], const void* X, int64_t c, int64_t cols, At row_at) {
    if (cols >= C) {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i].request(X, row_at(i), c, cols);
        if (c > cols - C) {
#pragma unroll
            for (int i = 0; i < N; ++i) x[i].settle(c, cols);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i].gather(X, row_at(i), c, cols);
    }
}

// 16 lanes' block of 128 elements, eight each: its codes and its scale.
__device__ __forceinline__ uint2 quantize_block(float (&x)[8], float& scale) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = umax(top, abs_bits(x[j]));
    scale = fp8_scale(__uint_as_float(max16(top)));
    const float inv = 1.0f / scale;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] *= inv;
    return to_fp8x8(x);
}

}  // namespace crisp
