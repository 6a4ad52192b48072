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

// Eight elements of a row from column c on; what lies at or behind `cols` counts as zero.  vec: the address is a multiple of
// 16 bytes wherever c is a multiple of 8.
template <bool BF16>
__device__ __forceinline__ void load8(const void* X, int64_t at, int64_t left, bool vec, float (&x)[8]) {
    if (vec && left >= 8) {
        if constexpr (BF16) {
            from_bf16x8(*reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(X) + at), x);
        } else {
            const f32x4 a = *reinterpret_cast<const f32x4*>(static_cast<const float*>(X) + at);
            const f32x4 b = *reinterpret_cast<const f32x4*>(static_cast<const float*>(X) + at + 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) { x[j] = a[j]; x[4 + j] = b[j]; }
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        x[j] = 0.0f;
        if (j < left) {
            if constexpr (BF16) x[j] = __uint_as_float((uint32_t)static_cast<const uint16_t*>(X)[at + j] << 16);
            else x[j] = static_cast<const float*>(X)[at + j];
        }
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
