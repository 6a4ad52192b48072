// One AdamW step over many tensors, and the bit mask of the hybrid pattern.  Both are bound by memory: every element is
// read and written once, the arithmetic of the step (two roots' worth of it) hides behind that.
#include "crisp_adamw.h"
#include "crisp_internal.h"
#include "fp8_common.h"
#include "select_layer.h"

namespace crisp {

constexpr int ADAMW_CAP = 40;            // tensors per launch: they travel in the kernel's arguments, 3.7 of 4 KB
constexpr int ADAMW_THREADS = 256;
constexpr int ADAMW_PASS = ADAMW_THREADS * 8;   // elements that a workgroup takes at a time
constexpr int ADAMW_PASSES = 4;          // passes of a workgroup where the tensors have work for all CUs (then fewer look for their
                                         // tensor), else one: 10 tensors of 37 000 elements 10.2 us with four

// fp32 scalars of a step, rounded from fp64.
struct AdamwScalars { float b1, c1, b2, c2, gs, root, eps, step_size; double lr; };

__host__ __device__ inline double power(double base, int64_t n) {
    double r = 1.0;
    for (; n > 0; n >>= 1, base *= base)
        if (n & 1) r *= base;
    return r;
}

__host__ __device__ inline AdamwScalars adamw_scalars(double lr, double beta1, double beta2, double eps, double gs, int64_t step) {
    AdamwScalars s;
    s.b1 = (float)beta1; s.c1 = (float)(1.0 - beta1);
    s.b2 = (float)beta2; s.c2 = (float)(1.0 - beta2);
    s.gs = (float)gs; s.eps = (float)eps;
    s.root = (float)(1.0 / sqrt(1.0 - power(beta2, step)));
    s.step_size = (float)(lr / (1.0 - power(beta1, step)));
    s.lr = lr;
    return s;
}

struct AdamwTensor {
    void* w; const void* g; void *m, *v;
    float *ms, *vs;
    uint16_t* copy;
    const uint32_t* mask;
    int64_t numel;
    int32_t row_len;
    float decay;
};

struct AdamwArgs {
    AdamwScalars s;
    double beta1, beta2;
    const crisp_adamw_live* live;
    int n, passes;
    int first[ADAMW_CAP + 1];            // first workgroup of each tensor
    AdamwTensor t[ADAMW_CAP];
};
static_assert(sizeof(AdamwArgs) <= 4096, "kernel arguments");

// Keep bits of elements e .. e+7 of a masked tensor; bits of elements that are not there (n of eight are) are clear.  Eight elements of
// rows of any length lie in two words of a row and the first of the next one, requested together.
__device__ __forceinline__ uint32_t keep_bits(const AdamwTensor& t, int64_t e, int n) {
    const uint32_t K = (uint32_t)t.row_len, words = (K + 31) / 32;
    uint32_t row = (uint32_t)e / K, col = (uint32_t)e - row * K;
    const uint32_t* m = t.mask + (int64_t)row * words;
    uint32_t bits = 0;
    if (K % 8 == 0) {
        bits = m[col / 32] >> (col % 32) & 0xffu;
    } else if (K >= 8) {
        const uint32_t here = min(8u, K - col);                  // (the last word of a row holds all that is left of it)
        const uint32_t lo = m[col / 32], hi = m[min(col / 32 + 1, words - 1)], next = m[(uint32_t)n > here ? words : col / 32];
        bits = ((uint32_t)(((uint64_t)hi << 32 | lo) >> (col % 32)) & ((1u << here) - 1u)) | next << here;
    } else {
        for (int j = 0; j < n; ++j) {
            bits |= (t.mask[(int64_t)row * words + col / 32] >> (col % 32) & 1u) << j;
            if (++col == K) { col = 0; ++row; }
        }
    }
    return bits & ((1u << n) - 1u);
}

// A thread takes eight consecutive elements, 16 of them a block of 8-bit moments, whose largest magnitudes they exchange in registers.
// Eight elements that are all pruned cost their moments' zeros alone.  0.82 G parameters in bf16 with 8-bit moments 1.64 ms (8.35 GB,
// 5.1 TB/s; a copy reaches 4.9), 155 M in fp32 with bf16 gradients and copy, pruned 2:4 in 60 % of the blocks, 0.66 ms: the lines that hold a kept
// element are 3.1 GB (4.7 TB/s), the kept elements alone 2.2.
template <bool W32, bool G32, bool M8>
__global__ __launch_bounds__(ADAMW_THREADS) void adamw_kernel(AdamwArgs a) {
    const int which = layer_by_ballots<ADAMW_THREADS, ADAMW_CAP>(a.n, a.first, (int)blockIdx.x, [](auto p) {
        return __ballot(p((int)(threadIdx.x % 64)));
    });
    const AdamwTensor& t = a.t[which];
    AdamwScalars s = a.s;
    if (a.live) {
        if (a.live->skip) return;
        s = adamw_scalars(a.live->lr, a.beta1, a.beta2, 0.0, a.live->grad_scale, max(a.live->step, 1));
        s.eps = a.s.eps;
    }
    const float decay = (float)(1.0 - s.lr * (double)t.decay);
    const int64_t base = (int64_t)(blockIdx.x - a.first[which]) * (ADAMW_PASS * a.passes) + threadIdx.x * 8;
#pragma unroll 1
    for (int k = 0; k < a.passes; ++k) {
        const int64_t e = base + k * ADAMW_PASS;
        const int64_t left = t.numel - e;
        const int n = left >= 8 ? 8 : left > 0 ? (int)left : 0;
        // 16 lanes share a block of 128 elements: they go on as long as one of them has an element
        if (M8 ? e / FP8_BLOCK * FP8_BLOCK >= t.numel : n == 0) break;
        const uint32_t keep = t.mask && n ? keep_bits(t, e, n) : (1u << n) - 1u;
        // eight threads' weights in bf16 are a line of 128 bytes: all of it leaves, or nothing (a part has to be merged in memory:
        // 78 M pruned parameters in fp32 with rows of 1022, whose blocks begin inside lines, 464 us against 395)
        const bool line = __ballot(keep != 0) >> (threadIdx.x % 64 / 8 * 8) & 0xffu;
        float w[8] = {}, g[8] = {}, m[8] = {}, v[8] = {};
        if (line && n == 8) {
            if constexpr (W32) {
                const f32x4 x = *reinterpret_cast<const f32x4*>(static_cast<float*>(t.w) + e), y = *reinterpret_cast<const f32x4*>(static_cast<float*>(t.w) + e + 4);
#pragma unroll
                for (int j = 0; j < 4; ++j) { w[j] = x[j]; w[4 + j] = y[j]; }
            } else {
                from_bf16x8(*reinterpret_cast<const uint4*>(static_cast<uint16_t*>(t.w) + e), w);
            }
        }
        if (keep) {
            if constexpr (M8) {
                const float ms = t.ms[e / FP8_BLOCK], vs = t.vs[e / FP8_BLOCK];
                uint2 qm = {}, qv = {};
                if (n == 8) {
                    qm = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(t.m) + e);
                    qv = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(t.v) + e);
                } else {
                    for (int j = 0; j < n; ++j) {
                        const uint32_t x = static_cast<const uint8_t*>(t.m)[e + j], y = static_cast<const uint8_t*>(t.v)[e + j];
                        (j < 4 ? qm.x : qm.y) |= x << (8 * (j & 3));
                        (j < 4 ? qv.x : qv.y) |= y << (8 * (j & 3));
                    }
                }
                from_fp8x8(qm, m);
                from_fp8x8(qv, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) { m[j] *= ms; v[j] *= vs; v[j] *= v[j]; }
            }
            if (n == 8) {
                if constexpr (G32) {
                    const f32x4 x = *reinterpret_cast<const f32x4*>(static_cast<const float*>(t.g) + e), y = *reinterpret_cast<const f32x4*>(static_cast<const float*>(t.g) + e + 4);
#pragma unroll
                    for (int j = 0; j < 4; ++j) { g[j] = x[j]; g[4 + j] = y[j]; }
                } else {
                    from_bf16x8(*reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(t.g) + e), g);
                }
                if constexpr (!M8) {
                    const float *pm = static_cast<float*>(t.m) + e, *pv = static_cast<float*>(t.v) + e;
                    const f32x4 x = *reinterpret_cast<const f32x4*>(pm), y = *reinterpret_cast<const f32x4*>(pm + 4);
                    const f32x4 p = *reinterpret_cast<const f32x4*>(pv), q = *reinterpret_cast<const f32x4*>(pv + 4);
#pragma unroll
                    for (int j = 0; j < 4; ++j) { m[j] = x[j]; m[4 + j] = y[j]; v[j] = p[j]; v[4 + j] = q[j]; }
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if (j >= n) break;
                    if constexpr (W32) w[j] = static_cast<float*>(t.w)[e + j];
                    else w[j] = bf16_bits_to_float(static_cast<uint16_t*>(t.w)[e + j]);
                    if constexpr (G32) g[j] = static_cast<const float*>(t.g)[e + j];
                    else g[j] = bf16_bits_to_float(static_cast<const uint16_t*>(t.g)[e + j]);
                    if constexpr (!M8) { m[j] = static_cast<float*>(t.m)[e + j]; v[j] = static_cast<float*>(t.v)[e + j]; }
                }
            }
        }
        float u[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool kept = keep >> j & 1u;
            const float gj = g[j] * s.gs;
            const float mj = s.b1 * m[j] + s.c1 * gj, vj = s.b2 * v[j] + s.c2 * (gj * gj);
            u[j] = sqrtf(vj);
            const float up = mj / (u[j] * s.root + s.eps);
            const float nw = w[j] * decay - s.step_size * up;
            w[j] = kept ? nw : w[j];
            m[j] = kept ? mj : 0.0f;
            v[j] = kept ? vj : 0.0f;
            u[j] = kept ? u[j] : 0.0f;
        }
        if constexpr (M8) {
            uint32_t tm = 0, tu = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) { tm = umax(tm, abs_bits(m[j])); tu = umax(tu, abs_bits(u[j])); }
            const float ms = fp8_scale(__uint_as_float(max16(tm))), vs = fp8_scale(__uint_as_float(max16(tu)));
            const float im = 1.0f / ms, iv = 1.0f / vs;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                m[j] *= im;
                const float q = u[j] * iv;
                v[j] = u[j] > 0.0f && q < 0x1p-9f ? 0x1p-9f : q;
            }
            const uint2 qm = to_fp8x8(m), qv = to_fp8x8(v);
            if (threadIdx.x % 16 == 0) { t.ms[e / FP8_BLOCK] = ms; t.vs[e / FP8_BLOCK] = vs; }
            if (n == 8) {
                *reinterpret_cast<uint2*>(static_cast<uint8_t*>(t.m) + e) = qm;
                *reinterpret_cast<uint2*>(static_cast<uint8_t*>(t.v) + e) = qv;
            } else {
                for (int j = 0; j < n; ++j) {
                    static_cast<uint8_t*>(t.m)[e + j] = (uint8_t)((j < 4 ? qm.x : qm.y) >> (8 * (j & 3)));
                    static_cast<uint8_t*>(t.v)[e + j] = (uint8_t)((j < 4 ? qv.x : qv.y) >> (8 * (j & 3)));
                }
            }
        }
        if (n == 8) {
            if constexpr (!M8) {
                float *pm = static_cast<float*>(t.m) + e, *pv = static_cast<float*>(t.v) + e;
                *reinterpret_cast<f32x4*>(pm) = f32x4{m[0], m[1], m[2], m[3]};
                *reinterpret_cast<f32x4*>(pm + 4) = f32x4{m[4], m[5], m[6], m[7]};
                *reinterpret_cast<f32x4*>(pv) = f32x4{v[0], v[1], v[2], v[3]};
                *reinterpret_cast<f32x4*>(pv + 4) = f32x4{v[4], v[5], v[6], v[7]};
            }
            if (line) {
                const uint4 b = {to_bf16x2(w[0], w[1]), to_bf16x2(w[2], w[3]), to_bf16x2(w[4], w[5]), to_bf16x2(w[6], w[7])};
                if constexpr (W32) {
                    float* pw = static_cast<float*>(t.w) + e;
                    *reinterpret_cast<f32x4*>(pw) = f32x4{w[0], w[1], w[2], w[3]};
                    *reinterpret_cast<f32x4*>(pw + 4) = f32x4{w[4], w[5], w[6], w[7]};
                    if (t.copy) *reinterpret_cast<uint4*>(t.copy + e) = b;
                } else {
                    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(t.w) + e) = b;
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (j >= n) break;
                if constexpr (!M8) { static_cast<float*>(t.m)[e + j] = m[j]; static_cast<float*>(t.v)[e + j] = v[j]; }
                if (!(keep >> j & 1u)) continue;
                if constexpr (W32) {
                    static_cast<float*>(t.w)[e + j] = w[j];
                    if (t.copy) t.copy[e + j] = to_bf16(w[j]);
                } else {
                    static_cast<uint16_t*>(t.w)[e + j] = to_bf16(w[j]);
                }
            }
        }
    }
}

typedef void (*AdamwKernel)(AdamwArgs);

// 4: weights in fp32, 2: gradients in fp32, 1: moments in 8 bits
static int types_of(const crisp_adamw_tensor& t) {
    return (t.w_type == CRISP_P_F32) * 4 + (t.g_type == CRISP_P_F32) * 2 + (t.moments == CRISP_MOMENTS_8);
}
static const AdamwKernel ADAMW_KERNELS[8] = {adamw_kernel<false, false, false>, adamw_kernel<false, false, true>, adamw_kernel<false, true, false>,
                                             adamw_kernel<false, true, true>,   adamw_kernel<true, false, false>, adamw_kernel<true, false, true>,
                                             adamw_kernel<true, true, false>,   adamw_kernel<true, true, true>};

static bool off16(const void* p) { return ((uintptr_t)p & 15) != 0; }
static bool off4(const void* p) { return ((uintptr_t)p & 3) != 0; }

static crisp_status check_tensor(const crisp_adamw_tensor& t) {
    if ((t.w_type != CRISP_P_F32 && t.w_type != CRISP_P_BF16) || (t.g_type != CRISP_P_F32 && t.g_type != CRISP_P_BF16) ||
        (t.moments != CRISP_MOMENTS_32 && t.moments != CRISP_MOMENTS_8))
        return CRISP_EINVAL;
    if (!(t.weight_decay >= 0.0f) || t.weight_decay > 1e30f) return CRISP_EINVAL;
    if (t.numel < 0 || t.numel > (int64_t)(ADAMW_PASS * ADAMW_PASSES) << 22) return CRISP_ESHAPE;
    if (t.numel == 0) return CRISP_OK;
    if (!t.w || !t.g || !t.m || !t.v) return CRISP_EINVAL;
    if (t.moments == CRISP_MOMENTS_8 ? !t.m_scale || !t.v_scale : t.m_scale || t.v_scale) return CRISP_EINVAL;
    if (t.w_copy && t.w_type != CRISP_P_F32) return CRISP_EINVAL;
    if (t.mask && (t.row_len < 1 || t.numel >= (int64_t)1 << 31 || t.numel % t.row_len)) return CRISP_ESHAPE;
    if (off16(t.w) || off16(t.g) || off16(t.m) || off16(t.v) || off16(t.w_copy) || off4(t.m_scale) || off4(t.v_scale) || off4(t.mask))
        return CRISP_EALIGN;
    return CRISP_OK;
}

// A word of the mask per thread: the kept blocks of its block-row are ascending, so each is found by halving the list.
__global__ __launch_bounds__(256) void hybrid_mask_kernel(int S, int mwpr, int log2b, int nk, const uint32_t* nm_mask,
                                                          const int32_t* __restrict__ row_ptr,
                                                          const int32_t* __restrict__ col_idx, uint32_t* mask) {
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (id >= (int64_t)S * mwpr) return;
    const int s = (int)(id / mwpr), word = (int)(id - (int64_t)s * mwpr);
    const int from = max(row_ptr[s >> log2b], 0), to = min(row_ptr[(s >> log2b) + 1], nk);
    uint32_t keep = 0;
    for (int part = 0; part < (log2b == 4 ? 2 : 1); ++part) {
        const int block = (word * 32 + part * 16) >> log2b;
        int lo = from, hi = to;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (col_idx[mid] < block) lo = mid + 1; else hi = mid;
        }
        if (lo < to && col_idx[lo] == block) keep |= log2b == 4 ? 0xffffu << (16 * part) : 0xffffffffu;
    }
    mask[id] = nm_mask[id] & keep;
}

}  // namespace crisp

using namespace crisp;

extern "C" {

crisp_status crisp_adamw_batch(int32_t n_tensors, const crisp_adamw_tensor* tensors, const crisp_adamw_hyper* hyper, void* stream) {
    if (n_tensors < 1 || n_tensors > 1 << 20 || !tensors || !hyper) return CRISP_EINVAL;
    const crisp_adamw_hyper& h = *hyper;
    if (!(h.beta1 >= 0.0 && h.beta1 < 1.0) || !(h.beta2 >= 0.0 && h.beta2 < 1.0) || !((float)h.eps > 0.0f && h.eps <= 1e30)) return CRISP_EINVAL;
    if (!h.live) {
        if (!(h.lr >= 0.0 && h.lr <= 1e30) || !(h.grad_scale >= -1e30 && h.grad_scale <= 1e30)) return CRISP_EINVAL;
        if (h.step < 1 || h.step > INT32_MAX) return CRISP_EINVAL;
    }
    if (off4(h.live)) return CRISP_EALIGN;
    for (int32_t i = 0; i < n_tensors; ++i) {      // everything is checked before anything is enqueued
        const crisp_status st = check_tensor(tensors[i]);
        if (st != CRISP_OK) return st;
    }
    AdamwArgs a;
    a.s = h.live ? adamw_scalars(0.0, h.beta1, h.beta2, h.eps, 1.0, 1) : adamw_scalars(h.lr, h.beta1, h.beta2, h.eps, h.grad_scale, h.step);
    a.beta1 = h.beta1; a.beta2 = h.beta2; a.live = h.live;
    int64_t work[8] = {};                          // passes of each combination of types
    for (int32_t i = 0; i < n_tensors; ++i) work[types_of(tensors[i])] += (tensors[i].numel + ADAMW_PASS - 1) / ADAMW_PASS;
    for (int k = 0; k < 8; ++k) {                  // the tensors of one combination share launches
        a.n = 0;
        a.first[0] = 0;
        a.passes = work[k] >= 4 * ADAMW_PASSES * 256 ? ADAMW_PASSES : 1;
        const int64_t chunk = (int64_t)ADAMW_PASS * a.passes;
        for (int32_t i = 0; i <= n_tensors && work[k]; ++i) {
            const crisp_adamw_tensor* t = i < n_tensors ? &tensors[i] : nullptr;
            if (t && (t->numel == 0 || types_of(*t) != k)) continue;
            const int64_t chunks = t ? (t->numel + chunk - 1) / chunk : 0;
            if (a.n && (!t || a.n == ADAMW_CAP || a.first[a.n] + chunks > 1 << 23)) {
                ADAMW_KERNELS[k]<<<(unsigned)a.first[a.n], ADAMW_THREADS, 0, (hipStream_t)stream>>>(a);
                if (hipGetLastError() != hipSuccess) return CRISP_EDEVICE;
                a.n = 0;
            }
            if (!t) break;
            a.t[a.n] = AdamwTensor{t->w, t->g, t->m, t->v, t->m_scale, t->v_scale, t->w_copy, t->mask, t->numel, (int32_t)t->row_len, t->weight_decay};
            a.first[a.n + 1] = a.first[a.n] + (int)chunks;
            ++a.n;
        }
    }
    return CRISP_OK;
}

crisp_status crisp_hybrid_mask(const crisp_layer_desc* desc, const uint32_t* nm_mask, const int32_t* row_ptr, const int32_t* col_idx,
                               uint32_t* mask, void* stream) {
    Geometry g;
    const crisp_status st = make_geometry(desc, true, &g);
    if (st != CRISP_OK) return st;
    if (!nm_mask || !row_ptr || !col_idx || !mask) return CRISP_EINVAL;
    if (off4(nm_mask) || off4(row_ptr) || off4(col_idx) || off4(mask)) return CRISP_EALIGN;
    const int64_t groups = ((int64_t)g.S * g.mwpr + 255) / 256;
    if (groups >= 1 << 24) return CRISP_ESHAPE;      // a launch takes fewer than 2^32 threads
    hybrid_mask_kernel<<<(unsigned)groups, 256, 0, (hipStream_t)stream>>>(g.S, g.mwpr, g.B == 16 ? 4 : g.B == 32 ? 5 : 6, g.nk, nm_mask,
                                                                        row_ptr, col_idx, mask);
    return hipGetLastError() == hipSuccess ? CRISP_OK : CRISP_EDEVICE;
}

}  // extern "C"
