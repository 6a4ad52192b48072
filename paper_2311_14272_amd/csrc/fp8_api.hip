// C ABI of the 8-bit layers: argument checks on the host, then the launchers.
#include "fp8_common.h"
#include "fp8_internal.h"

namespace crisp {

static bool off(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

constexpr int64_t MOST = (int64_t)1 << 27;      // rows, columns
constexpr int64_t MOST_LD = (int64_t)1 << 30;   // leading dimensions

static int64_t blocks(int64_t n) { return (n + FP8_BLOCK - 1) / FP8_BLOCK; }

static crisp_status check_mat(const crisp_fp8_mat* m) {
    if (!m->q || !m->scale) return CRISP_EINVAL;
    if ((m->kind != CRISP_FP8_ROWS && m->kind != CRISP_FP8_TILES) || m->reserved != 0) return CRISP_EINVAL;
    if (m->rows < 1 || m->cols < 1 || m->rows > MOST || m->cols > MOST) return CRISP_ESHAPE;
    if (m->ld < blocks(m->cols) * FP8_BLOCK || m->ld > MOST_LD) return CRISP_ESHAPE;
    if (m->lds < (m->kind == CRISP_FP8_ROWS ? m->rows : blocks(m->cols)) || m->lds > MOST_LD) return CRISP_ESHAPE;
    if ((m->ld & 15) || off(m->q, 16) || off(m->scale, 4)) return CRISP_EALIGN;
    return CRISP_OK;
}

// A launch takes fewer than 2^32 threads: 16 of them for a block of 128 columns.
static bool too_many(int64_t rows, int64_t cols) { return rows * blocks(cols) > ((int64_t)1 << 28) - 16; }

static crisp_status check_out(const void* Y, int64_t T, int64_t S, int64_t most_ld, int64_t ldy, int32_t y_type, const crisp_epilogue* ep) {
    if (!Y) return CRISP_EINVAL;
    if (y_type != CRISP_Y_F32 && y_type != CRISP_Y_BF16) return CRISP_EINVAL;
    if (ldy < S || ldy > MOST_LD) return CRISP_ESHAPE;
    const size_t size = y_type == CRISP_Y_BF16 ? 2 : 4;
    if (off(Y, size)) return CRISP_EALIGN;
    // a launch takes fewer than 2^32 threads: up to 1024 for 16 x 16 results, or 512 for 64 x 64
    const int64_t tiles = ((T + 15) / 16) * ((S + 15) / 16);
    if (tiles > (fp8_may_split(T, S, most_ld) ? ((int64_t)1 << 22) - 1 : ((int64_t)1 << 26))) return CRISP_ESHAPE;
    if (!ep) return CRISP_OK;
    if (ep->relu != 0 && ep->relu != 1) return CRISP_EINVAL;
    if (ep->residual && (ep->ldr < S || ep->ldr > MOST_LD)) return CRISP_ESHAPE;
    if (ep->residual == Y && ep->ldr != ldy) return CRISP_ESHAPE;
    if (off(ep->scale, 4) || off(ep->bias, 4) || off(ep->residual, size)) return CRISP_EALIGN;
    return CRISP_OK;
}

static crisp_status check_in(const void* X, int32_t in_type, int64_t rows, int64_t cols, int64_t ldx) {
    if (!X || (in_type != CRISP_IN_F32 && in_type != CRISP_IN_BF16)) return CRISP_EINVAL;
    if (rows < 1 || cols < 1 || rows > MOST || cols > MOST || ldx < cols || ldx > MOST_LD || too_many(rows, cols)) return CRISP_ESHAPE;
    if (off(X, in_type == CRISP_IN_BF16 ? 2 : 4)) return CRISP_EALIGN;
    return CRISP_OK;
}

}  // namespace crisp

using namespace crisp;

extern "C" {

crisp_status crisp_fp8_quant(const void* X, int32_t in_type, int64_t rows, int64_t cols, int64_t ldx, const uint32_t* mask,
                             const crisp_fp8_mat* Q, const crisp_fp8_mat* Qt, void* stream) {
    if (!Q && !Qt) return CRISP_EINVAL;
    crisp_status st = check_in(X, in_type, rows, cols, ldx);
    if (st != CRISP_OK) return st;
    if (Q && (st = check_mat(Q)) != CRISP_OK) return st;
    if (Qt && (st = check_mat(Qt)) != CRISP_OK) return st;
    if (Q && Qt && Q->kind != Qt->kind) return CRISP_EINVAL;
    if ((Q && (Q->rows != rows || Q->cols != cols)) || (Qt && (Qt->rows != cols || Qt->cols != rows))) return CRISP_ESHAPE;
    if (off(mask, 4)) return CRISP_EALIGN;
    if (Q && Qt && (Q->q == Qt->q || Q->scale == Qt->scale)) return CRISP_EINVAL;
    return launch_fp8_quant(X, in_type, rows, cols, ldx, mask, Q, Qt, (hipStream_t)stream) == hipSuccess ? CRISP_OK : CRISP_EDEVICE;
}

crisp_status crisp_fp8_product(const crisp_fp8_mat* X, const crisp_fp8_mat* W, void* Y, int64_t ldy, int32_t y_type,
                               const crisp_epilogue* ep, void* stream) {
    if (!X || !W) return CRISP_EINVAL;
    crisp_status st = check_mat(X);
    if (st != CRISP_OK || (st = check_mat(W)) != CRISP_OK) return st;
    if (X->kind != CRISP_FP8_ROWS) return CRISP_EINVAL;
    if (X->cols != W->cols) return CRISP_ESHAPE;
    if ((st = check_out(Y, X->rows, W->rows, X->ld > W->ld ? X->ld : W->ld, ldy, y_type, ep)) != CRISP_OK) return st;
    return launch_fp8_product(*X, *W, Y, ldy, y_type, ep, (hipStream_t)stream) == hipSuccess ? CRISP_OK : CRISP_EDEVICE;
}

size_t crisp_fp8_linear_ws(int64_t T, int64_t K) {
    if (T < 1 || K < 1 || T > MOST || K > MOST || too_many(T, K) || fp8_takes_raw(T, blocks(K))) return 0;
    return (size_t)T * blocks(K) * (FP8_BLOCK + sizeof(float));
}

// A matrix in ROWS inside a workspace, codes first.
static crisp_fp8_mat mat_in(void* ws, int64_t rows, int64_t cols) {
    const int64_t ld = blocks(cols) * FP8_BLOCK;
    uint8_t* q = static_cast<uint8_t*>(ws);
    return crisp_fp8_mat{q, reinterpret_cast<float*>(q + rows * ld), ld, rows, rows, cols, CRISP_FP8_ROWS, 0};
}
static size_t mat_bytes(int64_t rows, int64_t cols) { return ((size_t)rows * blocks(cols) * (FP8_BLOCK + sizeof(float)) + 15) / 16 * 16; }

crisp_status crisp_fp8_linear(const void* X, int32_t in_type, int64_t T, int64_t ldx, const crisp_fp8_mat* W, void* Y, int64_t ldy,
                              int32_t y_type, const crisp_epilogue* ep, void* ws, size_t ws_bytes, void* stream) {
    if (!W) return CRISP_EINVAL;
    crisp_status st = check_mat(W);
    if (st != CRISP_OK || (st = check_in(X, in_type, T, W->cols, ldx)) != CRISP_OK) return st;
    if ((st = check_out(Y, T, W->rows, W->ld, ldy, y_type, ep)) != CRISP_OK) return st;
    hipError_t e;
    if (fp8_takes_raw(T, blocks(W->cols))) {
        e = launch_fp8_raw(X, in_type, T, ldx, *W, Y, ldy, y_type, ep, (hipStream_t)stream);
    } else {
        if (off(ws, 16)) return CRISP_EALIGN;
        if (!ws || ws_bytes < crisp_fp8_linear_ws(T, W->cols)) return CRISP_EBUFSIZE;
        const crisp_fp8_mat q = mat_in(ws, T, W->cols);
        e = launch_fp8_quant(X, in_type, T, W->cols, ldx, nullptr, &q, nullptr, (hipStream_t)stream);
        if (e == hipSuccess) e = launch_fp8_product(q, *W, Y, ldy, y_type, ep, (hipStream_t)stream);
    }
    return e == hipSuccess ? CRISP_OK : CRISP_EDEVICE;
}

size_t crisp_fp8_linear_backward_ws(int64_t T, int64_t S) {
    if (T < 1 || S < 1 || T > MOST || S > MOST || too_many(T, S) || too_many(S, T)) return 0;
    return mat_bytes(T, S) + mat_bytes(S, T);
}

crisp_status crisp_fp8_linear_backward(const void* dY, int32_t in_type, int64_t T, int64_t S, int64_t ldg, const crisp_fp8_mat* Xt,
                                       const crisp_fp8_mat* Wt, void* dX, int64_t lddx, int32_t dx_type, void* dW, int64_t lddw,
                                       int32_t dw_type, int32_t accumulate, void* ws, size_t ws_bytes, void* stream) {
    if (!dX && !dW) return CRISP_EINVAL;
    if ((dX && !Wt) || (dW && !Xt) || (accumulate != 0 && accumulate != 1)) return CRISP_EINVAL;
    crisp_status st = check_in(dY, in_type, T, S, ldg);
    if (st != CRISP_OK) return st;
    if (too_many(S, T)) return CRISP_ESHAPE;
    crisp_epilogue add = {};
    add.residual = dW; add.ldr = lddw;
    const crisp_epilogue* ep = accumulate ? &add : nullptr;
    if (dX) {
        if ((st = check_mat(Wt)) != CRISP_OK) return st;
        if (Wt->cols != S) return CRISP_ESHAPE;
        if ((st = check_out(dX, T, Wt->rows, Wt->ld, lddx, dx_type, nullptr)) != CRISP_OK) return st;
    }
    if (dW) {
        if ((st = check_mat(Xt)) != CRISP_OK) return st;
        if (Xt->cols != T || (dX && Xt->rows != Wt->rows)) return CRISP_ESHAPE;
        if ((st = check_out(dW, S, Xt->rows, Xt->ld, lddw, dw_type, ep)) != CRISP_OK) return st;
    }
    if (off(ws, 16)) return CRISP_EALIGN;
    if (!ws || ws_bytes < crisp_fp8_linear_backward_ws(T, S)) return CRISP_EBUFSIZE;
    if (dX == dW) return CRISP_EINVAL;
    const crisp_fp8_mat g = mat_in(ws, T, S), gt = mat_in(static_cast<uint8_t*>(ws) + mat_bytes(T, S), S, T);
    hipError_t e = launch_fp8_quant(dY, in_type, T, S, ldg, nullptr, dX ? &g : nullptr, dW ? &gt : nullptr, (hipStream_t)stream);
    if (e == hipSuccess && dX && dW) e = launch_fp8_gradients(g, *Wt, dX, lddx, dx_type, gt, *Xt, dW, lddw, dw_type, ep, (hipStream_t)stream);
    else if (e == hipSuccess && dX) e = launch_fp8_product(g, *Wt, dX, lddx, dx_type, nullptr, (hipStream_t)stream);
    else if (e == hipSuccess) e = launch_fp8_product(gt, *Xt, dW, lddw, dw_type, ep, (hipStream_t)stream);
    return e == hipSuccess ? CRISP_OK : CRISP_EDEVICE;
}

}  // extern "C"
