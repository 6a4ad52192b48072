// The 8-bit product's launchers.
#include "fp8_product.h"

namespace crisp {

static ProductArgs args_of(const crisp_fp8_mat& W, int64_t T, void* Y, int64_t ldy, int y_type, const crisp_epilogue* ep) {
    ProductArgs a = {};
    a.w = W.q; a.ws = W.scale; a.ldw = W.ld; a.ldws = W.lds;
    a.T = (int)T; a.S = (int)W.rows; a.K = (int)W.cols; a.kb = (int)((W.cols + FP8_BLOCK - 1) / FP8_BLOCK);
    a.w_tiles = W.kind == CRISP_FP8_TILES;
    a.y = Y; a.ldy = ldy; a.y_bf16 = y_type == CRISP_Y_BF16;
    if (ep) { a.scale = ep->scale; a.bias = ep->bias; a.residual = ep->residual; a.ldr = ep->ldr; a.relu = ep->relu; }
    return a;
}

static ProductArgs args_of(const crisp_fp8_mat& X, const crisp_fp8_mat& W, void* Y, int64_t ldy, int y_type, const crisp_epilogue* ep) {
    ProductArgs a = args_of(W, X.rows, Y, ldy, y_type, ep);
    a.x = X.q; a.xs = X.scale; a.ldx = X.ld; a.ldxs = X.lds;
    return a;
}

static bool takes_split(const ProductArgs& a) { return fp8_takes_split(size_of(a), a.ldx > a.ldw ? a.ldx : a.ldw); }

static hipError_t launch_product(const ProductArgs& a, hipStream_t st) { return takes_split(a) ? launch_fp8_split(a, st) : launch_fp8_tiled(a, st); }

hipError_t launch_fp8_product(const crisp_fp8_mat& X, const crisp_fp8_mat& W, void* Y, int64_t ldy, int y_type,
                              const crisp_epilogue* ep, hipStream_t st) {
    return launch_product(args_of(X, W, Y, ldy, y_type, ep), st);
}

hipError_t launch_fp8_gradients(const crisp_fp8_mat& G, const crisp_fp8_mat& Wt, void* dX, int64_t lddx, int dx_type, const crisp_fp8_mat& Gt,
                                const crisp_fp8_mat& Xt, void* dW, int64_t lddw, int dw_type, const crisp_epilogue* ep, hipStream_t st) {
    const ProductArgs a = args_of(G, Wt, dX, lddx, dx_type, nullptr), b = args_of(Gt, Xt, dW, lddw, dw_type, ep);
    const int pairs = takes_split(a) || takes_split(b) ? 0 : fp8_pairs(size_of(a), size_of(b));
    if (pairs) return launch_fp8_pair(pairs, a, b, st);
    const hipError_t e = launch_product(a, st);
    return e == hipSuccess ? launch_product(b, st) : e;
}

hipError_t launch_fp8_raw(const void* X, int in_type, int64_t T, int64_t ldx, const crisp_fp8_mat& W, void* Y, int64_t ldy, int y_type,
                          const crisp_epilogue* ep, hipStream_t st) {
    ProductArgs a = args_of(W, T, Y, ldy, y_type, ep);
    a.raw = X; a.ldraw = ldx; a.raw_bf16 = in_type == CRISP_IN_BF16;
    return launch_fp8_split(a, st);
}

}  // namespace crisp
