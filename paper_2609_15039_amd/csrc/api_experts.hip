// C ABI of the projections with an epilogue and of the expert path: argument validation and kernel
// launches.  Semantics of every entry point are documented in include/splitee.h.
#include "api_checks.hpp"
#include "linear_plan.hpp"
#include "splitee_probe.h"

namespace splitee_host {
// Bytes of the partial tiles of a dense product whose K is split (0: not split).
size_t linear_workspace_bytes(int64_t M, int64_t N, int64_t K, int prec, int gated);
int launch_linear(const splitee::LinArgs& p, int prec, int w_type, void* ws, hipStream_t s);
size_t route_workspace_bytes(int64_t T, int64_t E);
int launch_route(const float* logits, int64_t ldl, int64_t T, int64_t E, int64_t k, int score, int renorm,
                 int32_t* experts, float* weights, int32_t* offsets, int32_t* row_index, int32_t* slot, void* ws,
                 hipStream_t s);
int launch_combine(const void* H, bool h_bf16, int64_t ldh, int64_t h_rows, const int32_t* slot, const float* weights,
                   const void* res, int64_t ldres, void* Y, bool y_bf16, int64_t ldy, int64_t T, int64_t k, int64_t N,
                   hipStream_t s);
}  // namespace splitee_host

namespace {

constexpr int64_t LIN_MAX_LD = int64_t(1) << 20; // a tile's rows stay within 31 bits of its first one's address
constexpr int64_t LIN_MAX_N = int64_t(1) << 28;
constexpr int64_t ROUTE_MAX_E = 1024, ROUTE_MAX_K = 64;
// tokens: a launch has fewer than 2^32 threads (32 a token in the router, 256 in the weighted sum)
constexpr int64_t ROUTE_MAX_T = int64_t(1) << 26, COMBINE_MAX_T = (int64_t(1) << 24) - 1;

inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
inline bool valid_out(int t) { return t == SPLITEE_F32 || t == SPLITEE_BF16; }
inline int64_t out_elsize(int t) { return t == SPLITEE_F32 ? 4 : 2; }

// Checks of the epilogue against N output columns, pointers aside.
int check_epilogue(const splitee_epilogue_t* ep, int64_t N)
{
    if (!ep) return SPLITEE_ERR_ARG;
    if (ep->act < SPLITEE_ACT_NONE || ep->act > SPLITEE_ACT_RELU || ep->gated < 0 || ep->gated > 1) return SPLITEE_ERR_ARG;
    if (!valid_out(ep->out_type)) return SPLITEE_ERR_DTYPE;
    const int64_t nw = ep->gated ? 2 * N : N;
    if ((ep->C && ep->ldc < nw) || (ep->residual && ep->ldres < N) || ep->bias_stride < 0) return SPLITEE_ERR_SHAPE;
    return SPLITEE_OK;
}

int check_pointers(const void* A, int prec, int64_t lda, const splitee_epilogue_t* ep, const void* Y, int64_t ldy)
{
    if (!aligned16(A) || !pitch16(lda, prec_elsize(prec)) || !aligned16(Y) || !pitch16(ldy, out_elsize(ep->out_type)) ||
        (ep->C && (!aligned16(ep->C) || !pitch16(ep->ldc, 4))) || (ep->bias && !aligned4(ep->bias)) ||
        (ep->residual && (!aligned16(ep->residual) || !pitch16(ep->ldres, out_elsize(ep->out_type)))))
        return SPLITEE_ERR_ALIGN;
    return SPLITEE_OK;
}

splitee::LinArgs lin_args(const void* A, int64_t lda, int64_t a_rows, const void* W, int64_t ldw,
                          const splitee_epilogue_t* ep, void* Y, int64_t ldy, int64_t rows, int64_t N, int64_t K)
{
    splitee::LinArgs p{};
    p.A = A; p.lda = lda; p.pstride = a_rows * lda; p.a_rows = (int)a_rows;
    p.experts = 1;
    p.W = W; p.ldw = ldw;
    p.C = ep->C; p.ldc = ep->ldc;
    p.bias = ep->bias; p.bias_stride = ep->bias_stride;
    p.res = ep->residual; p.ldres = ep->ldres;
    p.Y = Y; p.ldy = ldy;
    p.act = ep->act; p.gated = ep->gated; p.out_bf16 = ep->out_type == SPLITEE_BF16;
    p.rows = (int)rows; p.N = (int)N; p.K = (int)K;
    return p;
}

}  // namespace

extern "C" {

size_t splitee_epilogue_workspace_bytes(int64_t M, int64_t N, int64_t K, int prec, int gated)
{
    if (!valid_prec(prec) || !dims_ok(M, N, K) || K % 8 != 0 || gated < 0 || gated > 1) return 0;
    if (M == 0 || N == 0 || N >= LIN_MAX_N || K >= LIN_MAX_LD) return 0;
    return splitee_host::linear_workspace_bytes(M, N, K, prec, gated);
}

int splitee_linear_epilogue(const void* A, int in_prec, int64_t lda, const void* W, int w_type, int64_t ldw,
                            const splitee_epilogue_t* ep, void* Y, int64_t ldy, int64_t M, int64_t N, int64_t K,
                            void* workspace, size_t workspace_bytes, void* stream)
{
    if (!valid_prec(in_prec)) return SPLITEE_ERR_UNSUPPORTED;
    if (!dims_ok(M, N, K) || K % 8 != 0 || lda < K || ldy < N) return SPLITEE_ERR_SHAPE;
    int rc = check_epilogue(ep, N);
    if (rc) return rc;
    rc = check_w(W, w_type, ldw, K, in_prec);
    if (rc) return rc;
    if (lda >= LIN_MAX_LD || K >= LIN_MAX_LD || N >= LIN_MAX_N || (w_type != SPLITEE_BF16_TILED && ldw >= LIN_MAX_LD))
        return SPLITEE_ERR_UNSUPPORTED;
    const size_t need = splitee_epilogue_workspace_bytes(M, N, K, in_prec, ep->gated);
    if (workspace_bytes < need || (need > 0 && workspace == nullptr)) return SPLITEE_ERR_WORKSPACE;
    if (workspace && (reinterpret_cast<uintptr_t>(workspace) & 255u)) return SPLITEE_ERR_ALIGN;
    if (M == 0 || N == 0) return SPLITEE_OK;
    if ((K > 0 && (!A || !W)) || !Y) return SPLITEE_ERR_ARG;
    rc = check_pointers(A, in_prec, lda, ep, Y, ldy);
    if (rc) return rc;
    return splitee_host::launch_linear(lin_args(A, lda, M, W, ldw, ep, Y, ldy, M, N, K), in_prec, w_type,
                                       need ? workspace : nullptr, as_stream(stream));
}

int splitee_grouped_linear(const void* A, int in_prec, int64_t lda, int64_t a_rows, const int32_t* row_index,
                           const int32_t* offsets, int64_t experts, const void* W, int w_type, int64_t ldw,
                           int64_t w_stride, const splitee_epilogue_t* ep, void* Y, int64_t ldy, int64_t rows,
                           int64_t N, int64_t K, void* stream)
{
    if (!valid_prec(in_prec)) return SPLITEE_ERR_UNSUPPORTED;
    if (!dims_ok(rows, N, K) || !dims_ok(a_rows, 0, 0) || experts < 0 || experts > MAX_DIM || K % 8 != 0 || lda < K || ldy < N ||
        w_stride < 0 || (rows > 0 && a_rows < 1) || (!row_index && a_rows < rows))
        return SPLITEE_ERR_SHAPE;
    int rc = check_epilogue(ep, N);
    if (rc) return rc;
    rc = check_w(W, w_type, ldw, K, in_prec);
    if (rc) return rc;
    if (lda >= LIN_MAX_LD || K >= LIN_MAX_LD || N >= LIN_MAX_N || (w_type != SPLITEE_BF16_TILED && ldw >= LIN_MAX_LD))
        return SPLITEE_ERR_UNSUPPORTED;
    // gathered rows are addressed from the first one's with 31 bits
    if (row_index && a_rows * lda * prec_elsize(in_prec) > INT32_MAX) return SPLITEE_ERR_UNSUPPORTED;
    if (!pitch16(w_stride, w_type == SPLITEE_F32 ? 4 : 2)) return SPLITEE_ERR_ALIGN;
    if (rows == 0 || N == 0 || experts == 0) return SPLITEE_OK;
    if ((K > 0 && (!A || !W)) || !Y || !offsets) return SPLITEE_ERR_ARG;
    rc = check_pointers(A, in_prec, lda, ep, Y, ldy);
    if (rc) return rc;
    if (!aligned4(offsets) || !aligned4(row_index)) return SPLITEE_ERR_ALIGN;
    splitee::LinArgs p = lin_args(A, lda, a_rows, W, ldw, ep, Y, ldy, rows, N, K);
    p.row_index = row_index;
    p.offsets = offsets;
    p.experts = (int)experts;
    p.w_stride = w_stride;
    return splitee_host::launch_linear(p, in_prec, w_type, nullptr, as_stream(stream));
}

int splitee_linear_plan_probe(int64_t rows, int64_t groups, int dense, int64_t N, int64_t K, int prec, int gated, int* plan)
{
    if (!plan || (prec != SPLITEE_PREC_BF16 && prec != SPLITEE_PREC_BF16X3) || !dims_ok(rows, N, K) || rows < 1 || N < 1 ||
        groups < 1 || groups > MAX_DIM || K % 8 != 0 || gated < 0 || gated > 1)
        return SPLITEE_ERR_ARG;
    const splitee_host::LinPlan p = splitee_host::plan_linear(rows, groups, dense != 0, N, K, prec == SPLITEE_PREC_BF16X3 ? 3 : 1, gated);
    const bool few = p.kind == splitee_host::LinPlan::ROWS;
    plan[0] = (int)p.kind;
    plan[1] = few ? p.bm : 0;
    plan[2] = few ? p.tn : 0;
    plan[3] = few ? p.nw : 0;
    plan[4] = p.ksplit;
    plan[5] = p.halve ? 1 : 0;
    return SPLITEE_OK;
}

size_t splitee_route_workspace_bytes(int64_t T, int64_t E, int64_t k)
{
    if (!dims_ok(T, E, k) || k < 1 || k > E || k > ROUTE_MAX_K || E > ROUTE_MAX_E || T > ROUTE_MAX_T || T * k > INT32_MAX) return 0;
    return splitee_host::route_workspace_bytes(T, E);
}

int splitee_route(const float* logits, int64_t ldl, int64_t T, int64_t E, int64_t k, int score, int renorm,
                  int32_t* experts, float* weights, int32_t* offsets, int32_t* row_index, int32_t* slot,
                  void* workspace, size_t workspace_bytes, void* stream)
{
    if (score != SPLITEE_SCORE_SOFTMAX && score != SPLITEE_SCORE_SIGMOID) return SPLITEE_ERR_ARG;
    if (!dims_ok(T, E, k) || k < 1 || k > E || ldl < E) return SPLITEE_ERR_SHAPE;
    if (E > ROUTE_MAX_E || k > ROUTE_MAX_K || T > ROUTE_MAX_T || T * k > INT32_MAX) return SPLITEE_ERR_UNSUPPORTED;
    const size_t need = splitee_host::route_workspace_bytes(T, E);
    if (!workspace || workspace_bytes < need) return SPLITEE_ERR_WORKSPACE;
    if (reinterpret_cast<uintptr_t>(workspace) & 255u) return SPLITEE_ERR_ALIGN;
    if (!offsets || (T > 0 && (!logits || !experts || !weights || !row_index || !slot))) return SPLITEE_ERR_ARG;
    if (!aligned4(logits) || !aligned4(experts) || !aligned4(weights) || !aligned4(offsets) || !aligned4(row_index) ||
        !aligned4(slot))
        return SPLITEE_ERR_ALIGN;
    return splitee_host::launch_route(logits, ldl, T, E, k, score, renorm != 0, experts, weights, offsets, row_index, slot,
                                      workspace, as_stream(stream));
}

int splitee_combine(const void* H, int h_type, int64_t ldh, int64_t h_rows, const int32_t* slot, const float* weights,
                    const void* residual, int64_t ldres, void* Y, int out_type, int64_t ldy, int64_t T, int64_t k,
                    int64_t N, void* stream)
{
    if (!valid_out(h_type) || !valid_out(out_type)) return SPLITEE_ERR_DTYPE;
    if (!dims_ok(T, N, k) || !dims_ok(h_rows, 0, 0) || k < 1 || ldh < N || ldy < N || (residual && ldres < N)) return SPLITEE_ERR_SHAPE;
    if (k > ROUTE_MAX_K || N >= LIN_MAX_LD || T > COMBINE_MAX_T) return SPLITEE_ERR_UNSUPPORTED;
    if (T == 0 || N == 0) return SPLITEE_OK;
    if ((!H && h_rows > 0) || !slot || !weights || !Y) return SPLITEE_ERR_ARG;
    if (!aligned16(H) || !pitch16(ldh, out_elsize(h_type)) || !aligned16(Y) || !pitch16(ldy, out_elsize(out_type)) ||
        !aligned4(slot) || !aligned4(weights) ||
        (residual && (!aligned16(residual) || !pitch16(ldres, out_elsize(out_type)))))
        return SPLITEE_ERR_ALIGN;
    return splitee_host::launch_combine(H, h_type == SPLITEE_BF16, ldh, h_rows, slot, weights, residual, ldres, Y,
                                        out_type == SPLITEE_BF16, ldy, T, k, N, as_stream(stream));
}

}  // extern "C"
