// Argument checks shared by the translation units of the C ABI.
#pragma once
#include <stdint.h>

#include <hip/hip_runtime.h>

#include "splitee.h"

namespace {

constexpr int64_t MAX_DIM = int64_t(1) << 30;

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool pitch16(int64_t ld, int64_t elsize) { return (ld * elsize) % 16 == 0; }
inline hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }


inline bool dims_ok(int64_t M, int64_t N, int64_t K)
{
    return M >= 0 && N >= 0 && K >= 0 && M <= MAX_DIM && N <= MAX_DIM && K <= MAX_DIM;
}

inline int64_t prec_elsize(int prec) { return prec == SPLITEE_PREC_F64 ? 8 : prec == SPLITEE_PREC_F32 ? 4 : 2; }
inline int64_t prec_planes(int prec) { return prec == SPLITEE_PREC_BF16X3 ? 3 : 1; }
inline bool valid_prec(int prec)
{
    return prec == SPLITEE_PREC_F32 || prec == SPLITEE_PREC_BF16 || prec == SPLITEE_PREC_BF16X3;
}
inline bool valid_dtype(int t) { return t == SPLITEE_F32 || t == SPLITEE_BF16 || t == SPLITEE_BF16_TILED; }

// GEMM operand checks shared by the GEMM entry points.
int check_w(const void* W, int w_type, int64_t ldw, int64_t K, int prec)
{
    if (!valid_dtype(w_type)) return SPLITEE_ERR_DTYPE;
    if (w_type == SPLITEE_BF16_TILED) { // ldw is not used: the layout is fixed by N and K
        if (prec == SPLITEE_PREC_F32) return SPLITEE_ERR_UNSUPPORTED;
        return aligned16(W) ? SPLITEE_OK : SPLITEE_ERR_ALIGN;
    }
    if (prec != SPLITEE_PREC_F32 && w_type != SPLITEE_BF16) return SPLITEE_ERR_UNSUPPORTED;
    const int64_t wes = w_type == SPLITEE_F32 ? 4 : 2;
    if (ldw < K) return SPLITEE_ERR_SHAPE;
    if (!aligned16(W) || !pitch16(ldw, wes)) return SPLITEE_ERR_ALIGN;
    return SPLITEE_OK;
}

}  // namespace
