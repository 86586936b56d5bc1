// Launches of the few-row kernels with NPL planes; included by one translation unit each.
#pragma once
#include "linear_plan.hpp"
#include "linear_rows.hpp"

namespace {

template <int NPL, int BM, int TN, int NW, bool GATED, bool TILED>
int rows_run(const LinArgs& p, hipStream_t s)
{
    constexpr int BNO = 16 * (GATED ? TN / 2 : TN);
    const int64_t nt = (p.N + BNO - 1) / BNO;
    const int64_t strips = p.offsets ? p.rows / BM + (int64_t)p.experts : (p.rows + BM - 1) / BM;
    if (!splitee_host::launch_fits(strips * nt, NW * WAVE)) return SPLITEE_ERR_UNSUPPORTED;
    hipLaunchKernelGGL((lin_rows_kernel<NPL, BM, TN, NW, GATED, TILED>), dim3((unsigned)(strips * nt)), dim3(NW * WAVE), 0, s, p,
                       (int)nt);
    return hipGetLastError() == hipSuccess ? SPLITEE_OK : SPLITEE_ERR_HIP;
}

template <int NPL, int BM, int NW, bool TILED>
int rows_tn(const LinArgs& p, int tn, hipStream_t s)
{
    if (p.gated) return rows_run<NPL, BM, 2, NW, true, TILED>(p, s);
    return tn == 1 ? rows_run<NPL, BM, 1, NW, false, TILED>(p, s) : rows_run<NPL, BM, 2, NW, false, TILED>(p, s);
}

template <int NPL, bool TILED>
int rows_bm(const LinArgs& p, const splitee_host::LinPlan& plan, hipStream_t s)
{
    if (plan.bm == 8) return plan.nw == 4 ? rows_tn<NPL, 8, 4, TILED>(p, plan.tn, s) : rows_tn<NPL, 8, 8, TILED>(p, plan.tn, s);
    return plan.nw == 4 ? rows_tn<NPL, 16, 4, TILED>(p, plan.tn, s) : rows_tn<NPL, 16, 8, TILED>(p, plan.tn, s);
}

}  // namespace
