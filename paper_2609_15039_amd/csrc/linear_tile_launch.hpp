// Launches of the tile kernels with NPL planes; included by one translation unit each.
#pragma once
#include "linear_plan.hpp"
#include "linear_tile.hpp"

namespace {

template <int NPL, int BM, int BN, int WGM, int WGN, int S, bool GATED, bool TILED>
int tile_run(const LinArgs& p, const splitee_host::LinPlan& plan, float* part, hipStream_t s)
{
    using T = LinTile<NPL, BM, BN, WGM, WGN, S, GATED, TILED>;
    const int64_t nt = (p.N + T::BNO - 1) / T::BNO;
    const int64_t strips = p.offsets ? p.rows / BM + (int64_t)p.experts : (p.rows + BM - 1) / BM;
    const int64_t wgs = p.offsets ? (strips * nt + 127) / 128 * 128 : strips * nt * plan.ksplit; // (by expert: the 8 x 16 order)
    if (wgs > INT32_MAX) return SPLITEE_ERR_UNSUPPORTED;
    const LtPlan lt{(int)nt, plan.ksplit, plan.ktps, part, (int)splitee_host::part_ld(p.N, GATED)};
    hipLaunchKernelGGL((lin_tile_kernel<NPL, BM, BN, WGM, WGN, S, GATED, TILED>), dim3((unsigned)wgs), dim3(T::NT), 0, s, p, lt);
    return hipGetLastError() == hipSuccess ? SPLITEE_OK : SPLITEE_ERR_HIP;
}

// Stages: of 64 x 128 tiles as many as let two workgroups share a CU's 160 KB, of 128 x 256 as many as fit.
template <int NPL, bool TILED>
int tile_size(const LinArgs& p, const splitee_host::LinPlan& plan, float* part, hipStream_t s)
{
    constexpr int S = NPL == 1 ? 3 : 2;
    if (plan.kind == splitee_host::LinPlan::TILE64)
        return p.gated ? tile_run<NPL, 64, 128, 2, 2, S, true, TILED>(p, plan, part, s)
                       : tile_run<NPL, 64, 128, 2, 2, S, false, TILED>(p, plan, part, s);
    return p.gated ? tile_run<NPL, 128, 256, 2, 4, S, true, TILED>(p, plan, part, s)
                   : tile_run<NPL, 128, 256, 2, 4, S, false, TILED>(p, plan, part, s);
}

}  // namespace
