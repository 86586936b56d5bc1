// Launches of the tile kernels with NPL planes; included by one translation unit each.
#pragma once
#include "linear_plan.hpp"
#include "linear_tile.hpp"

namespace {

template <int NPL, int BM, int BN, int WGM, int WGN, int S, bool HALF, bool GATED, bool TILED>
int tile_run(const LinArgs& p, const splitee_host::LinPlan& plan, float* part, hipStream_t s)
{
    using T = LinTile<NPL, BM, BN, WGM, WGN, S, GATED, TILED>;
    const int64_t nt = (p.N + T::BNO - 1) / T::BNO;
    const int64_t strips = p.offsets ? p.rows / BM + (int64_t)p.experts : (p.rows + BM - 1) / BM;
    const int64_t tiles = strips * nt, nbig = HALF && plan.halve ? tiles / 256 * 256 : tiles;
    const int64_t wgs = p.offsets ? (tiles + 255) / 256 * 256 // (by expert: the 8 x 32 order)
                                  : (nbig + 2 * (tiles - nbig)) * plan.ksplit;
    if (!splitee_host::launch_fits(wgs, T::NT)) return SPLITEE_ERR_UNSUPPORTED;
    const LtPlan lt{(int)nt, plan.ksplit, plan.ktps, part, (int)splitee_host::part_ld(p.N, GATED), (int)(2 * (tiles - nbig))};
    hipLaunchKernelGGL((lin_tile_kernel<NPL, BM, BN, WGM, WGN, S, GATED, TILED, HALF>), dim3((unsigned)wgs), dim3(T::NT), 0, s, p, lt);
    return hipGetLastError() == hipSuccess ? SPLITEE_OK : SPLITEE_ERR_HIP;
}

template <int NPL, int BM, int BN, int WGM, int WGN, int S, bool HALF, bool TILED>
int tile_gated(const LinArgs& p, const splitee_host::LinPlan& plan, float* part, hipStream_t s)
{
    return p.gated ? tile_run<NPL, BM, BN, WGM, WGN, S, HALF, true, TILED>(p, plan, part, s)
                   : tile_run<NPL, BM, BN, WGM, WGN, S, HALF, false, TILED>(p, plan, part, s);
}

// Stages: of 64 x 128 tiles as many as let two workgroups share a CU's 160 KB, of the others as many as fit.
template <int NPL, bool TILED>
int tile_size(const LinArgs& p, const splitee_host::LinPlan& plan, float* part, hipStream_t s)
{
    using splitee_host::LinPlan;
    constexpr int S = NPL == 1 ? 3 : 2;
    if (plan.kind == LinPlan::TILE64) return tile_gated<NPL, 64, 128, 2, 2, S, false, TILED>(p, plan, part, s);
    if constexpr (NPL == 1)
        if (plan.kind == LinPlan::TILE256) return tile_gated<1, 256, 256, 2, 4, 2, true, TILED>(p, plan, part, s);
    if (plan.ksplit == 1) return tile_gated<NPL, 128, 256, 2, 4, S, true, TILED>(p, plan, part, s);
    return tile_gated<NPL, 128, 256, 2, 4, S, false, TILED>(p, plan, part, s);
}

}  // namespace
