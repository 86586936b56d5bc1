// Which kernel a product with an epilogue takes, and the launches of the translation units that hold them.
#pragma once
#include "epilogue_dev.hpp"

namespace splitee_host {

// kind: few rows (BM rows, TN 16-row weight blocks, NW waves) or a tile (BM x BN, K split into ksplit)
struct LinPlan {
    enum Kind { ROWS, TILE64, TILE128, TILE256 } kind;
    int bm, tn, nw; // ROWS
    int ksplit, ktps;
    bool halve;     // the tiles of the last, partly filled round in two halves each
    double cost;    // microseconds
};

LinPlan plan_linear(int64_t rows, int64_t groups, bool dense, int64_t N, int64_t K, int npl, int gated);

// launches of one kernel family; part: the partial tiles of a split K, or null
int launch_linear_rows_bf16(const splitee::LinArgs& p, bool tiled, const LinPlan& plan, hipStream_t s);
int launch_linear_rows_bf16x3(const splitee::LinArgs& p, bool tiled, const LinPlan& plan, hipStream_t s);
int launch_linear_tile_bf16(const splitee::LinArgs& p, bool tiled, const LinPlan& plan, float* part, hipStream_t s);
int launch_linear_tile_bf16x3(const splitee::LinArgs& p, bool tiled, const LinPlan& plan, float* part, hipStream_t s);

int launch_grouped_f32(const splitee::LinArgs& p, bool w_bf16, hipStream_t s);

// Leading dimension of a split's partial product (16-byte rows; of a gated one, gate columns then up columns).
inline int64_t part_ld(int64_t N, int gated) { return (N + 3) / 4 * 4 * (gated ? 2 : 1); }

// A launch has fewer than 2^32 threads.
inline bool launch_fits(int64_t workgroups, int threads) { return workgroups <= (int64_t)UINT32_MAX / threads; }

}  // namespace splitee_host
