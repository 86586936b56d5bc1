// Products with an epilogue, dense and by expert (gfx950): splitee_linear_epilogue and
// splitee_grouped_linear.
//
//   Z = fl32(A W^T) - C + bias;  H = act(Z) or act(Z_gate) Z_up;  Y = round(H + residual)
#include <algorithm>
#include <cmath>

#include "linear_plan.hpp"

namespace {

using splitee::LinArgs;

constexpr int LS_T = 16;  // rows and columns of a tile
constexpr int LS_K = 32;  // k of one stage

__device__ __forceinline__ float ls_w(const LinArgs& p, int w_type, int e, int n, int k)
{
    const int64_t base = (int64_t)e * p.w_stride;
    if (w_type == SPLITEE_F32) return reinterpret_cast<const float*>(p.W)[base + (int64_t)n * p.ldw + k];
    const uint16_t* w = reinterpret_cast<const uint16_t*>(p.W) + base;
    if (w_type == SPLITEE_BF16) return splitee::bf16_bits_to_f32(w[(int64_t)n * p.ldw + k]);
    const int64_t kt = (p.K + 63) / 64;
    return splitee::bf16_bits_to_f32(
        w[((((int64_t)(n / 32) * kt + k / 64) * 4 + (k % 64) / 16) * 64 + ((k % 16) / 8) * 32 + n % 32) * 8 + k % 8]);
}

__device__ __forceinline__ float ls_a(const LinArgs& p, int prec, int64_t row, int k)
{
    const int64_t i = row * p.lda + k;
    if (prec == SPLITEE_PREC_F32) return reinterpret_cast<const float*>(p.A)[i];
    const uint16_t* a = reinterpret_cast<const uint16_t*>(p.A);
    float x = splitee::bf16_bits_to_f32(a[i]);
    if (prec == SPLITEE_PREC_BF16X3) // exact: the planes sum to a binary32 value
        x = (x + splitee::bf16_bits_to_f32(a[p.pstride + i])) + splitee::bf16_bits_to_f32(a[2 * p.pstride + i]);
    return x;
}

// One thread per output, operands through LDS as binary32.
__global__ void __launch_bounds__(LS_T * LS_T) linear_simple_kernel(LinArgs p, int prec, int w_type)
{
    __shared__ float sa[LS_T][LS_K + 1], sw[2][LS_T][LS_K + 1];
    splitee::Group g;
    if (!splitee::find_group<LS_T>(p, blockIdx.y, g)) return;
    const int e = g.e, m0 = g.begin + ((int)blockIdx.y - g.first) * LS_T, mend = g.end;
    const int n0 = blockIdx.x * LS_T, tid = threadIdx.x, r = tid / LS_T, c = tid % LS_T;
    const int halves = p.gated ? 2 : 1;
    float acc[2] = {0.f, 0.f};
    for (int k0 = 0; k0 < p.K; k0 += LS_K) {
        for (int i = tid; i < LS_T * LS_K; i += LS_T * LS_T) {
            const int ir = i / LS_K, k = k0 + i % LS_K;
            sa[ir][i % LS_K] = m0 + ir < mend && k < p.K ? ls_a(p, prec, splitee::a_row(p, m0 + ir), k) : 0.f;
            for (int h = 0; h < halves; ++h)
                sw[h][ir][i % LS_K] = n0 + ir < p.N && k < p.K ? ls_w(p, w_type, e, n0 + ir + h * p.N, k) : 0.f;
        }
        __syncthreads();
        for (int k = 0; k < LS_K; ++k)
            for (int h = 0; h < halves; ++h) acc[h] = fmaf(sa[r][k], sw[h][c][k], acc[h]);
        __syncthreads();
    }
    const int row = m0 + r, n = n0 + c;
    if (row >= mend || n >= p.N) return;
    float h = splitee::epi_act(splitee::epi_z(p, acc[0], e, row, n), p.act);
    if (p.gated) h *= splitee::epi_z(p, acc[1], e, row, n + p.N);
    splitee::epi_store(p, h, row, n);
}

// The partial products of a split K, added in split order, and the epilogue: four columns a thread.
template <bool GATED>
__global__ void __launch_bounds__(256) linear_sum_kernel(LinArgs p, const float* __restrict__ part, int ksplit, int ldpart)
{
    const int quads = (p.N + 3) / 4;
    const int64_t f = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int row = (int)(f / quads), n = (int)(f % quads) * 4;
    if (row >= p.rows) return;
    float z[2][4];
#pragma unroll
    for (int h = 0; h < (GATED ? 2 : 1); ++h) {
        const float* q = part + (int64_t)row * ldpart + h * (ldpart / 2) + n;
        float4 v = *reinterpret_cast<const float4*>(q);
        for (int s = 1; s < ksplit; ++s) {
            const float4 w = *reinterpret_cast<const float4*>(q + (int64_t)s * p.rows * ldpart);
            v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
        }
        z[h][0] = v.x; z[h][1] = v.y; z[h][2] = v.z; z[h][3] = v.w;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < p.N) z[h][i] = splitee::epi_z(p, z[h][i], 0, row, h * p.N + n + i);
    }
    splitee::epi_finish4<GATED>(p, make_float4(z[0][0], z[0][1], z[0][2], z[0][3]),
                                make_float4(z[GATED][0], z[GATED][1], z[GATED][2], z[GATED][3]),
                                splitee::epi_residual4(p, row, n, p.N - n), row, n, p.N - n);
}

}  // namespace

namespace splitee_host {

// The cheapest kernel by a model of the launch's time in microseconds, fitted to products of 1-4096 rows (1-64
// experts), 2560-9728 wide W dense and 768 x 2048 by expert:
//  few rows   5 + the larger of 5.5e-4 a workgroup and K tile (the rate of W from HBM) and 0.5 a K tile of a wave;
//  64 x 128   6 + rounds of 512 workgroups (two a CU) times K tiles at 0.70 us (three planes 1.06), 0.30 (0.90)
//             where each CU has one workgroup at most;
//  128 x 256  8 + rounds of 256 workgroups times K tiles at 1.0 us (2.15);
//  a split K  4 + its partial products written and read at 4 TB/s.
// groups: experts (1: dense, whose K may be split).  By expert only the total of the rows is known here: as many groups as
// there can be have rows, and each ends with half a tile.
LinPlan plan_linear(int64_t rows, int64_t groups, bool dense, int64_t N, int64_t K, int npl, int gated)
{
    const int64_t kt = std::max<int64_t>(1, (K + 63) / 64), live = std::max<int64_t>(1, std::min(groups, rows));
    auto strips = [&](int bm) {
        return dense ? (double)((rows + bm - 1) / bm) : live * std::max(1.0, (double)rows / live / bm + 0.5);
    };
    LinPlan best{};
    best.cost = 1e30;
    for (int bm = 8; bm <= 16; bm *= 2) {
        LinPlan p{LinPlan::ROWS, bm, 2, 4, 1, (int)kt, false, 0.0};
        auto wgs = [&]() { const int bno = 16 * p.tn / (gated ? 2 : 1); return strips(bm) * ((N + bno - 1) / bno); };
        if (!gated && wgs() < 256) p.tn = 1; // 16 columns each: more CUs at work
        // eight waves where K is long and their stages leave room for two workgroups, or there are few
        if (kt >= 32 && (npl * bm <= 24 || wgs() <= 256)) p.nw = 8;
        p.cost = 5 + std::max(wgs() * kt * 5.5e-4 * p.tn / 2, (double)((kt + p.nw - 1) / p.nw) * 0.5);
        if (p.cost < best.cost) best = p;
    }
    // microseconds of a K tile, alone on a CU (64 x 128) or with as many as fit, and of all else
    struct Tile { LinPlan::Kind kind; int bm, bn, slots; double alone, full, fixed; bool split, halves; };
    const Tile tiles[] = {
        {LinPlan::TILE64, 64, 128, 512, npl == 1 ? 0.30 : 0.90, npl == 1 ? 0.80 : 1.40, 6, true, false},
        {LinPlan::TILE128, 128, 256, 256, npl == 1 ? 1.0 : 2.15, npl == 1 ? 1.0 : 2.15, 8, true, npl == 3},
        {LinPlan::TILE256, 256, 256, 256, 1.5, 1.5, 12, false, true}};
    for (const Tile& t : tiles) {
        if (t.kind == LinPlan::TILE256 && npl != 1) continue;
        const int bno = t.bn / (gated ? 2 : 1);
        const double n = strips(t.bm) * ((N + bno - 1) / bno);
        const int most = dense && t.split ? (int)std::min<int64_t>(8, std::max<int64_t>(1, kt / 4)) : 1;
        for (int ks = 1; ks <= most; ++ks) {
            LinPlan p{t.kind, 0, 0, 0, ks, (int)((kt + ks - 1) / ks), false, 0.0};
            if ((int64_t)(ks - 1) * p.ktps >= kt) continue; // a split without K tiles
            const double wgs = n * ks, rounds = std::floor(wgs / t.slots);
            const double round = p.ktps * (t.alone + (t.full - t.alone) * std::min(1.0, std::max(0.0, (wgs - 256) / 256)));
            const double rest = wgs - rounds * t.slots;
            p.halve = dense && t.halves && ks == 1 && rest > 0 && rest <= t.slots / 2;
            p.cost = t.fixed + rounds * round + (rest == 0 ? 0 : p.halve ? 0.62 * round : !dense && rounds >= 2 ? rest / t.slots * round : round);
            if (ks > 1) p.cost += 4 + ks * rows * part_ld(N, gated) * 8.0 / 4e6;
            if (p.cost < best.cost) best = p;
        }
    }
    return best;
}

size_t linear_workspace_bytes(int64_t M, int64_t N, int64_t K, int prec, int gated)
{
    if (prec == SPLITEE_PREC_F32) return 0;
    const LinPlan plan = plan_linear(M, 1, true, N, K, prec == SPLITEE_PREC_BF16X3 ? 3 : 1, gated);
    return plan.ksplit > 1 ? (size_t)plan.ksplit * M * part_ld(N, gated) * 4 : 0;
}

int launch_linear(const LinArgs& p, int prec, int w_type, void* ws, hipStream_t s)
{
    if (prec == SPLITEE_PREC_F32) {
        // row tiles of all groups: at most one partly filled one each
        const int64_t tiles = p.offsets ? p.rows / LS_T + (int64_t)p.experts : (p.rows + LS_T - 1) / LS_T;
        if (tiles > 65535) return SPLITEE_ERR_UNSUPPORTED;
        hipLaunchKernelGGL(linear_simple_kernel, dim3((unsigned)((p.N + LS_T - 1) / LS_T), (unsigned)tiles),
                           dim3(LS_T * LS_T), 0, s, p, prec, w_type);
        return hipGetLastError() == hipSuccess ? SPLITEE_OK : SPLITEE_ERR_HIP;
    }
    const bool x3 = prec == SPLITEE_PREC_BF16X3, tiled = w_type == SPLITEE_BF16_TILED;
    const LinPlan plan = plan_linear(p.rows, p.experts, !p.offsets, p.N, p.K, x3 ? 3 : 1, p.gated);
    if (plan.kind == LinPlan::ROWS)
        return x3 ? launch_linear_rows_bf16x3(p, tiled, plan, s) : launch_linear_rows_bf16(p, tiled, plan, s);
    float* part = plan.ksplit > 1 ? reinterpret_cast<float*>(ws) : nullptr;
    const int rc = x3 ? launch_linear_tile_bf16x3(p, tiled, plan, part, s) : launch_linear_tile_bf16(p, tiled, plan, part, s);
    if (rc != SPLITEE_OK || !part) return rc;
    const int64_t quads = (int64_t)p.rows * ((p.N + 3) / 4);
    const int ld = (int)part_ld(p.N, p.gated);
    if ((quads + 255) / 256 > INT32_MAX) return SPLITEE_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)((quads + 255) / 256));
    if (p.gated) hipLaunchKernelGGL(linear_sum_kernel<true>, grid, dim3(256), 0, s, p, part, plan.ksplit, ld);
    else hipLaunchKernelGGL(linear_sum_kernel<false>, grid, dim3(256), 0, s, p, part, plan.ksplit, ld);
    return hipGetLastError() == hipSuccess ? SPLITEE_OK : SPLITEE_ERR_HIP;
}

}  // namespace splitee_host
