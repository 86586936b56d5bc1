// Products with an epilogue, dense and by expert (gfx950): splitee_linear_epilogue and
// splitee_grouped_linear.
//
//   Z = fl32(A W^T) - C + bias;  H = act(Z) or act(Z_gate) Z_up;  Y = round(H + residual)
#include <algorithm>
#include <cmath>

#include "gemm_dev.hpp"
#include "linear_plan.hpp"

namespace {

using splitee::LinArgs;

// The partial products of a split K, added in split order, and the epilogue: four columns a thread.  Bound by the
// partials, which are still in a cache (two splits of 333 x 2560: 4 us, most of it latency).
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
    float res[4];
    splitee::epi_residual(p, row, n, p.N - n, res);
    splitee::epi_finish<GATED, false>(p, z[0], z[GATED], res, row, n, p.N - n);
}

// The same from a binary32 GEMM's partial tiles (F32Partials): a wave takes 16 rows x 16 columns, a lane four rows of a
// column, all splits of them in flight together, C, bias and the residual too, and adds in the GEMM's order.  40 x 4096 x 2560
// with everything 17.8 us, with the sum and the epilogue in launches of their own 21.3; one row 2560 x 9728 17.2 and 20.1.
constexpr int FP_MAX_KS = 16;
template <bool GATED, int TN>
__global__ void __launch_bounds__(256) f32_partials_kernel(LinArgs p, splitee_host::F32Partials f, int colblocks)
{
    const int lane = threadIdx.x % 64, b = blockIdx.x * 4 + threadIdx.x / 64;
    const int rb = b / colblocks, row0 = 16 * rb + 4 * (lane / 16), col = 16 * (b % colblocks) + lane % 16;
    if (16 * rb >= p.rows) return;
    constexpr int H = GATED ? 2 : 1;
    float cv[H][4], bias[H], res[4];
#pragma unroll
    for (int h = 0; h < H; ++h) {
        bias[h] = p.bias ? p.bias[col < p.N ? h * p.N + col : 0] : 0.f;
#pragma unroll
        for (int r = 0; r < 4; ++r)
            cv[h][r] = p.C ? p.C[row0 + r < p.rows && col < p.N ? (int64_t)(row0 + r) * p.ldc + h * p.N + col : 0] : 0.f;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int64_t at = row0 + r < p.rows && col < p.N ? (int64_t)(row0 + r) * p.ldres + col : 0;
        res[r] = !p.res ? 0.f
                 : p.out_bf16 ? splitee::bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(p.res)[at])
                              : reinterpret_cast<const float*>(p.res)[at];
    }
    const int per = f.tm * TN * 64; // float4 of a wave's partial
    const __amdgpu_buffer_rsrc_t rp = make_rsrc(f.part, (uint32_t)((int64_t)f.tiles * f.ksplit * per * 64));
    f32x4_t v[H][FP_MAX_KS];
#pragma unroll
    for (int h = 0; h < H; ++h) {
        const int c = h * p.N + min(col, p.N - 1), in = c % (64 * TN);
        const int tile = c / (64 * TN) * f.mtiles + rb / f.tm;
        const int e = in / (16 * TN) * per + (rb % f.tm * TN + in / 16 % TN) * 64 + lane / 16 * 16 + c % 16;
#pragma unroll
        for (int q = 0; q < FP_MAX_KS; ++q)
            v[h][q] = __builtin_bit_cast(f32x4_t, load16(rp, q < f.ksplit ? (uint32_t)((q * f.tiles + tile) * 4 * per + e) * 16 : OOB));
    }
    float z[H][4];
#pragma unroll
    for (int h = 0; h < H; ++h) {
#pragma unroll
        for (int q = 1; q < FP_MAX_KS; ++q)
            if (q < f.ksplit) v[h][0] += v[h][q];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            z[h][r] = v[h][0][r];
            if (p.C) z[h][r] -= cv[h][r];
            if (p.bias) z[h][r] += bias[h];
        }
    }
    splitee::epi_act(z[0], p.act);
    if (col >= p.N) return;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if (row0 + r >= p.rows) return;
        float h = z[0][r];
        if (GATED) h *= z[H - 1][r];
        if (p.res) h += res[r];
        const int64_t at = (int64_t)(row0 + r) * p.ldy + col;
        if (p.out_bf16) reinterpret_cast<uint16_t*>(p.Y)[at] = (uint16_t)splitee::bf16_bits_rne(h);
        else reinterpret_cast<float*>(p.Y)[at] = h;
    }
}

}  // namespace

namespace splitee_host {

// The cheapest kernel by a model of the launch's time in microseconds, fitted to products of 1-4000 rows with 256-9728
// wide W dense, and of 8-48000 rows of 8-64 experts, W not in any cache (within 15% of most of them):
//  few rows   5 + the largest of W at 5.3 TB/s (16 rows of three planes: 4.4), 6.2e-4 (6.5e-4) a workgroup and K tile, and
//             0.5 a K tile of a wave;
//  64 x 128   6 + the larger of W at 4.8 TB/s and rounds of 512 workgroups (two a CU) times K tiles at 0.30 us (three
//             planes 0.90) where each CU has one at most, 0.85 (1.40) where it has two;
//  128 x 256  8 + rounds of 256 times K tiles at 1.0 us (2.2), 0.65 (1.8) where a quarter of the CUs is idle;
//  256 x 256  12 + rounds of 256 times K tiles at 1.5 us;
//  a split K  2 + its partial products written and read at 6 TB/s.
// Both sides of the borders, us: 512 rows of 64 experts (768 gated x 2048), few rows 80 and 64 x 128 88, 1024 rows 100 and
// 95; 100 rows of gate/up in three planes, 64 x 128 in three splits 54 and 128 x 256 in three 46; 333 rows of down, 33
// either way; 48000 rows of 64 experts 128 x 256 352, 256 x 256 357; 4096 rows x 9728 x 2560, 128 x 256 228, 256 x 256 207.
// groups: experts.  By expert only the total of the rows is known here: experts are taken to be chosen evenly, and each
// ends with half a tile.
LinPlan plan_linear(int64_t rows, int64_t groups, bool dense, int64_t N, int64_t K, int npl, int gated)
{
    const int64_t kt = std::max<int64_t>(1, (K + 63) / 64);
    const double live = dense ? 1.0 : std::max(1.0, groups * (1.0 - std::exp(-(double)rows / groups)));
    const double wbytes = live * N * (gated ? 2 : 1) * K * 2.0;
    auto strips = [&](int bm) { return dense ? (double)((rows + bm - 1) / bm) : live * std::max(1.0, rows / live / bm + 0.5); };
    const bool x3 = npl == 3;
    LinPlan best{};
    best.cost = 1e30;
    for (int bm = 8; bm <= 16; bm *= 2) {
        LinPlan p{LinPlan::ROWS, bm, 2, 4, 1, (int)kt, false, 0.0};
        auto wgs = [&]() { const int bno = 16 * p.tn / (gated ? 2 : 1); return strips(bm) * ((N + bno - 1) / bno); };
        if (!gated && wgs() < 128) p.tn = 1; // 16 columns each: more CUs at work
        // eight waves where K is long and their stages leave room for two workgroups, or there are few
        if (kt >= 32 && (npl * bm <= 24 || wgs() <= 256)) p.nw = 8;
        p.cost = 5 + std::max({wbytes / (x3 && bm == 16 ? 4.4e6 : 5.3e6), wgs() * kt * (x3 ? 6.5e-4 : 6.2e-4) * p.tn / 2,
                               (double)((kt + p.nw - 1) / p.nw) * 0.5});
        if (p.cost < best.cost) best = p;
    }
    // microseconds of a K tile, with few and with many workgroups, and of all else
    struct Tile { LinPlan::Kind kind; int bm, bn, slots; double few, full, fixed; bool split, halves; };
    const Tile tiles[] = {
        {LinPlan::TILE64, 64, 128, 512, x3 ? 0.90 : 0.30, x3 ? 1.40 : 0.85, 6, true, false},
        {LinPlan::TILE128, 128, 256, 256, x3 ? 1.8 : 0.65, x3 ? 2.2 : 1.0, 8, true, true},
        {LinPlan::TILE256, 256, 256, 256, 1.5, 1.5, 12, false, true}};
    for (const Tile& t : tiles) {
        if (t.kind == LinPlan::TILE256 && (x3 || !dense)) continue;
        const int bno = t.bn / (gated ? 2 : 1);
        const double n = strips(t.bm) * ((N + bno - 1) / bno);
        const int most = dense && t.split ? (int)std::min<int64_t>(8, std::max<int64_t>(1, kt / 4)) : 1;
        for (int ks = 1; ks <= most; ++ks) {
            LinPlan p{t.kind, 0, 0, 0, ks, (int)((kt + ks - 1) / ks), false, 0.0};
            if ((int64_t)(ks - 1) * p.ktps >= kt) continue; // a split without K tiles
            const double wgs = n * ks, rounds = std::floor(wgs / t.slots), rest = wgs - rounds * t.slots;
            const double fill = (rest - (t.kind == LinPlan::TILE64 ? 256 : 192)) / 64; // of the last round
            const double last = rest == 0 ? 0.0 : p.ktps * (t.few + (t.full - t.few) * std::min(1.0, std::max(0.0, fill)));
            p.halve = dense && t.halves && ks == 1 && rest > 0 && rest <= t.slots / 2 && rounds > 0;
            const double time = rounds * p.ktps * t.full + (p.halve ? 0.62 * p.ktps * t.full
                                                            : !dense && rounds >= 2 ? rest / t.slots * p.ktps * t.full : last);
            p.cost = t.fixed + std::max(time, wbytes / 4.8e6);
            if (ks > 1) p.cost += 2 + ks * rows * part_ld(N, gated) * 8.0 / 6e6;
            if (p.cost < best.cost) best = p;
        }
    }
    return best;
}

namespace {

// Dense binary32: the GEMM's partials (behind its counters, which it does not use), then the product, in the layout
// of one split; gate and up are two GEMMs where the up rows' columns would not be 16-byte aligned.
struct F32Dense {
    int64_t n;           // columns of a GEMM
    int halves;          // GEMMs
    int64_t ld;
    size_t gemm, bytes;  // of the GEMM's part and of all
};
F32Dense f32_dense(int64_t M, int64_t N, int64_t K, int gated)
{
    F32Dense d{};
    d.halves = gated && N % 4 != 0 ? 2 : 1;
    d.n = gated && d.halves == 1 ? 2 * N : N;
    d.ld = part_ld(N, gated);
    d.gemm = (splitee::WS_COUNTER_BYTES + f32_gemm_workspace_bytes(M, d.n, K) + 255) / 256 * 256;
    d.bytes = d.gemm + (size_t)M * d.ld * 4;
    return d;
}

int64_t sum_workgroups(const LinArgs& p) { return ((int64_t)p.rows * ((p.N + 3) / 4) + 255) / 256; }

int launch_sum(const LinArgs& p, const float* part, int ksplit, hipStream_t s)
{
    const int ld = (int)part_ld(p.N, p.gated);
    const dim3 grid((unsigned)sum_workgroups(p));
    if (p.gated) hipLaunchKernelGGL(linear_sum_kernel<true>, grid, dim3(256), 0, s, p, part, ksplit, ld);
    else hipLaunchKernelGGL(linear_sum_kernel<false>, grid, dim3(256), 0, s, p, part, ksplit, ld);
    return hipGetLastError() == hipSuccess ? SPLITEE_OK : SPLITEE_ERR_HIP;
}

int launch_f32_partials(const LinArgs& p, const F32Partials& f, hipStream_t s)
{
    const int64_t colblocks = (p.N + 15) / 16, wgs = ((int64_t)(p.rows + 15) / 16 * colblocks + 3) / 4;
    if (!launch_fits(wgs, 256)) return SPLITEE_ERR_UNSUPPORTED;
#define FP_RUN(GATED, TN) hipLaunchKernelGGL((f32_partials_kernel<GATED, TN>), dim3((unsigned)wgs), dim3(256), 0, s, p, f, (int)colblocks)
    if (p.gated) { if (f.tn == 1) FP_RUN(true, 1); else FP_RUN(true, 2); }
    else { if (f.tn == 1) FP_RUN(false, 1); else FP_RUN(false, 2); }
#undef FP_RUN
    return hipGetLastError() == hipSuccess ? SPLITEE_OK : SPLITEE_ERR_HIP;
}

int launch_dense_f32(const LinArgs& p, int w_type, void* ws, hipStream_t s)
{
    if (!launch_fits(sum_workgroups(p), 256)) return SPLITEE_ERR_UNSUPPORTED;
    const F32Dense d = f32_dense(p.rows, p.N, p.K, p.gated);
    const float* A = reinterpret_cast<const float*>(p.A);
    if (!p.gated && !p.bias && !p.res && p.act == SPLITEE_ACT_NONE && !p.out_bf16) // the unmask is the GEMM's own
        return launch_gemm_f32(A, p.lda, p.W, w_type, p.ldw, p.C, p.ldc, reinterpret_cast<float*>(p.Y), p.ldy, p.rows, p.N, p.K, ws,
                               d.gemm, s);
    float* R = reinterpret_cast<float*>(reinterpret_cast<char*>(ws) + d.gemm);
    F32Partials left{};
    for (int h = 0; h < d.halves; ++h) {
        const char* W = reinterpret_cast<const char*>(p.W) + (int64_t)h * p.N * p.ldw * (w_type == SPLITEE_F32 ? 4 : 2);
        const int rc = launch_gemm_f32(A, p.lda, W, w_type, p.ldw, nullptr, 0, R + h * (d.ld / 2), d.ld, p.rows, d.n, p.K, ws, d.gemm, s,
                                       d.halves == 1 ? &left : nullptr);
        if (rc != SPLITEE_OK) return rc;
    }
    if (left.part) return launch_f32_partials(p, left, s); // (all tiles split: rows few enough)
    return launch_sum(p, R, 1, s);
}

}  // namespace

size_t linear_workspace_bytes(int64_t M, int64_t N, int64_t K, int prec, int gated)
{
    if (prec == SPLITEE_PREC_F32) return f32_dense(M, N, K, gated).bytes;
    const LinPlan plan = plan_linear(M, 1, true, N, K, prec == SPLITEE_PREC_BF16X3 ? 3 : 1, gated);
    return plan.ksplit > 1 ? (size_t)plan.ksplit * M * part_ld(N, gated) * 4 : 0;
}

int launch_linear(const LinArgs& p, int prec, int w_type, void* ws, hipStream_t s)
{
    if (prec == SPLITEE_PREC_F32)
        return p.offsets ? launch_grouped_f32(p, w_type == SPLITEE_BF16, s) : launch_dense_f32(p, w_type, ws, s);
    const bool x3 = prec == SPLITEE_PREC_BF16X3, tiled = w_type == SPLITEE_BF16_TILED;
    const LinPlan plan = plan_linear(p.rows, p.experts, !p.offsets, p.N, p.K, x3 ? 3 : 1, p.gated);
    if (plan.kind == LinPlan::ROWS)
        return x3 ? launch_linear_rows_bf16x3(p, tiled, plan, s) : launch_linear_rows_bf16(p, tiled, plan, s);
    float* part = plan.ksplit > 1 ? reinterpret_cast<float*>(ws) : nullptr;
    if (part && !launch_fits(sum_workgroups(p), 256)) return SPLITEE_ERR_UNSUPPORTED;
    const int rc = x3 ? launch_linear_tile_bf16x3(p, tiled, plan, part, s) : launch_linear_tile_bf16(p, tiled, plan, part, s);
    return rc != SPLITEE_OK || !part ? rc : launch_sum(p, part, plan.ksplit, s);
}

}  // namespace splitee_host
