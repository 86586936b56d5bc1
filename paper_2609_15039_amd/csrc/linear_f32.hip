// Binary32 products by expert with an epilogue (gfx950), W float32 or bfloat16 (widened exactly) row-major.
// (The dense ones are the binary32 GEMM's, followed by the epilogue with the sum of its splits or as a launch of its own: at 120-130 of 154
// TFLOP/s the latter's second pass over the product costs 4% at 1000 rows of gate/up.)
//
// Bound by the matrix cores (v_mfma_f32_16x16x4_f32, 154 TFLOP/s) for many rows an expert, by W for few.  Tiles of 16
// or 64 rows x 64 outputs; both operands by 16-byte loads to LDS, three 32-k stages, swizzled; the four waves lie side
// by side along the columns, two or three workgroups share a CU.  An accumulator chain runs over 128 k and is then
// added into a second set of registers, as in the GEMM, so that the rounding error does not grow with K.
#include "linear_plan.hpp"
#include "linear_tile.hpp"

namespace {

constexpr int LF_NW = 4, LF_NT = LF_NW * WAVE, LF_BK = 32, LF_S = 3, LF_CHAIN = 4;

template <int I, int BYTES>
__device__ __forceinline__ unsigned char* lf_stage()
{
    __shared__ __attribute__((aligned(16))) unsigned char buf[BYTES];
    return buf;
}

// TM 16-row blocks; 64 outputs: a 16-column block of each wave, of a gated product one of gate and one of up rows
template <int TM, bool GATED, bool WBF16>
__global__ void __launch_bounds__(LF_NT)
lin_f32_kernel(const LinArgs p, const int ntiles)
{
    constexpr int BM = 16 * TM, TN = GATED ? 2 : 1, BN = 64 * TN, BNO = 64;
    constexpr int RA = BM < 32 ? 32 : BM; // A rows of a stage: a load of every wave
    constexpr int WB = WBF16 ? 64 : 128;  // bytes of a W row and stage
    constexpr int AB = RA * 128, SB = AB + BN * WB;
    constexpr int LA = RA / 8 / LF_NW, WR = WBF16 ? 16 : 8, LW = BN / WR / LF_NW;
    static_assert(LF_S == 3, "stages");
    const int tid = threadIdx.x, lane = tid % WAVE;
    const int wave = __builtin_amdgcn_readfirstlane(tid / WAVE);
    splitee::Group g;
    if (!splitee::find_group<BM>(p, (int)blockIdx.x / ntiles, g)) return;
    const int in = (int)blockIdx.x - g.first * ntiles;
    const int m0 = g.begin + (in % g.tiles) * BM, mend = min(m0 + BM, g.end), n0 = (in / g.tiles) * BNO;
    const int nk = (p.K + LF_BK - 1) / LF_BK;

    // A: load t of the wave fills stage rows 8 j .. 8 j + 7, j = wave + 4 t; lane l writes slot l % 8 of row l / 8,
    // which holds the row's 16-byte chunk slot ^ (row % 8)
    const float* const abase = reinterpret_cast<const float*>(p.A) + (p.row_index ? 0 : m0 * p.lda);
    const int achunk = (lane % 8) ^ (lane / 8);
    uint32_t aoff[LA];
#pragma unroll
    for (int t = 0; t < LA; ++t) {
        const int s = min(m0 + 8 * (wave + LF_NW * t) + lane / 8, mend - 1);
        aoff[t] = (uint32_t)(((p.row_index ? splitee::a_row(p, s) : s - m0) * p.lda + achunk * 4) * 4);
    }
    // W: 4 chunks of a 64-byte bfloat16 row at slot chunk ^ ((row / 4) % 4), 16 rows a load, or 8 chunks of a 128-byte
    // float32 row as in A; stage rows 64 on are up rows
    constexpr int WES = WBF16 ? 2 : 4, WC = WB / 16;
    const char* const wbase = reinterpret_cast<const char*>(p.W) + (int64_t)g.e * p.w_stride * WES;
    const char* wb[LW];
    uint32_t woff[LW];
    int wk[LW];
#pragma unroll
    for (int t = 0; t < LW; ++t) {
        const int j = wave + LF_NW * t, row = WR * j + lane / WC, up = WR * j >= 64 ? p.N : 0;
        const int first = min(n0 + (WR * j) % 64, p.N - 1) + up, n = min(n0 + row % 64, p.N - 1) + up;
        wk[t] = (WBF16 ? (lane % 4) ^ ((row >> 2) & 3) : (lane % 8) ^ (row & 7)) * (16 / WES);
        wb[t] = wbase + (int64_t)first * p.ldw * WES;
        woff[t] = (uint32_t)(((int64_t)(n - first) * p.ldw + wk[t]) * WES);
    }
    unsigned char* const st[3] = {lf_stage<0, SB>(), lf_stage<1, SB>(), lf_stage<2, SB>()};
    auto issue = [&](int t, int q) {
        const int kleft = t < nk ? p.K - t * LF_BK : 0;
#pragma unroll
        for (int i = 0; i < LA; ++i)
            lt_load(abase, achunk * 4 < kleft ? aoff[i] : OOB, t * (LF_BK * 4), st[q] + (wave + LF_NW * i) * 1024);
#pragma unroll
        for (int i = 0; i < LW; ++i)
            lt_load(wb[i], wk[i] < kleft ? woff[i] : OOB, t * (LF_BK * WES), st[q] + AB + (wave + LF_NW * i) * 1024);
    };
    f32x4_t acc[TM][TN], sum[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = sum[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    // lane (r, g) of the MFMA operands: row r of a 16-row block, k = 8 g + e in instruction e of the K tile's eight
    const int fr = lane % 16, fg = lane / 16;
    auto consume = [&](const unsigned char* s) {
        f32x4_t a[2][TM], w[2][TN];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const int row = 16 * i + fr;
                a[h][i] = *reinterpret_cast<const f32x4_t*>(s + row * 128 + (((2 * fg + h) ^ (row & 7)) << 4));
            }
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int row = 64 * j + 16 * wave + fr;
                if (!WBF16) w[h][j] = *reinterpret_cast<const f32x4_t*>(s + AB + row * 128 + (((2 * fg + h) ^ (row & 7)) << 4));
            }
        }
        if (WBF16) {
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int row = 64 * j + 16 * wave + fr;
                const uint4 d = *reinterpret_cast<const uint4*>(s + AB + row * 64 + ((fg ^ ((row >> 2) & 3)) << 4));
                const uint32_t q[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e / 4][j][e % 4] = __uint_as_float(e % 2 ? q[e / 2] & 0xFFFF0000u : q[e / 2] << 16);
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e / 4][i][e % 4], w[e / 4][j][e % 4], acc[i][j], 0, 0, 0);
    };
    auto flush = [&]() {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                sum[i][j] += acc[i][j];
                acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            }
    };
    // tile t in stage t % 3: its loads are in (all but the next tile's), every wave is done with tile t - 1, whose
    // stage takes tile t + 2
    auto step = [&](int t, int q) {
        wait_vmem<LA + LW>();
        lt_barrier();
        issue(t + 2, (q + 2) % 3);
        consume(st[q]);
        if (t % LF_CHAIN == LF_CHAIN - 1) flush();
    };
    issue(0, 0);
    issue(1, 1);
    int t = 0;
    for (; t + 3 <= nk; t += 3) {
        step(t, 0);
        step(t + 1, 1);
        step(t + 2, 2);
    }
    if (t < nk) step(t, 0);
    if (t + 1 < nk) step(t + 1, 1);
    flush();
    wait_vmem<0>();
    lt_barrier();
    // through LDS, four outputs a thread
    constexpr int LD = BN + 4, Z = BM * LD * 4;
    float* const zb = reinterpret_cast<float*>(Z <= SB ? st[0] : lf_stage<3, Z <= SB ? 16 : Z>());
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) zb[(16 * i + 4 * fg + r) * LD + 64 * j + 16 * wave + fr] = sum[i][j][r];
    lt_barrier();
    for (int f = tid; f < (mend - m0) * (BNO / 4); f += LF_NT) {
        const int r = f / (BNO / 4), c = f % (BNO / 4) * 4, row = m0 + r, n = n0 + c, left = p.N - n;
        if (left <= 0) continue;
        float z[2][4];
#pragma unroll
        for (int h = 0; h < TN; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                z[h][i] = zb[r * LD + 64 * h + c + i];
                if (i < left) z[h][i] = splitee::epi_z(p, z[h][i], g.e, row, h * p.N + n + i);
            }
        float res[4];
        splitee::epi_residual(p, row, n, left, res);
        splitee::epi_finish<GATED, false>(p, z[0], z[TN - 1], res, row, n, left);
    }
}

template <int TM, bool GATED>
int f32_run(const LinArgs& p, bool bf16, hipStream_t s)
{
    const int64_t nt = (p.N + 63) / 64, wgs = (p.rows / (16 * TM) + (int64_t)p.experts) * nt;
    if (!splitee_host::launch_fits(wgs, LF_NT)) return SPLITEE_ERR_UNSUPPORTED;
    if (bf16) hipLaunchKernelGGL((lin_f32_kernel<TM, GATED, true>), dim3((unsigned)wgs), dim3(LF_NT), 0, s, p, (int)nt);
    else hipLaunchKernelGGL((lin_f32_kernel<TM, GATED, false>), dim3((unsigned)wgs), dim3(LF_NT), 0, s, p, (int)nt);
    return hipGetLastError() == hipSuccess ? SPLITEE_OK : SPLITEE_ERR_HIP;
}

}  // namespace

namespace splitee_host {

// 16-row tiles up to 48 rows an expert on average (float32 W, whose every row tile costs twice the loads: 32), else 64-row
// tiles, which read W once for four times the rows but are fewer and, gated, leave a CU's LDS room for one workgroup.  Both sides, us,
// 16- and 64-row tiles, 2048 x 768, gated and not:
//   bfloat16 W, 32 experts  24 rows 84 182, 58 80;  48 rows 150 184, 82 81;  64 rows 170 269, 109 134
//               64 experts  24 rows 172 301, 86 148;  48 rows 252 363, 148 158;  8 of 4096 x 2560, 64 rows 371 352, 156 154
//   float32 W, 32 experts   24 rows 149 190, 71 87;  32 rows 153 190, 84 88;  36 rows 208 191, 127 88;  48 rows 218 191, 134 89
//               64 experts  32 rows 318 372, 162 164;  40 rows 380 373, 210 166
int launch_grouped_f32(const splitee::LinArgs& p, bool w_bf16, hipStream_t s)
{
    const bool few = (int64_t)p.rows <= (w_bf16 ? 48 : 32) * (int64_t)p.experts;
    if (p.gated) return few ? f32_run<1, true>(p, w_bf16, s) : f32_run<4, true>(p, w_bf16, s);
    return few ? f32_run<1, false>(p, w_bf16, s) : f32_run<4, false>(p, w_bf16, s);
}

}  // namespace splitee_host
