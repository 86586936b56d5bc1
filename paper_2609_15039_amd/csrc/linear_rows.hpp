// Few rows of bfloat16 products with an epilogue on the matrix cores (gfx950), dense and by expert.
//
// Bound by W, read once from HBM.  A workgroup owns BM rows (8 or 16) and 16 TN weight rows (gated: half of
// them gate, half up rows of the same outputs); its waves split K: wave w takes the 64-k tiles w, w + NW, ..,
// and the waves' sums meet in LDS and are added in wave order, so that the result does not depend on timing and
// no other workgroup is waited for.  W goes straight to the registers that the MFMA reads, two K tiles ahead; the rows
// of A go to LDS by 1 KB loads, 8 rows of whole 128-byte lines each, into a stage that belongs to one
// wave: no barrier in the loop.  Two K tiles ahead: three and four were slower (one token of 2 x 9728 x 2560 17.6, 21.8 and
// 23.7 us, W then partly in caches), and so were 32-row tiles (32 rows in three planes 34 us, twice 16 rows 33).
//
// One token of 2 x 9728 x 2560, three planes, gated, with its correction: 19.8 us (5.0 TB/s of W), 21.5 where none of W is in
// a cache; one token of 2560 x 9728 12.5; 64 rows of 64 experts, 2 x 768 x 2048, bfloat16: 46 us (about 5.4 TB/s of the experts that have rows).
#pragma once
#include "linear_tile.hpp"

namespace {

template <int I, int BYTES>
__device__ __forceinline__ unsigned char* lr_stage()
{
    __shared__ __attribute__((aligned(16))) unsigned char buf[BYTES];
    return buf;
}

// 16 bytes of each lane from base + voff + soff (zeros from 2 GB on)
__device__ __forceinline__ uint4 lr_load(const void* base, uint32_t voff, int soff)
{
    u32x4_t v = __builtin_amdgcn_raw_buffer_load_b128(make_rsrc(base, 0x7FFFFFFFu), (int)voff, soff, 0);
    return make_uint4(v.x, v.y, v.z, v.w);
}

template <int NPL, int BM, int TN, int NW, bool GATED, bool TILED>
__global__ void __launch_bounds__(NW * WAVE)
lin_rows_kernel(const LinArgs p, const int ntiles)
{
    constexpr int R = 2;                        // K tiles ahead
    constexpr int LA = NPL * BM / 8, LW = 2 * TN; // loads per K tile
    constexpr int TO = GATED ? TN / 2 : TN, BN = 16 * TN, BNO = 16 * TO;
    // LDS of a wave's stage: planes of BM rows; 8 rows fill half of a 16-row block, whose other rows hold whatever the next
    // bytes of LDS hold: they reach rows of the product that nobody reads
    constexpr int SB = NPL * BM * 128, SBP = BM < 16 ? SB + 1024 : SB;
    constexpr int LDR = BN + 4, RB = NW * BM * LDR * 4;
    constexpr int NT = NW * WAVE;
    static_assert(BM == 8 || BM == 16, "one 16-row block of the MFMA");
    static_assert(!GATED || TN % 2 == 0, "gate and up blocks in pairs");
    static_assert((R - 1) * (LA + LW) < 64, "loads in flight exceed the wait counter");
    const int tid = threadIdx.x, lane = tid % WAVE;
    const int wave = __builtin_amdgcn_readfirstlane(tid / WAVE);

    splitee::Group g;
    const int L = blockIdx.x;
    if (!splitee::find_group<BM>(p, L / ntiles, g)) return;
    const int in = L - g.first * ntiles;
    const int m0 = g.begin + (in % g.tiles) * BM, n0 = (in / g.tiles) * BNO;
    const int ktiles = (p.K + BK - 1) / BK;
    const int ng = ktiles > wave ? (ktiles - wave + NW - 1) / NW : 0; // this wave's K tiles
    const int fr = lane % 16, fq = lane / 16;

    // W: lane (r, q) takes weight row r of a 16-row block, 16 bytes at k = 32 s + 8 q of step s of the K tile
    const uint16_t* const wbase = reinterpret_cast<const uint16_t*>(p.W) + (int64_t)g.e * p.w_stride;
    const uint16_t* wb[TN];
    uint32_t woff[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const bool up = j >= TO;
        const int c0 = n0 + 16 * (j % TO), half = up ? p.N : 0;
        const int first = min(c0, p.N - 1) + half, n = min(c0 + fr, p.N - 1) + half;
        if (TILED) {
            wb[j] = wbase + (int64_t)(first / 32) * ktiles * 2048;
            woff[j] = (uint32_t)((((n / 32 - first / 32) * ktiles) * 2048 + (fq / 2) * 512 + (fq % 2) * 256 + (n % 32) * 8) * 2);
        } else {
            wb[j] = wbase + (int64_t)first * p.ldw;
            woff[j] = (uint32_t)(((int64_t)(n - first) * p.ldw + fq * 8) * 2);
        }
    }
    // A: load t fills stage rows 8 t .. 8 t + 7 (row BM pl + r of plane pl); lane l writes slot l % 8 of row
    // 8 t + l / 8, which holds the row's 16-byte chunk slot ^ ((row / 2) % 8)
    const uint16_t* const abase = reinterpret_cast<const uint16_t*>(p.A) + (p.row_index ? 0 : m0 * p.lda);
    uint32_t aoff[BM / 8];
    int akc[2]; // k of the lane's chunk, by parity of the load
#pragma unroll
    for (int i = 0; i < 2; ++i) akc[i] = ((lane % 8) ^ ((4 * i + lane / 16) & 7)) * 8;
#pragma unroll
    for (int t = 0; t < BM / 8; ++t) {
        const int s = min(m0 + 8 * t + lane / 8, g.end - 1);
        aoff[t] = (uint32_t)((p.row_index ? splitee::a_row(p, s) : s - m0) * p.lda * 2);
    }
    unsigned char* const st[R] = {lr_stage<0, NW * SBP>(), lr_stage<1, NW * SBP>()};
    uint4 wr[R][2][TN];
    // this wave's K tile gk into ring slot u (zeros past its last)
    auto issue = [&](int gk, int u) {
        const int kt = wave + NW * gk, k = kt * BK;
        const int kleft = gk < ng ? p.K - k : 0;
#pragma unroll
        for (int t = 0; t < LA; ++t) {
            const int kc = akc[t % 2];
            lt_load(abase + (t / (BM / 8)) * p.pstride, kc < kleft ? aoff[t % (BM / 8)] + kc * 2 : OOB, k * 2,
                    st[u] + wave * SBP + t * 1024);
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const bool dead = TILED ? kleft <= 0 : 32 * s + 8 * fq >= kleft;
#pragma unroll
            for (int j = 0; j < TN; ++j)
                wr[u][s][j] = lr_load(wb[j], dead ? OOB : woff[j] + (TILED ? s * 2048 : s * 64), TILED ? kt * 4096 : k * 2);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
#pragma unroll
    for (int u = 0; u < R; ++u) issue(u, u);

    f32x4_t acc[2][TN];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[s][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    auto consume = [&](int u) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            uint4 a[NPL];
#pragma unroll
            for (int pl = 0; pl < NPL; ++pl) {
                const int row = pl * BM + fr;
                a[pl] = *reinterpret_cast<const uint4*>(st[u] + wave * SBP + row * 128 + (((4 * s + fq) ^ ((row >> 1) & 7)) << 4));
            }
#pragma unroll
            for (int pl = 0; pl < NPL; ++pl)
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    acc[s][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a[pl]), as_bf16x8(wr[u][s][j]), acc[s][j], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    int gk = 0;
    for (; gk + R <= ng; gk += R) {
#pragma unroll
        for (int u = 0; u < R; ++u) {
            wait_vmem<(R - 1) * (LA + LW)>(); // this slot's loads are in; the younger slot's may be in flight
            __builtin_amdgcn_sched_barrier(0);
            consume(u);
            __builtin_amdgcn_s_waitcnt((0 << 8) | (7 << 4) | 15 | (3 << 14)); // lgkmcnt(0): the slot's rows are read
            issue(gk + u + R, u);
        }
    }
    wait_vmem<0>(); // the last tile of an odd count, and the loads past it (zeros)
    __builtin_amdgcn_sched_barrier(0);
    if (gk < ng) consume(0);

    // the waves' sums meet in LDS and are added in wave order
    float* const red = reinterpret_cast<float*>(RB <= NW * SBP ? st[0] : lr_stage<2, RB <= NW * SBP ? 16 : RB>());
    __syncthreads();
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const f32x4_t v = acc[0][j] + acc[1][j];
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (4 * fq + r < BM) red[(wave * BM + 4 * fq + r) * LDR + 16 * j + fr] = v[r];
    }
    __syncthreads();
    const int rows = min(BM, g.end - m0);
    for (int f = tid; f < rows * BNO; f += NT) {
        const int r = f / BNO, c = f % BNO, row = m0 + r, n = n0 + c;
        if (n >= p.N) continue;
        float z[2];
#pragma unroll
        for (int h = 0; h < (GATED ? 2 : 1); ++h) {
            z[h] = red[r * LDR + h * BNO + c];
#pragma unroll
            for (int v = 1; v < NW; ++v) z[h] += red[(v * BM + r) * LDR + h * BNO + c];
        }
        float act[1] = {splitee::epi_z(p, z[0], g.e, row, n)};
        splitee::epi_act(act, p.act);
        float y = act[0];
        if (GATED) y *= splitee::epi_z(p, z[GATED ? 1 : 0], g.e, row, p.N + n);
        splitee::epi_store(p, y, row, n);
    }
}

}  // namespace
