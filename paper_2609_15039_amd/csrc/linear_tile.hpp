// Tiles of bfloat16 products with an epilogue on the matrix cores (gfx950), dense and by expert.
//
// Both operands go to LDS by 1 KB buffer loads, S stages of 64 k, in a swizzled order that the fragment reads find free
// of bank conflicts (the tiled weight order needs none).  One barrier per K tile, before the last of its four steps:
// the fragments of a step are read under the MFMAs of the one before, the next tile's first ones under the last step's,
// and the freed stage is filled from there.  The epilogue takes C and bias off the accumulators where they are
// and passes 32-row blocks through LDS, so that activation, residual and stores go row by row, eight columns a lane.
//
// What bounds it: the operand tiles that every CU takes from its L2 (64 KB for 256 x 256 x 64: about 1.05 us without
// the MFMAs), which take the MFMAs' time (1.05 us at the 1.6 PFLOP/s that the matrix cores sustain on such data, 1.3 with
// their LDS reads and barriers) to 1.5; and a tile's beginning and end, 4 and 5 us, when nothing is multiplied.  4096 x 2560
// x 9728 with bias and GELU 188 us (1.09 PFLOP/s, the MFMAs busy 49% of the cycles, CUs 87%; 223 with operands from HBM, not the
// Infinity Cache); 1000 x 2560 x 2 x 9728 in three planes, gated, 272 us (1.10, busy 50%); 48000 rows of 64 experts x 2048 x 2 x 768
// 332 us (0.91, 45%).
// Built and measured against it, not kept: a ring of five operand slots instead of two stages (84 us against 80 for 4096 x
// 4096 x 2560), four waves of 128 x 128 (their accumulators do not stay in registers), wave priority around the MFMAs (within 1%),
// C's lines touched when a tile begins (277 against 273), 128 x 128 tiles, two workgroups a CU (383 against 340 for the experts).
#pragma once
#include "epilogue_dev.hpp"
#include "gemm_dev.hpp"

#include <type_traits>

namespace {

using splitee::LinArgs;

template <int I, int BYTES>
__device__ __forceinline__ unsigned char* lt_stage()
{
    __shared__ __attribute__((aligned(16))) unsigned char buf[BYTES];
    return buf;
}

template <int N>
using lt_int = std::integral_constant<int, N>;

// 16 bytes of each lane from base + voff + soff (zeros from 2 GB on) to 1 KB of LDS at `to`
__device__ __forceinline__ void lt_load(const void* base, uint32_t voff, int soff, unsigned char* to)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(make_rsrc(base, 0x7FFFFFFFu), (lds_ptr_t)to, 16, (int)voff, soff, 0, 0);
}

// Barrier of the workgroup for its LDS alone: stores to memory may still be on their way.
__device__ __forceinline__ void lt_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Tile of a workgroup: which rows, which weight rows, which K tiles.
struct LtPlan {
    int ntiles;          // column tiles
    int ksplit, ktps;    // splits of K and K tiles of one
    float* part;         // partial tiles of a split K: split s at part + s * rows * ldpart, row-major; of a gated product
    int ldpart;          // gate columns, then from ldpart / 2 up columns
    int nhalf;           // HALF, dense: workgroups with half tiles, of which two make one of the first nhalf / 2 tiles
};

template <int NPL, int BM, int BN, int WGM, int WGN, int S, bool GATED, bool TILED>
struct LinTile {
    static constexpr int NW = WGM * WGN, NT = NW * WAVE;
    static constexpr int TM = BM / WGM / 32, TN = BN / WGN / 32;
    static constexpr int AB = NPL * BM * 128;
    static constexpr int SB = AB + BN * 128;
    static constexpr int LA = NPL * BM / 8 / NW, LW = BN / 8 / NW; // 1 KB loads of a wave and stage
    static constexpr int BNO = GATED ? BN / 2 : BN;                // output columns
    static_assert(BN / 8 % NW == 0 && NW % 2 == 0, "loads");
    static_assert(!GATED || TN % 2 == 0, "gate and up blocks in pairs");
    static_assert(BM % (8 * NW) == 0, "a load lies in one plane");
};

// Rows m0 .. mend - 1 (at most BM of them) and the weight rows from output column n0 on.  SB: bytes of a stage, those
// of the largest tile that the kernel has.
template <int NPL, int BM, int BN, int WGM, int WGN, int S, bool GATED, bool TILED, int SB>
__device__ __forceinline__ void lin_tile(const LinArgs& p, const LtPlan& plan, const splitee::Group& g, int m0, int n0, int mend,
                                         int split)
{
    using T = LinTile<NPL, BM, BN, WGM, WGN, S, GATED, TILED>;
    constexpr int NW = T::NW, TM = T::TM, TN = T::TN, LA = T::LA, LW = T::LW, AB = T::AB;
    constexpr int TO = GATED ? TN / 2 : TN; // column blocks of outputs of a wave
    static_assert(T::SB <= SB, "stage");
    const int tid = threadIdx.x, lane = tid % WAVE;
    const int wave = __builtin_amdgcn_readfirstlane(tid / WAVE);
    const int ktiles = (p.K + BK - 1) / BK;
    const int kt0 = split * plan.ktps, nk = min(plan.ktps, ktiles - kt0);

    // ---- loads: 8 rows of 128 bytes each; lane l fills slot l % 8 of row l / 8 with the row's 16-byte chunk
    // slot ^ ((row / 2) % 8).  Loads j = wave + NW t, so (row / 2) % 8 is the same for all of a lane's.
    // Each is a buffer load from the tile's (of gathered rows: the matrix's) first row, its offset within the row
    // block fixed and the K tile in the scalar offset; an offset of 2 GB and more reads zeros.
    const int lchunk = (lane % 8) ^ ((4 * wave + lane / 16) & 7);
    // LDS row block b (32 weight rows) of the tile is column block b % TN of wave column b / TN; of a gated
    // tile the first TN / 2 are gate rows, the others the up rows of the same outputs
    const uint16_t* const wbase = reinterpret_cast<const uint16_t*>(p.W) + (int64_t)g.e * p.w_stride;
    const uint16_t* wb[LW]; // uniform
    uint32_t woff[LW];
#pragma unroll
    for (int t = 0; t < LW; ++t) {
        const int j = wave + NW * t, b = j / 4, wn = b / TN, jj = b % TN;
        const bool up = jj >= TO;
        const int c0 = n0 + 32 * (wn * TO + jj % TO); // the block's first output column
        const int first = min(c0, p.N - 1) + (up ? p.N : 0);                   // and weight row
        if (TILED) { // 1 KB: a 16-k step of a 32-row block, as the MFMA takes it
            const int n = min(c0 + lane % 32, p.N - 1) + (up ? p.N : 0);
            wb[t] = wbase + ((int64_t)(first / 32) * ktiles + kt0) * 2048;
            woff[t] = (uint32_t)((((n / 32 - first / 32) * ktiles) * 2048 + (j % 4) * 512 + (lane / 32) * 256 + (n % 32) * 8) * 2);
        } else {
            const int n = min(c0 + 8 * (j % 4) + lane / 8, p.N - 1) + (up ? p.N : 0);
            wb[t] = wbase + (int64_t)first * p.ldw + kt0 * BK;
            woff[t] = (uint32_t)(((int64_t)(n - first) * p.ldw + lchunk * 8) * 2);
        }
    }
    unsigned char* const st[3] = {lt_stage<0, SB>(), lt_stage<1, SB>(), lt_stage<(S > 2 ? 2 : 0), SB>()};
    static_assert(S == 2 || S == 3, "stages");
    // the operands' relative K tile t to the stage at `to`: zeros past K and past the split
    auto issue_w = [&](int t, unsigned char* to) {
        const int kleft = t < nk ? p.K - (kt0 + t) * BK : 0;
        const uint32_t dead = (TILED ? 0 : lchunk * 8) < kleft ? 0u : OOB;
#pragma unroll
        for (int i = 0; i < LW; ++i) lt_load(wb[i], woff[i] | dead, t * (TILED ? 4096 : BK * 2), to + AB + (wave + NW * i) * 1024);
    };
    issue_w(0, st[0]); // (ahead of the indexes of gathered rows)
    const uint16_t* const abase = reinterpret_cast<const uint16_t*>(p.A) + (p.row_index ? 0 : m0 * p.lda) + kt0 * BK;
    constexpr int TPL = LA / NPL; // loads of a plane
    uint32_t aoff[TPL];
#pragma unroll
    for (int t = 0; t < TPL; ++t) {
        const int s = min(m0 + 8 * (wave + NW * t) + lane / 8, mend - 1); // a row past the group's: any of its rows
        aoff[t] = (uint32_t)(((p.row_index ? splitee::a_row(p, s) : s - m0) * p.lda + lchunk * 8) * 2);
    }
    auto issue_a = [&](int t, unsigned char* to) {
        const uint32_t dead = lchunk * 8 < (t < nk ? p.K - (kt0 + t) * BK : 0) ? 0u : OOB;
#pragma unroll
        for (int i = 0; i < LA; ++i)
            lt_load(abase + (i / TPL) * p.pstride, aoff[i % TPL] | dead, t * (BK * 2), to + (wave + NW * i) * 1024);
    };

    f32x16_t acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

    // MFMA operands: lane (r, h) holds row r of a 32-row block, k = 8 h .. + 7 of the 16-k step
    const int wm = wave / WGN, wn = wave % WGN, fr = lane % 32, fh = lane / 32;
    const int fsw = (fr >> 1) & 7;
    uint4 fa[2][NPL][TM], fw[2][TN];
    auto read = [&](const unsigned char* sa, int step, int to) {
        const unsigned char* const sw = sa + AB;
        const int off = ((2 * step + fh) ^ fsw) << 4;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int b = wn * TN + j;
            fw[to][j] = TILED ? *reinterpret_cast<const uint4*>(sw + b * 4096 + step * 1024 + lane * 16)
                              : *reinterpret_cast<const uint4*>(sw + (32 * b + fr) * 128 + off);
        }
#pragma unroll
        for (int pl = 0; pl < NPL; ++pl)
#pragma unroll
            for (int i = 0; i < TM; ++i)
                fa[to][pl][i] = *reinterpret_cast<const uint4*>(sa + (pl * BM + 32 * (wm * TM + i) + fr) * 128 + off);
    };
    auto mul = [&](int from) {
#pragma unroll
        for (int pl = 0; pl < NPL; ++pl)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(fa[from][pl][i]), as_bf16x8(fw[from][j]), acc[i][j], 0, 0, 0);
    };
    constexpr int READS = TN + NPL * TM, MULS = NPL * TM * TN;
    // K tile t, its first fragments in registers.  Steps 0 .. 2 multiply while the next step's fragments are read.  Then
    // every wave is done with the tile, and tile t + 1 is in everywhere behind the barrier: the last step multiplies
    // while tile t + 1's first fragments are read and the loads into the freed LDS begin.  c: t modulo a turn.
    auto step = [&](int t, auto cc) {
        constexpr int c = decltype(cc)::value;
#pragma unroll
        for (int s = 0; s < 3; ++s) {
            read(st[c], s + 1, (s + 1) % 2);
            mul(s % 2);
#pragma unroll
            for (int i = 0; i < READS; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x008, MULS / READS > 0 ? MULS / READS : 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, MULS, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        wait_vmem<(S - 2) * (LA + LW)>();
        __builtin_amdgcn_s_waitcnt((0 << 8) | (7 << 4) | 15 | (3 << 14)); // lgkmcnt(0): the last fragments are in
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        read(st[(c + 1) % S], 0, 0);
        issue_a(t + S, st[c]);
        issue_w(t + S, st[c]);
        mul(1);
#pragma unroll
        for (int i = 0; i < READS; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        }
#pragma unroll
        for (int i = 0; i < LA + LW; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, MULS, 0);
        __builtin_amdgcn_sched_barrier(0);
    };

    issue_a(0, st[0]);
#pragma unroll
    for (int q = 1; q < S; ++q) {
        issue_a(q, st[q]);
        issue_w(q, st[q]);
    }
    wait_vmem<(S - 1) * (LA + LW)>();
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    read(st[0], 0, 0);
    int t = 0;
    for (; t + S <= nk; t += S) {
        step(t, lt_int<0>{});
        step(t + 1, lt_int<1>{});
        if constexpr (S > 2) step(t + 2, lt_int<2>{});
    }
    if (t < nk) step(t, lt_int<0>{});
    if constexpr (S > 2) if (t + 1 < nk) step(t + 1, lt_int<1>{});
    wait_vmem<0>(); // the loads past the last tile have landed before the workgroup ends

    // ---- epilogue.  Element e of lane (c, h): row 8 (e / 4) + 4 h + e % 4, column c of the 32 x 32 block.
    const int nw0 = n0 + 32 * wn * TO;      // the wave's first output column
    if (plan.part) {
        float* part = plan.part + (int64_t)split * p.rows * plan.ldpart;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int c = nw0 + 32 * (j % TO) + fr, n = j < TO ? c : plan.ldpart / 2 + c;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int row = m0 + 32 * (wm * TM + i) + 8 * (e / 4) + 4 * fh + e % 4;
                    if (row < mend && c < p.N) part[(int64_t)row * plan.ldpart + n] = acc[i][j][e];
                }
            }
        return;
    }
    // z = acc - C + bias where the accumulators are (a lane's column is the same for all its elements of a block: one
    // bias)
    float bias[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const int c = nw0 + 32 * (j % TO) + fr;
        bias[j] = p.bias && c < p.N ? p.bias[(int64_t)g.e * p.bias_stride + (j < TO ? 0 : p.N) + c] : 0.f;
    }
    // a 32-row block in LDS: columns of every second four rows 32 over, into the other half of the banks
    static_assert(32 * BN * 4 <= SB && WGM <= S, "a row block of each wave row fits a stage");
    auto z_at = [&](int r, int c) { return r * BN + (c ^ ((r >> 2 & 1) << 5)); };
    float* zb = nullptr;
#pragma unroll
    for (int q = 0; q < WGM; ++q)
        if (wm == q) zb = reinterpret_cast<float*>(st[q]);
    // the activation and the stores take rows of the wave row's block, 8 columns a lane: whole rows of the tile
    constexpr int BNO = T::BNO, CPL = 8, LPR = BNO / CPL, RPP = WAVE / LPR, RSTEP = WGN * RPP;
    static_assert(LPR <= WAVE && RSTEP <= 32, "columns of a row");
    const int pr = wn * RPP + lane / LPR, pc = lane % LPR * CPL, n = n0 + pc;
    const int left = p.N - n; // columns of the lane that exist
    // C of up to two row blocks of the wave ahead of both; elements outside load C[0].  (To wait for a load is to wait
    // for every store before it too.)
    constexpr int CB = TM < 2 ? TM : 2;
    float cv[CB][TN][16];
    auto load_c = [&](int i, int to) {
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int row = m0 + 32 * (wm * TM + i) + 8 * (e / 4) + 4 * fh + e % 4, c = nw0 + 32 * (j % TO) + fr;
                cv[to][j][e] = p.C[row < mend && c < p.N ? (int64_t)row * p.ldc + (j < TO ? 0 : p.N) + c : 0];
            }
    };
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int r0 = m0 + 32 * (wm * TM + i);
        if (p.C) {
            if (i % CB == 0) {
#pragma unroll
                for (int k = 0; k < CB; ++k) load_c(i + k, k);
            }
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] -= cv[i % CB][j][e];
        }
        lt_barrier(); // every wave is done with the stages, or with the row block before
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                zb[z_at(8 * (e / 4) + 4 * fh + e % 4, (j < TO ? 0 : BNO) + 32 * (wn * TO + j % TO) + fr)] =
                    p.bias ? acc[i][j][e] + bias[j] : acc[i][j][e];
        lt_barrier();
        const int rows_here = left > 0 ? min(32, mend - r0) : 0;
        auto finish = [&](int r, const float (&res)[CPL]) {
            float z[CPL], u[CPL];
#pragma unroll
            for (int c = 0; c < CPL / 4; ++c) {
                const f32x4_t a = *reinterpret_cast<const f32x4_t*>(zb + z_at(r, pc + 4 * c));
                const f32x4_t b = GATED ? *reinterpret_cast<const f32x4_t*>(zb + z_at(r, BNO + pc + 4 * c)) : a;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    z[4 * c + k] = a[k];
                    u[4 * c + k] = b[k];
                }
            }
            splitee::epi_finish<GATED, true>(p, z, u, res, r0 + r, n, left);
        };
        float res[CPL] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (!p.res) { // stores alone: with loads in the loop, each row would wait for the store before
#pragma unroll 1
            for (int r = pr; r < rows_here; r += RSTEP) finish(r, res);
        } else if (pr < rows_here) {
            splitee::epi_residual(p, r0 + pr, n, left, res);
#pragma unroll 1
            for (int r = pr; r < rows_here; r += RSTEP) {
                float next[CPL];
                splitee::epi_residual(p, r0 + min(r + RSTEP, rows_here - 1), n, left, next);
                finish(r, res);
#pragma unroll
                for (int k = 0; k < CPL; ++k) res[k] = next[k];
            }
        }
    }
}

// HALF: plan.nhalf workgroups take half tiles of BM / 2 rows, and so is a tile with at most BM / 2 rows computed: a partly
// filled round of workgroups then takes little more than half a round's time.  They come first, so that the CUs end
// their tiles, and write them, at different times.
template <int NPL, int BM, int BN, int WGM, int WGN, int S, bool GATED, bool TILED, bool HALF>
__global__ void __launch_bounds__(WGM * WGN * WAVE)
lin_tile_kernel(const LinArgs p, const LtPlan plan)
{
    using T = LinTile<NPL, BM, BN, WGM, WGN, S, GATED, TILED>;
    int L, split = 0, half = 0;
    if (p.offsets) {
        // 32 tiles in a row on one XCD, without the total, which only the offsets know (48000 rows of 64 experts, 96 in a row:
        // 417 us, 32: 346, 16: 350, 8: 360)
        constexpr int C = 32;
        const int b = blockIdx.x, x = b % 8, i = b / 8;
        L = (i / C) * (8 * C) + x * C + i % C;
    } else if (HALF && (int)blockIdx.x < plan.nhalf) {
        const int h = (int)splitee::xcd_logical_block(blockIdx.x, (uint32_t)plan.nhalf);
        L = h / 2;
        half = 1 + h % 2;
    } else {
        const uint32_t first = HALF ? (uint32_t)plan.nhalf : 0u;
        L = (int)splitee::xcd_logical_block(blockIdx.x - first, gridDim.x - first) + (int)first / 2;
        split = L % plan.ksplit;
        L /= plan.ksplit;
    }
    splitee::Group g;
    if (!splitee::find_group<BM>(p, L / plan.ntiles, g)) return;
    const int in = L - g.first * plan.ntiles;
    // eight row tiles times all columns at a time: the 32 tiles that an XCD has at once then share 8 + 4 operand tiles
    // (128 x 256 tiles of 4096 x 4096 x 2560: 89 -> 86 us)
    const int m1 = in / (8 * plan.ntiles) * 8, ms = min(8, g.tiles - m1), rest = in - m1 * plan.ntiles;
    int m0 = g.begin + (m1 + rest % ms) * BM, mend = min(m0 + BM, g.end);
    const int n0 = rest / ms * T::BNO;
    if constexpr (HALF) {
        if (half == 1) mend = min(mend, m0 + BM / 2);
        if (half == 2) m0 += BM / 2;
        if (m0 >= mend) return;
        if (mend - m0 <= BM / 2) {
            lin_tile<NPL, BM / 2, BN, WGM, WGN, S, GATED, TILED, T::SB>(p, plan, g, m0, n0, mend, split);
            return;
        }
    }
    lin_tile<NPL, BM, BN, WGM, WGN, S, GATED, TILED, T::SB>(p, plan, g, m0, n0, mend, split);
}

}  // namespace
