// The epilogue of a projection and the rows of a group, shared by the kernels of splitee_linear_epilogue
// and splitee_grouped_linear (gfx950).
#pragma once
#include "common.hpp"

namespace splitee {

// One product with its epilogue, dense (offsets null: one group of all rows) or by expert.  Strides
// in elements.
struct LinArgs {
    const void* A; int64_t lda, pstride; int a_rows;
    const int32_t* row_index;
    const int32_t* offsets; int experts;
    const void* W; int64_t ldw, w_stride;
    const float* C; int64_t ldc;
    const float* bias; int64_t bias_stride;
    const void* res; int64_t ldres;
    void* Y; int64_t ldy;
    int act, gated, out_bf16;
    int rows, N, K;
};

// act(z) in binary32.  The logistic function 1 / (1 + exp(-x)) takes one hardware exponential of base 2 and one
// hardware reciprocal (1 unit in the last place each; the product x log2 e is rounded, |x| 2^-24 of the
// exponential, which matters where that is not small against 1: |x| below 17), a dozen instructions fewer than expf
// and a division; tanh in the GELU's approximation is (1 + tanh u) / 2 = 1 / (1 + exp(-2 u)), without the cancellation
// of 1 + tanh u.  A NaN passes through each.
__device__ __forceinline__ float epi_logistic(float x)
{
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896341f * x));
}
// The normal distribution Phi(z) = (1 + erf(z / sqrt 2)) / 2 of the GELU: 1/2 + z p(z^2) for |z| < 1.4, beyond exp(-z^2 / 2) t q(t),
// t = 1 / (1 + 0.41 |z|), or 1 less that.  p and q are minimax polynomials fitted to erf and to exp(x^2) erfc(x) in 64 bits,
// off by 0.03 and 0.5 2^-24 of Phi.  With the roundings Phi is off by 12 2^-24 of itself at most and, below -1.4, by
// 1.2 z^2 2^-24 more of it for the exponent's (measured: 6, and 14 from -4 to -3), so that the GELU's error is no larger than that
// of the formula step by step in binary32 (root mean square from -3 to -2: 2.9e-9 against 2.2e-8).  4096 x 12288 outputs
// of 2560 products take 259 us; with the device library's erff 268, its erfcf 286, a five-term erfc off by 1.5e-7 255.
__device__ __forceinline__ float epi_normal(float z)
{
    const float s = z * z, t = __builtin_amdgcn_rcpf(fmaf(0.41f, fabsf(z), 1.0f));
    float p = fmaf(4.8862097e-07f, s, -9.20364e-06f);
    p = fmaf(p, s, 0.00011552812f);
    p = fmaf(p, s, -0.0011878415f);
    p = fmaf(p, s, 0.009973998f);
    p = fmaf(p, s, -0.066490516f);
    p = fmaf(p, s, 0.3989423f);
    float q = fmaf(0.07622011f, t, -0.19209301f);
    q = fmaf(q, t, 0.092467114f);
    q = fmaf(q, t, 0.057039957f);
    q = fmaf(q, t, 0.14024942f);
    q = fmaf(q, t, 0.16317481f);
    q = fmaf(q, t, 0.16358161f) * t * __builtin_amdgcn_exp2f(-0.72134752f * s); // log2 e / 2
    return fabsf(z) < 1.4f ? fmaf(z, p, 0.5f) : z < 0.0f ? q : 1.0f - q;
}
template <int ACT>
__device__ __forceinline__ float epi_act1(float z)
{
    if (ACT == SPLITEE_ACT_SILU) return z * epi_logistic(z);
    if (ACT == SPLITEE_ACT_GELU_TANH) return z * epi_logistic(1.59576912160573071f * (z + 0.044715f * z * z * z));
    if (ACT == SPLITEE_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if (ACT == SPLITEE_ACT_GELU) return z * epi_normal(z);
    return z;
}
// of n values, one choice for all
template <int N>
__device__ __forceinline__ void epi_act(float (&z)[N], int act)
{
#define EPI_CASE(A)                                             \
    case A:                                                     \
        _Pragma("unroll") for (int i = 0; i < N; ++i) z[i] = epi_act1<A>(z[i]); \
        break
    switch (act) {
        EPI_CASE(SPLITEE_ACT_SILU);
        EPI_CASE(SPLITEE_ACT_GELU);
        EPI_CASE(SPLITEE_ACT_GELU_TANH);
        EPI_CASE(SPLITEE_ACT_RELU);
    default: break;
    }
#undef EPI_CASE
}

// fl32(r - C) + bias of one element of the product: weight row n of group e, output row `row`
__device__ __forceinline__ float epi_z(const LinArgs& p, float r, int e, int row, int n)
{
    if (p.C) r = r - p.C[(int64_t)row * p.ldc + n];
    if (p.bias) r = r + p.bias[(int64_t)e * p.bias_stride + n];
    return r;
}

__device__ __forceinline__ void epi_store(const LinArgs& p, float h, int row, int n)
{
    if (p.out_bf16) {
        if (p.res) h += bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(p.res)[(int64_t)row * p.ldres + n]);
        reinterpret_cast<uint16_t*>(p.Y)[(int64_t)row * p.ldy + n] = (uint16_t)bf16_bits_rne(h);
    } else {
        if (p.res) h += reinterpret_cast<const float*>(p.res)[(int64_t)row * p.ldres + n];
        reinterpret_cast<float*>(p.Y)[(int64_t)row * p.ldy + n] = h;
    }
}

// N (4 or 8) columns of a row of the residual from column n on (left of them exist), zeros without one.
template <int N>
__device__ __forceinline__ void epi_residual(const LinArgs& p, int row, int n, int left, float (&r)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = 0.f;
    if (!p.res) return;
    const int64_t at = (int64_t)row * p.ldres + n;
    if (p.out_bf16) {
        const uint16_t* q = reinterpret_cast<const uint16_t*>(p.res) + at;
        if (left >= N) {
#pragma unroll
            for (int c = 0; c < N / 4; ++c) {
                const uint2 v = reinterpret_cast<const uint2*>(q)[c];
                r[4 * c] = __uint_as_float(v.x << 16);
                r[4 * c + 1] = __uint_as_float(v.x & 0xFFFF0000u);
                r[4 * c + 2] = __uint_as_float(v.y << 16);
                r[4 * c + 3] = __uint_as_float(v.y & 0xFFFF0000u);
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < left) r[i] = bf16_bits_to_f32(q[i]);
    } else {
        const float* q = reinterpret_cast<const float*>(p.res) + at;
        if (left >= N) {
#pragma unroll
            for (int c = 0; c < N / 4; ++c) {
                const f32x4_t v = reinterpret_cast<const f32x4_t*>(q)[c];
#pragma unroll
                for (int i = 0; i < 4; ++i) r[4 * c + i] = v[i];
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < left) r[i] = q[i];
    }
}

// The activation of N (4 or 8) z of a row, the gate's product with up (gated), the residual's sum and the store, from
// column n on; left: columns that exist (N and more: 8- or 16-byte stores).  STREAM: stores that do not stay in the L2, for
// results larger than it (4096 x 4096 bfloat16: 2 us less).
template <bool GATED, bool STREAM, int N>
__device__ __forceinline__ void epi_finish(const LinArgs& p, float (&h)[N], const float (&up)[N], const float (&res)[N], int row, int n,
                                           int left)
{
    epi_act(h, p.act);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (GATED) h[i] *= up[i];
        if (p.res) h[i] += res[i]; // (-0 stays -0 without one)
    }
    const int64_t at = (int64_t)row * p.ldy + n;
    if (p.out_bf16) {
        typedef uint32_t words_t __attribute__((ext_vector_type(N / 2)));
        uint16_t* y = reinterpret_cast<uint16_t*>(p.Y) + at;
        words_t v;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) v[i] = bf16x2_rne(h[2 * i], h[2 * i + 1]);
        if (left >= N) {
            if (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<words_t*>(y));
            else *reinterpret_cast<words_t*>(y) = v;
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (i < left) y[i] = (uint16_t)(v[i / 2] >> (16 * (i % 2)));
        }
    } else {
        float* y = reinterpret_cast<float*>(p.Y) + at;
        if (left >= N) {
#pragma unroll
            for (int c = 0; c < N / 4; ++c) {
                const f32x4_t v = {h[4 * c], h[4 * c + 1], h[4 * c + 2], h[4 * c + 3]};
                if (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<f32x4_t*>(y) + c);
                else reinterpret_cast<f32x4_t*>(y)[c] = v;
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (i < left) y[i] = h[i];
        }
    }
}

// Group e's rows: begin .. end - 1, within 0 .. rows whatever offsets holds.
__device__ __forceinline__ void group_rows(const LinArgs& p, int e, int& begin, int& end)
{
    begin = min(max(p.offsets[e], 0), p.rows);
    end = min(max(p.offsets[e + 1], begin), p.rows);
}

// Inclusive sums over the lanes of the wave, by DPP.
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_plus(int v)
{
    return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, false);
}
__device__ __forceinline__ int wave_scan(int v)
{
    v = dpp_plus<0x111, 0xF>(v); // row_shr:1, 2, 4, 8
    v = dpp_plus<0x112, 0xF>(v);
    v = dpp_plus<0x114, 0xF>(v);
    v = dpp_plus<0x118, 0xF>(v);
    v = dpp_plus<0x142, 0xA>(v); // row_bcast:15, row_bcast:31
    return dpp_plus<0x143, 0xC>(v);
}

// The group that holds row tile `at` of BM rows, the row tiles of all groups counted one group after
// another, found by the whole wave: lanes take 64 groups at a time and scan their tile counts.  False where at
// is past the last tile.  The offsets are read by every wave of a launch, a few hundred bytes from L2.
struct Group {
    int e, begin, end; // the group and its rows
    int first, tiles;  // its first row tile and how many it has
};
template <int BM>
__device__ __forceinline__ bool find_group(const LinArgs& p, int at, Group& g)
{
    if (!p.offsets) {
        g = Group{0, 0, p.rows, 0, (p.rows + BM - 1) / BM};
        return at < g.tiles;
    }
    const int lane = threadIdx.x % 64;
    int before = 0;
    for (int e0 = 0; e0 < p.experts; e0 += 64) {
        int begin = 0, end = 0;
        if (e0 + lane < p.experts) group_rows(p, e0 + lane, begin, end);
        const int tiles = (end - begin + BM - 1) / BM;
        const int incl = wave_scan(tiles), first = before + incl - tiles;
        const uint64_t mine = __ballot(at >= first && at < first + tiles);
        if (mine) {
            const int src = __ffsll((unsigned long long)mine) - 1;
            g.e = __builtin_amdgcn_readfirstlane(e0 + src);
            g.begin = __builtin_amdgcn_readlane(begin, src);
            g.end = __builtin_amdgcn_readlane(end, src);
            g.first = __builtin_amdgcn_readlane(first, src);
            g.tiles = __builtin_amdgcn_readlane(tiles, src);
            return true;
        }
        before = __builtin_amdgcn_readlane(before + incl, 63);
    }
    return false;
}

// Row of A of output row s.
__device__ __forceinline__ int64_t a_row(const LinArgs& p, int s)
{
    return p.row_index ? min(max(p.row_index[s], 0), p.a_rows - 1) : s;
}

}  // namespace splitee
