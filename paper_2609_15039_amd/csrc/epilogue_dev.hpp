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

// act(z) in binary32.  expf, erff and tanhf are the device library's (a few units in the last place);
// a NaN passes through each.
__device__ __forceinline__ float epi_act(float z, int act)
{
    switch (act) {
    case SPLITEE_ACT_SILU: return z / (1.0f + expf(-z));
    case SPLITEE_ACT_GELU: return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
    case SPLITEE_ACT_GELU_TANH: return 0.5f * z * (1.0f + tanhf(0.79788456080286536f * (z + 0.044715f * z * z * z)));
    case SPLITEE_ACT_RELU: return z < 0.0f ? 0.0f : z;
    default: return z;
    }
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

// Group e's rows: begin .. end - 1, within 0 .. rows whatever offsets holds.
__device__ __forceinline__ void group_rows(const LinArgs& p, int e, int& begin, int& end)
{
    begin = min(max(p.offsets[e], 0), p.rows);
    end = min(max(p.offsets[e + 1], begin), p.rows);
}

// The tile of BM rows at place `at` of the row tiles of all groups, counted group by group, found by the
// whole wave: lanes take 64 groups at a time and scan their tile counts.  Returns the number of tiles of all
// groups; e, m0 and mend (the tile's first row, the group's end) are set where at is below it.  The
// offsets are read by every wave of a launch, a few hundred bytes from L2.
template <int BM>
__device__ __forceinline__ int find_tile(const LinArgs& p, int at, int& e, int& m0, int& mend)
{
    if (!p.offsets) {
        e = 0;
        m0 = at * BM;
        mend = p.rows;
        return (p.rows + BM - 1) / BM;
    }
    const int lane = threadIdx.x % 64;
    int total = 0;
    e = -1;
    for (int e0 = 0; e0 < p.experts; e0 += 64) {
        const int g = e0 + lane;
        int begin = 0, end = 0;
        if (g < p.experts) group_rows(p, g, begin, end);
        const int tiles = (end - begin + BM - 1) / BM;
        int incl = tiles;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int up = __shfl_up(incl, d, 64);
            if (lane >= d) incl += up;
        }
        const int first = total + incl - tiles; // this group's first tile
        const uint64_t mine = __ballot(at >= first && at < first + tiles);
        if (mine) {
            const int src = __ffsll((unsigned long long)mine) - 1;
            e = e0 + src;
            m0 = __shfl(begin + (at - first) * BM, src, 64);
            mend = __shfl(end, src, 64);
        }
        total += __shfl(incl, 63, 64);
    }
    return total;
}

// Row of A of output row s.
__device__ __forceinline__ int64_t a_row(const LinArgs& p, int s)
{
    return p.row_index ? min(max(p.row_index[s], 0), p.a_rows - 1) : s;
}

}  // namespace splitee
