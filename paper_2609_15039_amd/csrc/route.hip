// Router of a mixture-of-experts layer and the weighted sum that ends it (gfx950): splitee_route and
// splitee_combine.
//
// Router.  A wave takes a token: its E logits lie in the lanes' registers (expert i in lane i % 64, register
// i / 64) as integers in the logits' order, and the k choices are k rounds of a wave-wide maximum by DPP (six
// instructions and a lane read; by shuffles through LDS the 8000 x 256 case took 71 us here), the lowest index among
// equals found by ballots, register by register.  The next token's logits are on their way meanwhile.  The rows of an
// expert are numbered by token without atomics whose order could show: a workgroup keeps for every expert a bit mask
// of its 64 tokens, so that a choice's place among the workgroup's rows is a population count, and the workgroups'
// counts are summed in order: for one workgroup in the same launch, up to 32 by each workgroup for itself, above by a
// launch of their own.
// Combine.  Bound by memory: each row read once, 16 bytes a lane, all of a token's rows in flight together.
#include "common.hpp"

namespace {

constexpr int RT_TOKENS = 64; // tokens of a workgroup: bits of a mask
constexpr int RT_WAVES = 16, RT_NT = RT_WAVES * 64;
constexpr int RT_MAX_E = 1024;
constexpr int RT_MAX_K = 64;
constexpr int RT_FEW = 32; // workgroups whose counts each of them sums itself

// lane 63: the maximum / the sum (in a fixed order) over the wave.  A lane without a source keeps its own value.
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp(int old, int v)
{
    return __builtin_amdgcn_update_dpp(old, v, CTRL, ROWS, 0xF, false);
}
__device__ __forceinline__ int wave_max(int v)
{
    v = max(v, dpp<0x111, 0xF>(v, v)); // row_shr:1, 2, 4, 8: lane 15 of each row of 16
    v = max(v, dpp<0x112, 0xF>(v, v));
    v = max(v, dpp<0x114, 0xF>(v, v));
    v = max(v, dpp<0x118, 0xF>(v, v));
    v = max(v, dpp<0x142, 0xA>(v, v)); // row_bcast:15 into rows 1 and 3, row_bcast:31 into rows 2 and 3
    v = max(v, dpp<0x143, 0xC>(v, v));
    return __builtin_amdgcn_readlane(v, 63);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_add(float v)
{
    return v + __int_as_float(dpp<CTRL, ROWS>(0, __float_as_int(v)));
}
__device__ __forceinline__ float wave_sum(float v)
{
    v = dpp_add<0x111, 0xF>(v);
    v = dpp_add<0x112, 0xF>(v);
    v = dpp_add<0x114, 0xF>(v);
    v = dpp_add<0x118, 0xF>(v);
    v = dpp_add<0x142, 0xA>(v);
    v = dpp_add<0x143, 0xC>(v);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// binary32 to integers of the same order and back; -0 counts as 0, -inf and NaN (masked experts) as the least
constexpr int RT_MASKED = INT32_MIN;
__device__ __forceinline__ int key_of(float x)
{
    const int b = __float_as_int(x + 0.0f);
    return x != x || x == -INFINITY ? RT_MASKED : b ^ ((b >> 31) & 0x7FFFFFFF);
}
__device__ __forceinline__ float of_key(int k) { return k == RT_MASKED ? -INFINITY : __int_as_float(k ^ ((k >> 31) & 0x7FFFFFFF)); }

// Exclusive sums over c(0) .. c(E - 1) to off, the total to off[E], by one wave.
template <typename F>
__device__ __forceinline__ void scan_experts(int E, int* off, F c)
{
    const int lane = threadIdx.x % 64;
    int before = 0;
    for (int e0 = 0; e0 < E; e0 += 64) {
        const int mine = e0 + lane < E ? c(e0 + lane) : 0;
        int incl = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int up = __shfl_up(incl, d, 64);
            if (lane >= d) incl += up;
        }
        if (e0 + lane < E) off[e0 + lane] = before + incl - mine;
        before += __shfl(incl, 63, 64);
    }
    if (lane == 0) off[E] = before;
}

// experts and weights.  One workgroup (ONE): the rest too.  More: slot holds each choice's place among its
// workgroup's rows of the expert, counts[b][e] the workgroup's rows of expert e.
template <int V, bool ONE>
__global__ void __launch_bounds__(RT_NT)
route_topk_kernel(const float* __restrict__ logits, int64_t ldl, int T, int E, int k, int score, int renorm,
                  int32_t* __restrict__ experts, float* __restrict__ weights, int32_t* __restrict__ slot,
                  int32_t* __restrict__ counts, int32_t* __restrict__ offsets, int32_t* __restrict__ row_index)
{
    __shared__ uint32_t mask[2][RT_MAX_E];
    __shared__ int16_t chosen[RT_TOKENS * RT_MAX_K];
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
    const int t0 = blockIdx.x * RT_TOKENS, tokens = min(RT_TOKENS, T - t0);
    for (int e = tid; e < E; e += RT_NT) mask[0][e] = mask[1][e] = 0u;
    float x[V];
    auto fetch = [&](int i) {
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = 64 * v + lane < E ? logits[(int64_t)(t0 + i) * ldl + 64 * v + lane] : -INFINITY;
    };
    if (wave < tokens) fetch(wave);
    __syncthreads();
    for (int i = wave; i < tokens; i += RT_WAVES) {
        const int64_t t = t0 + i;
        int l[V];
#pragma unroll
        for (int v = 0; v < V; ++v) l[v] = key_of(x[v]);
        if (i + RT_WAVES < tokens) fetch(i + RT_WAVES);
        float m = 0.f, total = 0.f;
        // lane j keeps choice j
        int mine = -1, best = RT_MASKED;
        for (int j = 0; j < k; ++j) {
            int top = l[0];
#pragma unroll
            for (int v = 1; v < V; ++v) top = max(top, l[v]);
            top = wave_max(top);
            if (top == RT_MASKED) break; // every expert left is masked
            if (j == 0) {
                m = of_key(top);
                if (score == SPLITEE_SCORE_SOFTMAX && !renorm) {
#pragma unroll
                    for (int v = 0; v < V; ++v) total += l[v] == RT_MASKED ? 0.f : expf(of_key(l[v]) - m);
                    total = wave_sum(total);
                }
            }
            int e = -1;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const uint64_t at = __ballot(l[v] == top);
                if (e < 0 && at) {
                    const int src = __ffsll((unsigned long long)at) - 1;
                    e = 64 * v + src;
                    if (lane == src) l[v] = RT_MASKED;
                }
            }
            if (lane == j) {
                mine = e;
                best = top;
            }
        }
        const float b = of_key(best);
        float w = mine < 0 ? 0.f : score == SPLITEE_SCORE_SOFTMAX ? expf(b - m) : 1.0f / (1.0f + expf(-b));
        if (renorm) total = wave_sum(w);
        if ((renorm || score == SPLITEE_SCORE_SOFTMAX) && total != 0.f) w = w / total;
        if (lane < k) {
            experts[t * k + lane] = mine;
            weights[t * k + lane] = mine < 0 ? 0.f : w;
            chosen[i * k + lane] = (int16_t)mine;
            if (mine >= 0) atomicOr(&mask[i / 32][mine], 1u << (i % 32));
        }
    }
    __syncthreads();
    __shared__ int off[ONE ? RT_MAX_E + 1 : 1];
    auto rows_of = [&](int e) { return __popc(mask[0][e]) + __popc(mask[1][e]); };
    if constexpr (ONE) {
        if (wave == 0) scan_experts(E, off, rows_of);
        __syncthreads();
        for (int e = tid; e <= E; e += RT_NT) offsets[e] = off[e];
        for (int r = off[E] + tid; r < T * k; r += RT_NT) row_index[r] = -1;
    } else {
        for (int e = tid; e < E; e += RT_NT) counts[(int64_t)blockIdx.x * E + e] = rows_of(e);
    }
    for (int a = tid; a < tokens * k; a += RT_NT) {
        const int i = a / k, e = chosen[a];
        int place = -1;
        if (e >= 0) {
            place = __popc(mask[i / 32][e] & ((1u << (i % 32)) - 1u));
            if (i >= 32) place += __popc(mask[0][e]);
            if constexpr (ONE) {
                place += off[e];
                row_index[place] = i;
            }
        }
        slot[(int64_t)t0 * k + a] = place;
    }
}

// Workgroup e: counts[b][e] to the rows of expert e in the workgroups before b; totals[e].
__global__ void __launch_bounds__(256) route_scan_kernel(int32_t* __restrict__ counts, int blocks, int E,
                                                         int32_t* __restrict__ totals)
{
    __shared__ int part[4];
    const int e = blockIdx.x, tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
    int before = 0;
    for (int b0 = 0; b0 < blocks; b0 += 256) {
        const int b = b0 + tid;
        const int c = b < blocks ? counts[(int64_t)b * E + e] : 0;
        int incl = c;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int up = __shfl_up(incl, d, 64);
            if (lane >= d) incl += up;
        }
        if (lane == 63) part[wave] = incl;
        __syncthreads();
        int base = before;
        for (int w = 0; w < wave; ++w) base += part[w];
        if (b < blocks) counts[(int64_t)b * E + e] = base + incl - c;
        before += part[0] + part[1] + part[2] + part[3];
        __syncthreads();
    }
    if (tid == 0) totals[e] = before;
}

// offsets from the totals, then every choice's row.  FEW: counts are the workgroups' own, else scanned.
template <bool FEW>
__global__ void __launch_bounds__(256) route_place_kernel(const int32_t* __restrict__ counts, const int32_t* __restrict__ totals,
                                                          int T, int E, int k, const int32_t* __restrict__ experts,
                                                          int32_t* __restrict__ offsets, int32_t* __restrict__ row_index,
                                                          int32_t* __restrict__ slot)
{
    __shared__ int off[RT_MAX_E + 1], before[RT_MAX_E], total[RT_MAX_E];
    const int tid = threadIdx.x, b = blockIdx.x;
    for (int e = tid; e < E; e += 256) {
        if constexpr (FEW) {
            int sum = 0, mine = 0;
#pragma unroll 8
            for (int q = 0; q < (int)gridDim.x; ++q) {
                if (q == b) mine = sum;
                sum += counts[(int64_t)q * E + e];
            }
            before[e] = mine;
            total[e] = sum;
        } else {
            before[e] = counts[(int64_t)b * E + e];
            total[e] = totals[e];
        }
    }
    __syncthreads();
    if (tid < 64) scan_experts(E, off, [&](int e) { return total[e]; });
    __syncthreads();
    if (b == 0)
        for (int e = tid; e <= E; e += 256) offsets[e] = off[e];
    const int64_t t0 = (int64_t)b * RT_TOKENS;
    const int64_t end = min(t0 + RT_TOKENS, (int64_t)T) * k;
    for (int64_t at = t0 * k + tid; at < end; at += 256) {
        const int e = experts[at];
        if (e < 0) continue; // slot is -1 already
        const int row = off[e] + before[e] + slot[at];
        slot[at] = row;
        row_index[row] = (int32_t)(at / k);
    }
    for (int64_t r = off[E] + (int64_t)b * 256 + tid; r < (int64_t)T * k; r += (int64_t)gridDim.x * 256) row_index[r] = -1;
}

__global__ void route_empty_kernel(int32_t* offsets, int E)
{
    for (int e = threadIdx.x; e <= E; e += blockDim.x) offsets[e] = 0;
}

// ------------------------------------------------------------------------ combine

constexpr int CB_NT = 256;
constexpr int CB_UNROLL = 8; // rows in flight

template <bool HB, bool YB>
__global__ void __launch_bounds__(CB_NT)
combine_kernel(const void* H, int64_t ldh, int64_t h_rows, const int32_t* __restrict__ slot,
               const float* __restrict__ weights, const void* res, int64_t ldres, void* Y, int64_t ldy, int k, int N)
{
    const int64_t t = blockIdx.x;
    const int n0 = (blockIdx.y * CB_NT + threadIdx.x) * 8;
    if (n0 >= N) return;
    const int width = min(8, N - n0);
    auto load8 = [&](const void* base, int64_t at, bool b16, float (&x)[8]) {
        if (width == 8) {
            if (b16) {
                const uint4 q = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(base) + at);
                const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[2 * i] = __uint_as_float(w[i] << 16);
                    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
                }
            } else {
                const float4 a = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(base) + at);
                const float4 b = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(base) + at + 4);
                x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
                x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                x[i] = i >= width ? 0.f
                       : b16 ? splitee::bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(base)[at + i])
                             : reinterpret_cast<const float*>(base)[at + i];
        }
    };
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int j0 = 0; j0 < k; j0 += CB_UNROLL) {
        int row[CB_UNROLL];
        float w[CB_UNROLL], x[CB_UNROLL][8];
#pragma unroll
        for (int j = 0; j < CB_UNROLL; ++j) {
            const bool in = j0 + j < k;
            row[j] = in ? slot[t * k + j0 + j] : -1;
            w[j] = in ? weights[t * k + j0 + j] : 0.f;
            if (row[j] >= h_rows) row[j] = -1;
        }
#pragma unroll
        for (int j = 0; j < CB_UNROLL; ++j)
            if (row[j] >= 0) load8(H, (int64_t)row[j] * ldh + n0, HB, x[j]);
#pragma unroll
        for (int j = 0; j < CB_UNROLL; ++j)
            if (row[j] >= 0) {
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[i] = fmaf(w[j], x[j][i], acc[i]);
            }
    }
    if (res) {
        float x[8];
        load8(res, t * ldres + n0, YB, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] += x[i];
    }
    if (YB) {
        uint16_t* y = reinterpret_cast<uint16_t*>(Y) + t * ldy + n0;
        if (width == 8) {
            *reinterpret_cast<uint4*>(y) = make_uint4(splitee::bf16x2_rne(acc[0], acc[1]), splitee::bf16x2_rne(acc[2], acc[3]),
                                                      splitee::bf16x2_rne(acc[4], acc[5]), splitee::bf16x2_rne(acc[6], acc[7]));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < width) y[i] = (uint16_t)splitee::bf16_bits_rne(acc[i]);
        }
    } else {
        float* y = reinterpret_cast<float*>(Y) + t * ldy + n0;
        if (width == 8) {
            *reinterpret_cast<float4*>(y) = make_float4(acc[0], acc[1], acc[2], acc[3]);
            *reinterpret_cast<float4*>(y + 4) = make_float4(acc[4], acc[5], acc[6], acc[7]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < width) y[i] = acc[i];
        }
    }
}

}  // namespace

namespace splitee_host {

// per workgroup of 64 tokens and expert one count, then the experts' totals
size_t route_workspace_bytes(int64_t T, int64_t E)
{
    return (size_t)((T + RT_TOKENS - 1) / RT_TOKENS + 1) * (size_t)E * 4;
}

int launch_route(const float* logits, int64_t ldl, int64_t T, int64_t E, int64_t k, int score, int renorm,
                 int32_t* experts, float* weights, int32_t* offsets, int32_t* row_index, int32_t* slot, void* ws,
                 hipStream_t s)
{
    if (T == 0) {
        hipLaunchKernelGGL(route_empty_kernel, dim3(1), dim3(256), 0, s, offsets, (int)E);
        return hipGetLastError() == hipSuccess ? SPLITEE_OK : SPLITEE_ERR_HIP;
    }
    const int blocks = (int)((T + RT_TOKENS - 1) / RT_TOKENS);
    int32_t* counts = reinterpret_cast<int32_t*>(ws);
    int32_t* totals = counts + (int64_t)blocks * E;
#define RT_RUN(V, ONE)                                                                                                \
    hipLaunchKernelGGL((route_topk_kernel<V, ONE>), dim3(blocks), dim3(RT_NT), 0, s, logits, ldl, (int)T, (int)E, (int)k, score, \
                       renorm, experts, weights, slot, counts, offsets, row_index)
#define RT(V) if (blocks == 1) RT_RUN(V, true); else RT_RUN(V, false)
    if (E <= 64) { RT(1); } else if (E <= 128) { RT(2); } else if (E <= 256) { RT(4); } else if (E <= 512) { RT(8); } else { RT(16); }
#undef RT
#undef RT_RUN
    if (blocks > 1 && blocks <= RT_FEW) {
        hipLaunchKernelGGL(route_place_kernel<true>, dim3(blocks), dim3(256), 0, s, counts, totals, (int)T, (int)E, (int)k, experts,
                           offsets, row_index, slot);
    } else if (blocks > 1) {
        hipLaunchKernelGGL(route_scan_kernel, dim3((unsigned)E), dim3(256), 0, s, counts, blocks, (int)E, totals);
        hipLaunchKernelGGL(route_place_kernel<false>, dim3(blocks), dim3(256), 0, s, counts, totals, (int)T, (int)E, (int)k, experts,
                           offsets, row_index, slot);
    }
    return hipGetLastError() == hipSuccess ? SPLITEE_OK : SPLITEE_ERR_HIP;
}

int launch_combine(const void* H, bool h_bf16, int64_t ldh, int64_t h_rows, const int32_t* slot, const float* weights,
                   const void* res, int64_t ldres, void* Y, bool y_bf16, int64_t ldy, int64_t T, int64_t k, int64_t N,
                   hipStream_t s)
{
    const dim3 grid((unsigned)T, (unsigned)((N + 8 * CB_NT - 1) / (8 * CB_NT)));
#define CB(HB, YB) \
    hipLaunchKernelGGL((combine_kernel<HB, YB>), grid, dim3(CB_NT), 0, s, H, ldh, h_rows, slot, weights, res, ldres, Y, ldy, (int)k, (int)N)
    if (h_bf16) { if (y_bf16) CB(true, true); else CB(true, false); }
    else { if (y_bf16) CB(false, true); else CB(false, false); }
#undef CB
    return hipGetLastError() == hipSuccess ? SPLITEE_OK : SPLITEE_ERR_HIP;
}

}  // namespace splitee_host
