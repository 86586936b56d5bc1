// Router of a mixture-of-experts layer and the weighted sum that ends it (gfx950): splitee_route and
// splitee_combine.
//
// Router.  A wave takes two tokens: the E logits of each lie in the lanes' registers as integers in the logits' order,
// consecutive experts in a lane, which sorts its own once.  The k choices are k rounds of a maximum of the lanes' heads by
// DPP (six instructions and a lane read), the lowest lane among equals found by a ballot, and a shift in that lane: about
// 20 vector instructions a choice, which is what bounds it.  (8000 x 256: 71 us with the maxima by shuffles through
// LDS, 11 us without the sorting, where each choice looked through all registers.)  The rows of an
// expert are numbered by token without atomics whose order could show: a workgroup keeps for every expert a bit mask
// of its tokens, so that a choice's place among the workgroup's rows is a population count, and the workgroups'
// counts are summed in order: for one workgroup in the same launch, up to 32 by each workgroup for itself, above by a
// launch of their own.
// 8000 x 256, 8 choices: 9 us for the choices, 8 for the two launches that place them; one token 3.7 us.
// Combine.  Bound by memory: each row read once, 16 bytes a lane, all of a token's rows in flight together.  6000 tokens of 8
// rows x 2048 bfloat16 with the residual 50 us (4.5 TB/s read and written; a copy reaches 4.7).
#include "common.hpp"

namespace {

constexpr int RT_ONE = 64;    // most tokens of a launch of one workgroup
constexpr int RT_TOKENS = 32; // tokens of a workgroup of several: two for each wave, and enough workgroups for the chip
constexpr int RT_WAVES = 16, RT_NT = RT_WAVES * 64;
constexpr int RT_MAX_E = 1024;
constexpr int RT_MAX_K = 64;
constexpr int RT_FEW = 32; // workgroups whose counts each of them sums itself

// The maximum / the sum (in a fixed order) over the wave, which lane 63 ends with.
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp(int old, int v)
{
    return __builtin_amdgcn_update_dpp(old, v, CTRL, ROWS, 0xF, false);
}
__device__ __forceinline__ void wave_max(int& a, int& b)
{
    // (a lane without a source gets the least integer, which the compiler folds into one v_max_i32_dpp)
#define RT_STEP(CTRL, ROWS) a = max(a, dpp<CTRL, ROWS>(INT32_MIN, a)); b = max(b, dpp<CTRL, ROWS>(INT32_MIN, b))
    RT_STEP(0x111, 0xF); // row_shr:1, 2, 4, 8: lane 15 of each row of 16
    RT_STEP(0x112, 0xF);
    RT_STEP(0x114, 0xF);
    RT_STEP(0x118, 0xF);
    RT_STEP(0x142, 0xA); // row_bcast:15 into rows 1 and 3, row_bcast:31 into rows 2 and 3
    RT_STEP(0x143, 0xC);
#undef RT_STEP
    a = __builtin_amdgcn_readlane(a, 63);
    b = __builtin_amdgcn_readlane(b, 63);
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
    constexpr int TOKENS = ONE ? RT_ONE : RT_TOKENS;
    __shared__ uint32_t mask[TOKENS / 32][RT_MAX_E];
    __shared__ int16_t chosen[TOKENS * RT_MAX_K];
    const int tid = threadIdx.x, lane = tid % 64, wave = tid / 64;
    const int t0 = blockIdx.x * TOKENS, tokens = min(TOKENS, T - t0);
    for (int e = tid; e < E; e += RT_NT) mask[0][e] = mask[TOKENS / 32 - 1][e] = 0u;
    __syncthreads();
    // two tokens at a time: one's instructions fill the waits of the other's
    for (int i0 = 2 * wave; i0 < tokens; i0 += 2 * RT_WAVES) {
        // a lane has experts V lane .. V lane + V - 1, largest first and equal ones by rising index: l[.][0] is its
        // head, of[.][v] the place of l[.][v] among them
        int l[2][V], of[2][V], mine[2], best[2];
        float m[2] = {0.f, 0.f}, total[2] = {0.f, 0.f}, x[2][V];
        // every load unconditional (past the experts: the last), so that they are in flight together
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int v = 0; v < V; ++v)
                x[q][v] = logits[(int64_t)(t0 + min(i0 + q, tokens - 1)) * ldl + min(V * lane + v, E - 1)];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            mine[q] = -1; // lane j keeps choice j
            best[q] = RT_MASKED;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                l[q][v] = V * lane + v < E ? key_of(x[q][v]) : RT_MASKED;
                of[q][v] = v;
            }
#pragma unroll
            for (int n = V - 1; n > 0; --n) // exchanges of neighbours, which leave equal ones in their order
#pragma unroll
                for (int v = 0; v < n; ++v) {
                    const bool swap = l[q][v] < l[q][v + 1];
                    const int big = max(l[q][v], l[q][v + 1]), low = min(l[q][v], l[q][v + 1]);
                    const int ob = swap ? of[q][v + 1] : of[q][v], ol = swap ? of[q][v] : of[q][v + 1];
                    l[q][v] = big; l[q][v + 1] = low;
                    of[q][v] = ob; of[q][v + 1] = ol;
                }
        }
        for (int j = 0; j < k; ++j) {
            int top[2] = {l[0][0], l[1][0]};
            wave_max(top[0], top[1]);
            if (j == 0) {
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    m[q] = of_key(top[q]);
                    if (score == SPLITEE_SCORE_SOFTMAX && !renorm) {
#pragma unroll
                        for (int v = 0; v < V; ++v) total[q] += l[q][v] == RT_MASKED ? 0.f : expf(of_key(l[q][v]) - m[q]);
                        total[q] = wave_sum(total[q]);
                    }
                }
            }
            if (top[0] == RT_MASKED && top[1] == RT_MASKED) break; // every expert left is masked
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int src = __ffsll((unsigned long long)__ballot(l[q][0] == top[q])) - 1; // the lowest of equal ones
                const int e = V * src + __builtin_amdgcn_readlane(of[q][0], src);
                const bool taken = lane == src;
#pragma unroll
                for (int v = 0; v + 1 < V; ++v) {
                    l[q][v] = taken ? l[q][v + 1] : l[q][v];
                    of[q][v] = taken ? of[q][v + 1] : of[q][v];
                }
                l[q][V - 1] = taken ? RT_MASKED : l[q][V - 1];
                if (lane == j && top[q] != RT_MASKED) {
                    mine[q] = e;
                    best[q] = top[q];
                }
            }
        }
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int i = i0 + q;
            if (i >= tokens) break;
            const int64_t t = t0 + i;
            const float b = of_key(best[q]);
            // of low sigmoids only the quotients matter, which exp(-m) times each has too: exp(-b) overflows from 88.7 on
            const bool soft = score == SPLITEE_SCORE_SOFTMAX, low = !soft && renorm && m[q] < 0.f;
            float w = soft || low ? expf(b - m[q]) : 1.0f;
            if (!soft) w = low && b < -700.f ? 0.f : w / (1.0f + expf(low ? b : -b));
            if (mine[q] < 0) w = 0.f;
            const float sum = renorm ? wave_sum(w) : total[q];
            if ((renorm || soft) && sum != 0.f) w = w / sum;
            if (lane < k) {
                experts[t * k + lane] = mine[q];
                weights[t * k + lane] = mine[q] < 0 ? 0.f : w;
                chosen[i * k + lane] = (int16_t)mine[q];
                if (mine[q] >= 0) atomicOr(&mask[i / 32][mine[q]], 1u << (i % 32));
            }
        }
    }
    __syncthreads();
    __shared__ int off[ONE ? RT_MAX_E + 1 : 1];
    auto rows_of = [&](int e) { return __popc(mask[0][e]) + (ONE ? __popc(mask[TOKENS / 32 - 1][e]) : 0); };
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
            if constexpr (ONE) {
                if (i >= 32) place += __popc(mask[0][e]);
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

// per workgroup and expert one count, then the experts' totals
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
    const int blocks = T <= RT_ONE ? 1 : (int)((T + RT_TOKENS - 1) / RT_TOKENS);
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
