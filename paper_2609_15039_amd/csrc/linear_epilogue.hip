// Products with an epilogue, dense and by expert (gfx950): splitee_linear_epilogue and
// splitee_grouped_linear.
//
//   Z = fl32(A W^T) - C + bias;  H = act(Z) or act(Z_gate) Z_up;  Y = round(H + residual)
#include "epilogue_dev.hpp"

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
    int e, m0, mend;
    if ((int)blockIdx.y >= splitee::find_tile<LS_T>(p, blockIdx.y, e, m0, mend)) return;
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

}  // namespace

namespace splitee_host {

size_t linear_workspace_bytes(int64_t, int64_t, int64_t, int, int) { return 0; }

int launch_linear(const LinArgs& p, int prec, int w_type, void*, hipStream_t s)
{
    // row tiles of all groups: at most one partly filled one each
    const int64_t tiles = p.offsets ? p.rows / LS_T + p.experts : (p.rows + LS_T - 1) / LS_T;
    hipLaunchKernelGGL(linear_simple_kernel, dim3((unsigned)((p.N + LS_T - 1) / LS_T), (unsigned)tiles),
                       dim3(LS_T * LS_T), 0, s, p, prec, w_type);
    return hipGetLastError() == hipSuccess ? SPLITEE_OK : SPLITEE_ERR_HIP;
}

}  // namespace splitee_host
