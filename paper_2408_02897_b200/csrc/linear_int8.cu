// The products of a layer whose codes are INT8 (qm_linear_int8, qm_gated_linear_int8):
//   y_ij = (sum_k x_ik w_jk) dx_i dw_j + bias_j          the sum in int32, exact
//   h_ij = act(g_ij) u_ij, g and u two such products     of the same x
// written in bf16 or fp32.
#include <cuda_bf16.h>

#include "qm_internal.h"

namespace qm {
namespace {

constexpr int kTile = 64, kChunk = 64;         // outputs per side of a block's tile, contraction entries per step

// act(g) in fp32.  The tanh form is g / (1 + exp(-2 t)), t the tanh's argument: 1/2 (1 + tanh t) is that quotient, and
// unlike 1 + tanhf(t) it keeps its relative precision where t is negative.
__device__ __forceinline__ float activate(float g, int act) {
  if (act == QM_ACT_GELU) return 0.5f * g * (1.f + erff(g * 0.70710678f));
  const float t = act == QM_ACT_SILU ? g : 1.5957691f * fmaf(0.044715f * g * g, g, g);
  return g / (1.f + expf(-t));
}

__device__ __forceinline__ int load4(const uint8_t* row, int k, int K) {
  uint32_t v = 0;
  for (int i = 0; i < 4; ++i) v |= (k + i < K ? (uint32_t)row[k + i] : 0u) << (8 * i);
  return (int)v;
}

template <typename T, bool GATED>
__global__ void __launch_bounds__(256) linear_tile(const LinearArgs a) {
  pdl_prologue();
  __shared__ int sx[kChunk / 4][kTile + 1], sw[GATED ? 2 : 1][kChunk / 4][kTile + 1];
  const int64_t m0 = (int64_t)blockIdx.y * kTile, n0 = (int64_t)blockIdx.x * kTile;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  int acc[GATED ? 2 : 1][4][4] = {};
  for (int k0 = 0; k0 < a.K; k0 += kChunk) {
    for (int i = threadIdx.x; i < kTile * kChunk / 4; i += 256) {
      const int row = i / (kChunk / 4), c = i % (kChunk / 4);
      sx[c][row] = m0 + row < a.M ? load4(a.x + (m0 + row) * a.ld_x, k0 + 4 * c, (int)a.K) : 0;
#pragma unroll
      for (int p = 0; p < (GATED ? 2 : 1); ++p)
        sw[p][c][row] = n0 + row < a.N ? load4(a.w[p] + (n0 + row) * a.ld_w[p], k0 + 4 * c, (int)a.K) : 0;
    }
    __syncthreads();
    for (int c = 0; c < kChunk / 4; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int p = 0; p < (GATED ? 2 : 1); ++p)
            acc[p][i][j] = __dp4a(sx[c][ty + 16 * i], sw[p][c][tx + 16 * j], acc[p][i][j]);
    __syncthreads();
  }
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int64_t m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
      if (m >= a.M || n >= a.N) continue;
      float y = (float)acc[0][i][j] * (a.dx[m] * a.dw[0][n]);
      if (GATED) y = activate(y, a.act) * ((float)acc[GATED ? 1 : 0][i][j] * (a.dx[m] * a.dw[1][n]));
      else if (a.bias) y += a.bias_dtype == QM_DT_BF16 ? (float)static_cast<const __nv_bfloat16*>(a.bias)[n]
                                                       : static_cast<const float*>(a.bias)[n];
      static_cast<T*>(a.out)[m * a.ld_out + n] = (T)y;
    }
}

}  // namespace

qm_status launch_linear_int8(const LinearArgs& a, cudaStream_t s) {
  const bool gated = a.w[1] != nullptr, bf16 = a.out_dtype == QM_DT_BF16;
  auto kern = gated ? (bf16 ? linear_tile<__nv_bfloat16, true> : linear_tile<float, true>)
                    : (bf16 ? linear_tile<__nv_bfloat16, false> : linear_tile<float, false>);
  const int64_t tiles_m = (a.M + kTile - 1) / kTile, tiles_n = (a.N + kTile - 1) / kTile;
  if (tiles_m > 65535) return QM_ERR_UNSUPPORTED;
  QM_CUDA_OK(launch_pdl(kern, dim3((unsigned)tiles_n, (unsigned)tiles_m), dim3(256), 0, s, a));
  count_launch();
  return QM_OK;
}

}  // namespace qm
