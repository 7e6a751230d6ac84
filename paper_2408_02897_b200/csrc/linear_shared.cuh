// What the products of a layer share (linear_int8.cu, linear_fp8.cu): the blocks that they stage, two-wide fp32 arithmetic, the give-up
// path's waits, stores of outputs, tensor maps and launches.  Included by .cu files only; everything sits in the including file's
// anonymous namespace.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>

#include "qm_internal.h"
#include "tc_ptx.cuh"

namespace qm {
namespace {

constexpr int kBlock = 128;                               // rows of a staged block, and its contraction entries
constexpr uint32_t kBlockBytes = kBlock * kBlock;         // 16 KB
constexpr int kEpiWarps = 8;
constexpr int kThreads = 64 + 32 * kEpiWarps;             // TMA warp, MMA warp, epilogue

struct Waits { uint64_t limit_ns; uint32_t stop_after; };

// Two fp32 values per register pair: one instruction for both.
__device__ __forceinline__ uint64_t pair_of(float lo, float hi) { uint64_t v; asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi)); return v; }
__device__ __forceinline__ void halves(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t add2(uint64_t x, uint64_t y) { uint64_t d; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(x), "l"(y)); return d; }
__device__ __forceinline__ uint64_t mul2(uint64_t x, uint64_t y) { uint64_t d; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(x), "l"(y)); return d; }
__device__ __forceinline__ uint64_t fma2(uint64_t x, uint64_t y, uint64_t z) { uint64_t d; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(x), "l"(y), "l"(z)); return d; }
__device__ __forceinline__ uint64_t both(float v) { return pair_of(v, v); }

// A wait of the give-up path, whatever the CTA has been flagged with.
__device__ __forceinline__ void wait_limited(uint32_t bar, uint32_t parity, uint64_t limit_ns) {
  const uint64_t t0 = global_timer_ns();
  while (!mbar_try_wait(bar, parity) && global_timer_ns() - t0 < limit_ns) {}
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }

__device__ __forceinline__ float nan_f() { return __int_as_float(0x7fffffff); }

__device__ __forceinline__ void sts_cluster(uint32_t addr, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ void store4(float* p, const float (&y)[4], int n, bool vec) {
  if (vec && n >= 4) *reinterpret_cast<float4*>(p) = make_float4(y[0], y[1], y[2], y[3]);
  else
#pragma unroll
    for (int k = 0; k < 4; ++k) if (k < n) p[k] = y[k];
}
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float (&y)[4], int n, bool vec) {
  if (vec && n >= 4) {
    __nv_bfloat162 h[2] = {__floats2bfloat162_rn(y[0], y[1]), __floats2bfloat162_rn(y[2], y[3])};
    *reinterpret_cast<uint2*>(p) = *reinterpret_cast<uint2*>(h);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) if (k < n) p[k] = __float2bfloat16_rn(y[k]);
  }
}

// The warp's 32 rows x 128 bytes of output out of shared memory (16-byte units permuted with the row) a word or, where rows start on
// two bytes, an element per lane: for rows that do not start on 16 bytes.  Others go out by bulk copies, which the epilogue does not wait for.
template <typename W>
__device__ __forceinline__ void store_rows(const uint4* stage, int lane, W* out, int64_t ld, int rows, int cols) {
  constexpr int kCols = 128 / sizeof(W), kUnit = 16 / sizeof(W);
  const W* w = reinterpret_cast<const W*>(stage);
#pragma unroll 4
  for (int row = 0; row < rows; ++row)
#pragma unroll
    for (int c = lane; c < kCols; c += 32)
      if (c < cols) out[row * ld + c] = w[row * kCols + ((c / kUnit) ^ (row & 7)) * kUnit + c % kUnit];
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, uint32_t src, int c0, int c1) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map), "r"(src), "r"(c0), "r"(c1)
               : "memory");
}

// ------------------------------------------------------------------ host side
// Rows of K codes, `ld` bytes apart: boxes of 128 codes x box_rows; what lies beyond K or the last row is filled with zeros.
bool code_map(CUtensorMap* m, const uint8_t* base, int64_t K, int64_t rows, int64_t ld, int box_rows) {
  const EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {(cuuint64_t)K, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld};
  const cuuint32_t box[2] = {(cuuint32_t)kBlock, (cuuint32_t)box_rows}, step[2] = {1, 1};
  return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The output: boxes of 32 rows of 128 bytes.
bool out_map(CUtensorMap* m, void* base, int dtype, int64_t M, int64_t N, int64_t ld) {
  const EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const bool bf16 = dtype == QM_DT_BF16;
  const cuuint64_t dims[2] = {(cuuint64_t)N, (cuuint64_t)M}, strides[1] = {(cuuint64_t)ld * (bf16 ? 2 : 4)};
  const cuuint32_t box[2] = {bf16 ? 64u : 32u, 32u}, step[2] = {1, 1};
  return fn(m, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, base, dims, strides, box, step,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename K, typename... P>
qm_status launch_cluster(K kern, std::atomic<bool> (&ready)[kMaxDevices], size_t smem, size_t smem_most, unsigned grid, unsigned threads,
                         unsigned cluster, cudaStream_t s, const P&... params) {
  const int dev = current_device();
  if (dev < 0) return QM_ERR_UNSUPPORTED;
  if (!ready[dev].load(std::memory_order_acquire)) {
    QM_CUDA_OK(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_most));
    ready[dev].store(true, std::memory_order_release);
  }
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(grid); cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem; cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = cluster; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at; cfg.numAttrs = pdl_enabled() ? 2 : 1;
  QM_CUDA_OK(cudaLaunchKernelEx(&cfg, kern, params...));
  count_launch();
  return QM_OK;
}

}  // namespace
}  // namespace qm
