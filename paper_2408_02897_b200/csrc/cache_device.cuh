// What the cache's kernels share: its geometry, a sequence's extents with their checks, and 8-bit codes as pairs of fp16.  Included by .cu
// files only; everything sits in the including file's anonymous namespace.
#pragma once
#include <cuda_fp16.h>

#include "quant_device.cuh"

namespace qm {
namespace {

// Codes [blocks][kv_heads][block_tokens][dim], scales [blocks][kv_heads]; a sequence's blocks by its row of `tables`.
struct CacheView {
  uint8_t *k, *v;
  float *dk, *dv;
  int blocks, kv_heads, shift, dim;          // block_tokens is 1 << shift
  const int32_t *tables, *lens, *starts;     // starts null: a new token for each sequence
  int64_t ld_tables;
  int table_width, batch;
  int64_t tokens;
};

// A sequence's new tokens and its length with them.  What does not fit the tensors counts as no tokens at all.
// `reach`: the length, or one more than the table's blocks hold: a token that sees a position without a block gets NaN, however many
// there are, so a length that makes no sense costs no time.
struct Extent { int64_t first; int n, len, reach; };
__device__ __forceinline__ Extent extent_of(const CacheView& c, int b) {
  Extent e;
  e.first = c.starts ? c.starts[b] : b;
  const int64_t end = c.starts ? c.starts[b + 1] : b + 1;
  e.n = e.first >= 0 && end >= e.first && end <= c.tokens ? (int)(end - e.first) : 0;
  e.len = min(max(c.lens[b], 0), 0x7fff0000);       // (what is added to it stays inside 32 bits)
  e.reach = (int)min((int64_t)e.len, ((int64_t)c.table_width << c.shift) + 1);
  return e;
}

// The page that holds a sequence's block `i`; -1 where the table does not say or names none.
__device__ __forceinline__ int page_of(const CacheView& c, int b, int i) {
  if (i >= c.table_width) return -1;
  const int p = __ldg(c.tables + (int64_t)b * c.ld_tables + i);
  return p >= 0 && p < c.blocks ? p : -1;
}

// Items of all sequences in one line, sequence b's count(b) of them behind those before it, less than 2^31 in all: the sequence b that has item `want`
// (-1: none), where its items begin and how many they are. Goes by each sequence's checked extent, so that what one sequence's entries say moves no
// other's items. For all threads of a block.
struct Place { int b, begin, n; };
template <int THREADS, typename Count>
__device__ __forceinline__ Place place_of(int batch, int want, Count count) {
  __shared__ int sums[THREADS / 32];
  __shared__ Place place;
  constexpr int kEach = 4;                                     // neighbouring sequences to a thread, where there are many
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, each = batch <= THREADS ? 1 : kEach;
  if (tid == 0) place = Place{-1, 0, 0};
  int before = 0;
  for (int base = 0; base < batch && before <= want; base += THREADS * each) {
    const int b0 = base + tid * each;
    int mine[kEach], up = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      mine[i] = i < each && b0 + i < batch ? count(b0 + i) : 0;
      up += mine[i];
    }
    const int all = up;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int t = __shfl_up_sync(0xffffffffu, up, o); if (lane >= o) up += t; }
    if (lane == 31) sums[warp] = up;
    __syncthreads();
    int begin = before + up - all;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
      if (w < warp) begin += sums[w];
      before += sums[w];
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      if (begin <= want && want < begin + mine[i]) place = Place{b0 + i, begin, mine[i]};
      begin += mine[i];
    }
    __syncthreads();
  }
  return place;
}

// Four codes as two pairs of fp16; all of them are on fp16's grid.
template <int FMT>
__device__ __forceinline__ void half4_of(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if (FMT == QM_FMT_E4M3) {
    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(w));
  } else if (FMT == QM_FMT_E5M2) {
    lo = __byte_perm(w, 0u, 0x1404);
    hi = __byte_perm(w, 0u, 0x3424);
  } else {
    const uint32_t x = w ^ 0x80808080u;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(__byte_perm(x, 0x64646464u, 0x4140)), "r"(0x64806480u));
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(__byte_perm(x, 0x64646464u, 0x4342)), "r"(0x64806480u));
  }
}

inline CacheView view_of(const CacheArgs& a) {
  CacheView c{};
  c.k = a.k; c.v = a.v; c.dk = a.dk; c.dv = a.dv;
  c.blocks = (int)a.blocks; c.kv_heads = a.kv_heads; c.dim = a.dim;
  while ((1 << c.shift) < a.block_tokens) ++c.shift;
  c.tables = a.tables; c.lens = a.lens; c.starts = a.starts;
  c.ld_tables = a.ld_tables; c.table_width = a.table_width; c.batch = a.batch; c.tokens = a.tokens;
  return c;
}

// Scales below this count as 0 (a magnitude of 5e-14 at most): the attention's sums weigh by their inverses.
constexpr float kLeastScale = 8.6736174e-19f;                  // 2^-60

}  // namespace
}  // namespace qm
