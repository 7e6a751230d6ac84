// Attention over the 8-bit cache (qm_cache_attention).
//
//   x_ij = scale q_i . (dk k_j),   o_i = sum_j p_ij (dv v_j) / sum_j p_ij,   p_ij = exp(x_ij - max), j up to the position of i
// in one pass over the keys, with a running maximum. dk and dv are one number for a block of tokens: dk goes into the score. dv goes into
// the exponent: with x'_ij = x_ij log2 e + log2 dv and M its running maximum, P_ij = 2^(x'_ij - M) is what is rounded to fp16 and multiplied
// with the codes, and the denominator adds P_ij / dv: both are relative to the same maximum, o_i = sum P_ij v_j / sum (P_ij / dv), and no block's
// codes are scaled. Codes are exact in fp16 (8 bits or less of significand), queries too under a power of two for each row; products are
// exact in the tensor cores' fp32 sums, P has 11 bits (2^14 is its largest value, so that 2^-28 of it is still a normal number), the
// statistics and both sums are fp32.
//
// attention_rows: 16 query rows (tokens x query heads of one cached head) at a time against all keys, mma.sync m16n8k16 from registers: a
// thread loads 16 bytes of keys or values straight from the cache in the places that the instruction's operands have, so nothing goes through
// shared memory. A thread block takes an equal share of the cells (32 or 16 tokens for 16 rows and a head) of all sequences together, wherever they begin
// and end; what is left of rows whose keys were shared out is joined by attention_join, in the order of the keys.
//
// attention_tiles, for sequences with many query rows: 128 or 256 of them to a thread block. Tiles of 32 keys and values are turned into fp16
// in shared memory once for all of its warps, the next tile's codes on their way meanwhile.
//
// 64 sequences of up to 8192 tokens, 32 heads on 8 of 128: 149 us, 3.7 TB/s of codes; instructions (conversions, products, softmax) bound it, not HBM. 2048 tokens on
// 4096, the same heads: 474 us, 218 TFLOP/s of the 592 that mma.sync has here (8 cycles a product and scheduler); two warps a scheduler leave its latencies open.
#include <algorithm>
#include <atomic>

#include "cache_device.cuh"

namespace qm {
namespace {

constexpr int kWarps = 8, kMostRows = 16;
constexpr int kMaxBlocks = 512;                 // of a launch

struct RowsArgs {
  CacheView c;
  const __nv_bfloat16* q; int64_t ld_q;
  int heads, group;                              // group: query heads of a cached head
  float scale_log2;                              // of scores to the base 2
  __nv_bfloat16* out; int64_t ld_out;
  float* lse;
  int rows, cell;                                // to a cell of attention_rows, 8 or 16, and its tokens
  int most_rows;                                 // sequences with as many query rows of a cached head or more are attention_tiles'
  struct Share* shares;                          // one a thread block
  int* tiles_again;                              // whether some row of attention_tiles may have lost too much
  float* parts;                                  // [2 * blocks][16][padded dim + 2]
};

// A thread block's share of the cells, and the rows that it begins in. again: whether rows that it had all of may have lost too much (see kFewLost).
struct Share { int64_t lo, hi, start, end; int b, item, again, pad; };

__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float lg2(float x) { float y; asm("lg2.approx.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

__device__ __forceinline__ float key_scale(float dk) { return dk < kLeastScale ? 0.f : dk; }
// Blocks' scales may lie far apart, and both sums are relative to one maximum that has dv in it, which a denominator's terms may be far above or
// below. 2^16 / dv is what they are multiplied with: for dv from 2^-61 to 2^128 that, and the sums from a weight of 1 to 2^31 of them, are normal numbers
// (2^-112 .. 2^77, 2^-98 .. 2^122). weigh_of: log2 dv, of what counts as 0 less than any other's.
constexpr float kDenominators = 65536.f, kLogDenominators = 16.f, kNoValues = -60.5f;
__device__ __forceinline__ float weigh_of(float dv) { return dv < kLeastScale ? -61.f : lg2(dv); }
// What fp32 cannot hold on the way to a denominator: the factor 2^d, d <= 0, of a new maximum is 0 below 2^-126, and a weight below 2^-140 of the
// largest one. With log2 dv at least -61, terms so lost are below 2^(M - 65) each. The sum itself is 2^M over the largest of p dv, p a row's softmax (2^30 of
// it in these units): where that is at most 2^16, n terms lost are below n 2^-49 of the sum. Rows where it is more are done again by attention_join: the
// kernels only say so (what is kept for it in their loops, or done behind them, costs them 3 to 15 %).
constexpr float kFewLost = 16384.f;                            // 2^30 / 2^16
// The logarithm of a denominator whose sum is relative to 2^(top - 14).
__device__ __forceinline__ float log_of(float sum, float top) {
  return sum == 0.f ? -INFINITY : (log2f(sum) + (top - (14.f + kLogDenominators))) * 0.69314718f;
}

__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

// The power of two that brings a row's largest magnitude to 2^14 .. 2^15 (1 where that is 0 or not finite).
__device__ __forceinline__ float row_scale(float top) {
  const int ex = (int)(__float_as_uint(top) >> 23) - 127;
  return __uint_as_float((uint32_t)(127 + (top == 0.f || ex == 128 ? 0 : max(min(14 - ex, 120), -126))) << 23);
}

template <int N> struct Words { uint32_t w[N]; };
__device__ __forceinline__ Words<4> load_words(const uint8_t* p, Words<4>) {
  Words<4> r;
  asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]) : "l"(p));
  return r;
}
__device__ __forceinline__ Words<2> load_words(const uint8_t* p, Words<2>) {
  Words<2> r;
  asm volatile("ld.global.nc.L1::no_allocate.v2.b32 {%0, %1}, [%2];" : "=r"(r.w[0]), "=r"(r.w[1]) : "l"(p));
  return r;
}

// Tokens of a cell, whose keys and values a warp has in registers or on their way there.
__host__ __device__ constexpr int cell_of(int dim, bool narrow) { return narrow || dim == 64 ? 32 : 16; }
__device__ __forceinline__ int64_t cells_of(const RowsArgs& a, const Extent& e, int kRows, int kCell) {
  if (e.n == 0 || (int64_t)e.n * a.group >= a.most_rows) return 0;
  return (int64_t)a.c.kv_heads * (((int64_t)e.n * a.group + kRows - 1) / kRows) * max(1, (e.reach + kCell - 1) / kCell);
}

__device__ __forceinline__ uint32_t turned(uint32_t x) {            // 8x8 of 16 bits, a row to four lanes
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}

// NARROW: eight query rows instead of 16, as the products' N: keys and values are their left operands then, and half as many products, exponentials
// and sums make a cell. A token at a time with up to eight query heads to a cached one leaves the wider form's rows empty (64 tokens on 8192 172 us).
template <int FMT, int DIM, bool NARROW>
__global__ void __launch_bounds__(kWarps * 32, 2) attention_rows(const RowsArgs a) {
  constexpr int kChunks = DIM / 64;              // 16-byte pieces of a key in a thread
  constexpr int kWide = DIM / 32;                // words of a value in a thread
  constexpr int kTiles = DIM / 8;                // output tiles of eight dims
  constexpr int kCell = cell_of(DIM, NARROW), kN = kCell / 16, kRows = NARROW ? 8 : 16, kSums = NARROW ? kTiles / 2 : kTiles;
  __shared__ uint4 queries[4 * kChunks][32];     // as the products' operands
  __shared__ int64_t sums[kWarps];
  __shared__ int64_t found_lo;
  __shared__ int found_b;
  __shared__ float stat_m[kWarps][kRows], stat_l[kWarps][kRows];
  extern __shared__ float joined[];              // [warps][16][DIM + 4]
  pdl_prologue();
  const CacheView& c = a.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, cc = lane & 3;

  if (blockIdx.x == 0 && tid == 0) *a.tiles_again = 0;                        // (attention_tiles comes behind this kernel)

  // ---- this thread block's share: all cells in one line, sequence by sequence, head by head, rows by rows
  auto scan = [&](int base, int64_t& mine) {     // this thread's sequence's cells; the sum up to and with it
    const int b = base + tid;
    mine = b < c.batch ? cells_of(a, extent_of(c, b), kRows, kCell) : 0;
    int64_t up = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int64_t t = __shfl_up_sync(0xffffffffu, up, o); if (lane >= o) up += t; }
    if (lane == 31) sums[warp] = up;
    __syncthreads();
    for (int w = 0; w < warp; ++w) up += sums[w];
    return up;
  };
  int64_t total = 0, mine;
  for (int base = 0; base < c.batch; base += kWarps * 32) {
    scan(base, mine);
    for (int w = 0; w < kWarps; ++w) total += sums[w];
    __syncthreads();
  }
  const int blocks = (int)min((int64_t)gridDim.x, (total + kWarps - 1) / kWarps);      // a cell for each warp at least
  const int64_t lo = (int)blockIdx.x < blocks ? total * blockIdx.x / blocks : total;
  const int64_t hi = (int)blockIdx.x < blocks ? total * (blockIdx.x + 1) / blocks : total;
  if (lo >= hi) {
    if (tid == 0) a.shares[blockIdx.x] = Share{total, total, total, total, 0, 0, 0, 0};
    return;
  }
  int64_t before = 0;
  for (int base = 0; base < c.batch; base += kWarps * 32) {
    const int64_t up = scan(base, mine) + before;
    if (up - mine <= lo && lo < up) { found_b = base + tid; found_lo = up - mine; }
    for (int w = 0; w < kWarps; ++w) before += sums[w];
    __syncthreads();
    if (before > lo) break;
  }
  int b = found_b;
  int64_t at = found_lo;                         // where sequence b's cells begin

  // ---- its rows one after another
  bool first = true;
  for (int64_t pos = lo; pos < hi; ++b) {
    const Extent e = extent_of(c, b);
    const int64_t mine_all = cells_of(a, e, kRows, kCell);
    if (mine_all == 0) continue;
    const int per = max(1, (e.reach + kCell - 1) / kCell), tiles = (int)(((int64_t)e.n * a.group + kRows - 1) / kRows);
    for (int item = (int)((pos - at) / per); pos < hi && item < c.kv_heads * tiles; ++item) {
      const int64_t start = at + (int64_t)item * per, end = start + per;
      if (first && tid == 0) a.shares[blockIdx.x] = Share{lo, hi, start, end, b, item, 0, 0};
      const int head = item / tiles, row0 = (item - head * tiles) * kRows;
      const int rows = min(kRows, e.n * a.group - row0);
      // keys up to the position of the row's token; a token whose position is below 0 sees none
      auto limit_of = [&](int r) { return r < rows ? min(e.reach, max(0, e.len - e.n + (row0 + r) / a.group + 1)) : 0; };
      const int limit[2] = {limit_of(NARROW ? 2 * cc : g), limit_of(NARROW ? 2 * cc + 1 : g + 8)};      // of the rows whose statistics this thread has
      const int least = limit_of(0), most = limit_of(rows - 1);
      // (written as min(end, hi) - start this is compiled to per in all but a share's first rows, as recorded in the kernel: nvcc 12.9.86, at ptxas' -O1
      // too. The tests of single tokens show it; the same walk by itself, without the products, does not.)
      const int cell0 = (int)(pos - start), quota = hi < end ? (int)(hi - start) : per, cell1 = min(quota, (most + kCell - 1) / kCell);

      // ---- queries: row g, or rows g and g + 8, in the order of dims in which a thread has its part of a key
      float factor[2];
      {
        constexpr int kR = NARROW ? 1 : 2;
        uint32_t q[4 * kChunks][4] = {};
#pragma unroll
        for (int r = 0; r < kR; ++r) {
          float top = 0.f;
          uint2 raw[4 * kChunks];
          const int row = row0 + g + 8 * r, token = row / a.group;
          const __nv_bfloat16* const from = a.q + (e.first + token) * a.ld_q + ((int64_t)head * a.group + row - token * a.group) * c.dim;
#pragma unroll
          for (int s = 0; s < 4 * kChunks; ++s) {
            const int d = (cc + 4 * (s >> 2)) * 16 + 4 * (s & 3);
            raw[s] = g + 8 * r < rows && d < c.dim ? *reinterpret_cast<const uint2*>(from + d) : make_uint2(0u, 0u);
            top = fmaxf(top, fmaxf(fmaxf(fabsf(bf16_lo(raw[s].x)), fabsf(bf16_hi(raw[s].x))), fmaxf(fabsf(bf16_lo(raw[s].y)), fabsf(bf16_hi(raw[s].y)))));
          }
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
          top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
          const float by = row_scale(top);
          factor[r] = a.scale_log2 / by;
#pragma unroll
          for (int s = 0; s < 4 * kChunks; ++s) {
            q[s][r] = pack_half2(bf16_lo(raw[s].x) * by, bf16_hi(raw[s].x) * by);
            q[s][2 + r] = pack_half2(bf16_lo(raw[s].y) * by, bf16_hi(raw[s].y) * by);
          }
        }
        if (NARROW) {
          const float mine = factor[0];
          factor[0] = __shfl_sync(0xffffffffu, mine, 8 * cc);
          factor[1] = __shfl_sync(0xffffffffu, mine, 8 * cc + 4);
        }
        // (the barriers: the last rows' queries have been read by all; these are there)
        __syncthreads();
#pragma unroll
        for (int s = 0; s < 4 * kChunks; ++s)
          if (s == warp) queries[s][lane] = make_uint4(q[s][0], q[s][1], q[s][2], q[s][3]);
        __syncthreads();
      }
      float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
      float o[kSums][4];
#pragma unroll
      for (int t = 0; t < kSums; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[t][i] = 0.f;

      // ---- cells: their keys and values in registers, the next cell's on their way
      Words<4> k[2 * kN][kChunks];
      Words<kWide> v[kN][4];
      float dk[kN], dv[kN];
      auto pages = [&](int cell, int (&p)[kN]) {
#pragma unroll
        for (int i = 0; i < kN; ++i) {
          const int token = cell * kCell + 16 * i;
          p[i] = cell < cell1 && token < most ? page_of(c, b, token >> c.shift) : -1;
        }
      };
      auto base_of = [&](int cell, int i, int page) {
        const int token = cell * kCell + 16 * i;
        return ((((int64_t)page * c.kv_heads + head) << c.shift) + (token & ((1 << c.shift) - 1))) * c.dim;
      };
      // A cell that all rows see, of a head that fills the registers' places, is loaded without a condition or an offset to be computed.
      const bool fits = c.dim == DIM;
      auto load_k = [&](int cell, const int (&p)[kN]) {
        if (fits && p[0] >= 0 && p[kN - 1] >= 0) {
#pragma unroll
          for (int i = 0; i < kN; ++i) {
            const uint8_t* const from = c.k + base_of(cell, i, p[i]) + g * DIM + cc * 16;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int h = 0; h < kChunks; ++h) k[2 * i + t][h] = load_words(from + 8 * t * DIM + 64 * h, Words<4>());
          }
        } else {
#pragma unroll
          for (int i = 0; i < kN; ++i) {
            const int64_t base = base_of(cell, i, max(p[i], 0));
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int h = 0; h < kChunks; ++h) {
                const int d = (cc + 4 * h) * 16;
                k[2 * i + t][h] = p[i] >= 0 && d < c.dim ? load_words(c.k + base + (8 * t + g) * c.dim + d, Words<4>()) : Words<4>{};
              }
          }
        }
        // (a page that the table does not have, or has wrong: NaN for whoever sees its tokens)
#pragma unroll
        for (int i = 0; i < kN; ++i) dk[i] = p[i] >= 0 ? __ldg(c.dk + (int64_t)p[i] * c.kv_heads + head) : __int_as_float(0x7fffffff);
      };
      auto load_v = [&](int cell, const int (&p)[kN]) {
        if (fits && p[0] >= 0 && p[kN - 1] >= 0 && (cell + 1) * kCell <= most) {
#pragma unroll
          for (int i = 0; i < kN; ++i) {
            const uint8_t* const from = c.v + base_of(cell, i, p[i]) + 2 * cc * DIM + g * 4 * kWide;
#pragma unroll
            for (int t = 0; t < 4; ++t) v[i][t] = load_words(from + ((t & 1) + 8 * (t >> 1)) * DIM, Words<kWide>());
          }
        } else {
#pragma unroll
          for (int i = 0; i < kN; ++i) {
            const int64_t base = base_of(cell, i, max(p[i], 0));
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              const int token = 2 * cc + (t & 1) + 8 * (t >> 1), d = g * 4 * kWide;
              // (nothing of what lies behind the last key that is seen: its codes may be anything, and 0 times NaN is not 0)
              v[i][t] = p[i] >= 0 && d < c.dim && cell * kCell + 16 * i + token < most ? load_words(c.v + base + token * c.dim + d, Words<kWide>())
                                                                                      : Words<kWide>{};
            }
          }
        }
#pragma unroll
        for (int i = 0; i < kN; ++i) dv[i] = p[i] >= 0 ? __ldg(c.dv + (int64_t)p[i] * c.kv_heads + head) : __int_as_float(0x7fffffff);
      };
      int here[kN], next[kN];
      int cell = cell0 + warp;
      pages(cell, here);
      if (cell < cell1) { load_k(cell, here); load_v(cell, here); }
      pages(cell + kWarps, next);
      for (; cell < cell1; cell += kWarps) {
        // scores: s[t][i] of row i / 2 (g or g + 8) and key 8 t + 2 cc + i % 2, or narrow of row 2 cc + i % 2 and key 16 t + g + 8 (i / 2)
        constexpr int kS = NARROW ? kN : 2 * kN;
        float s[kS][4];
#pragma unroll
        for (int t = 0; t < kS; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[t][i] = 0.f;
#pragma unroll
        for (int h = 0; h < kChunks; ++h)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint4 w = queries[4 * h + j][lane];
            const uint32_t q[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int t = 0; t < kN; ++t) {
              uint32_t x[4];
              half4_of<FMT>(k[2 * t][h].w[j], x[0], x[2]);
              half4_of<FMT>(k[2 * t + 1][h].w[j], x[1], x[3]);
              if (NARROW) mma16(s[t], x, q[0], q[2]);
              else {
                mma16(s[NARROW ? 0 : 2 * t], q, x[0], x[2]);
                mma16(s[NARROW ? 0 : 2 * t + 1], q, x[1], x[3]);
              }
            }
          }
        float ck[kN], cv[kN];
#pragma unroll
        for (int i = 0; i < kN; ++i) { ck[i] = key_scale(dk[i]); cv[i] = dv[i]; }
        const bool more = cell + kWarps < cell1;
        if (more) load_k(cell + kWarps, next);
        // to the base 2, with the values' scales, masked
        float top[2] = {m[0], m[1]};
        float weigh[kN];
#pragma unroll
        for (int i = 0; i < kN; ++i) weigh[i] = weigh_of(cv[i]);
#pragma unroll
        for (int t = 0; t < kS; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int r = NARROW ? i & 1 : i >> 1, n = NARROW ? t : t >> 1;
            s[t][i] = fmaf(s[t][i], factor[r] * ck[n], weigh[n]);
          }
        if ((cell + 1) * kCell > least) {
#pragma unroll
          for (int t = 0; t < kS; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (cell * kCell + (NARROW ? 16 * t + g + 8 * (i >> 1) : 8 * t + 2 * cc + (i & 1)) >= limit[NARROW ? i & 1 : i >> 1]) s[t][i] = -INFINITY;
        }
#pragma unroll
        for (int t = 0; t < kS; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) top[NARROW ? i & 1 : i >> 1] = fmaxf(top[NARROW ? i & 1 : i >> 1], s[t][i]);
        float from[2];
        bool moved = false;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          if (NARROW) {
#pragma unroll
            for (int x = 4; x < 32; x *= 2) top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], x));
          } else {
            top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 1));
            top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 2));
          }
          moved |= top[r] > m[r];
        }
        if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const float shrink = m[r] == top[r] ? 1.f : ex2(m[r] - top[r]);
            m[r] = top[r];
            l[r] *= shrink;
#pragma unroll
            for (int t = 0; t < kSums; ++t) {
              o[t][NARROW ? r : 2 * r] *= shrink;
              o[t][NARROW ? 2 + r : 2 * r + 1] *= shrink;
            }
          }
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) from[r] = m[r] == -INFINITY ? 0.f : m[r] - 14.f;
        // weights, in the places of an operand
        uint32_t p[kN][4];
#pragma unroll
        for (int n = 0; n < kN; ++n) {
          const bool none = weigh[n] < kNoValues;
          const float inverse = ex2(kLogDenominators - weigh[n]);
          float x[2][4];                                                     // [row][key]
#pragma unroll
          for (int r = 0; r < 2; ++r) {
#pragma unroll
            for (int i = 0; i < (NARROW ? 2 : 4); ++i) x[r][i] = ex2((NARROW ? s[n][2 * i + r] : s[NARROW ? 0 : 2 * n + (i >> 1)][2 * r + (i & 1)]) - from[r]);
            const float sum = NARROW ? x[r][0] + x[r][1] : (x[r][0] + x[r][1]) + (x[r][2] + x[r][3]);
            if (sum != 0.f) l[r] = fmaf(sum, inverse, l[r]);            // (nothing of a block that the row does not see, whatever its scale)
          }
          if (NARROW) {
            p[n][0] = turned(none ? 0u : pack_half2(x[0][0], x[1][0]));
            p[n][1] = turned(none ? 0u : pack_half2(x[0][1], x[1][1]));
          } else {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              p[n][r] = none ? 0u : pack_half2(x[r][0], x[r][1]);
              p[n][2 + r] = none ? 0u : pack_half2(x[r][2], x[r][3]);
            }
          }
        }
#pragma unroll
        for (int i = 0; i < kN; ++i)
#pragma unroll
          for (int w = 0; w < kWide; ++w) {
            uint32_t b[4][2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t x = v[i][2 * h].w[w], y = v[i][2 * h + 1].w[w];
              half4_of<FMT>(__byte_perm(x, y, 0x5140), b[0][h], b[1][h]);
              half4_of<FMT>(__byte_perm(x, y, 0x7362), b[2][h], b[3][h]);
            }
            if (NARROW) {
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                const uint32_t x[4] = {b[2 * j][0], b[2 * j + 1][0], b[2 * j][1], b[2 * j + 1][1]};
                mma16(o[2 * w + j], x, p[i][0], p[i][1]);
              }
            } else {
#pragma unroll
              for (int j = 0; j < 4; ++j) mma16(o[NARROW ? 0 : 4 * w + j], p[i], b[j][0], b[j][1]);
            }
          }
        if (more) {
          load_v(cell + kWarps, next);
          pages(cell + 2 * kWarps, next);
        }
      }

      // ---- the warps' sums together, and out
      __syncthreads();                                                   // (the last rows' have been read)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const int row = NARROW ? 2 * cc + r : g + 8 * r;
#pragma unroll
        for (int x = NARROW ? 4 : 1; x < (NARROW ? 32 : 4); x *= 2) l[r] += __shfl_xor_sync(0xffffffffu, l[r], x);
        if ((NARROW ? g : cc) == 0) { stat_m[warp][row] = m[r]; stat_l[warp][row] = l[r]; }
        if (row < rows) {
          float* const to = joined + (warp * kRows + row) * (DIM + 4);
          // tile t, column n stands for dim n * kTiles + t (wide: a thread has columns 2 cc and 2 cc + 1; narrow: column g, tiles 2 t and 2 t + 1)
          if (NARROW) {
#pragma unroll
            for (int t = 0; t < kSums; t += 2)
              *reinterpret_cast<float4*>(to + g * kTiles + 2 * t) = make_float4(o[t][r], o[t][2 + r], o[t + 1][r], o[t + 1][2 + r]);
          } else {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int t = 0; t + 3 < kSums; t += 4)
                *reinterpret_cast<float4*>(to + (2 * cc + h) * kTiles + t) =
                    make_float4(o[t][2 * r + h], o[t + 1][2 * r + h], o[t + 2][2 * r + h], o[t + 3][2 * r + h]);
          }
        }
      }
      __syncthreads();
      const bool whole = start >= lo && end <= hi;
      const int slot = 2 * (int)blockIdx.x + (start < lo ? 0 : 1);
      for (int i = tid; i < rows * (DIM / 4); i += kWarps * 32) {
        const int r = i / (DIM / 4), d = i % (DIM / 4) * 4;
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) top = fmaxf(top, stat_m[w][r]);
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float by = stat_m[w][r] == top ? 1.f : ex2(stat_m[w][r] - top);
          const float4 x = *reinterpret_cast<const float4*>(joined + (w * kRows + r) * (DIM + 4) + d);
          sum = fmaf(stat_l[w][r], by, sum);
          y.x = fmaf(x.x, by, y.x); y.y = fmaf(x.y, by, y.y); y.z = fmaf(x.z, by, y.z); y.w = fmaf(x.w, by, y.w);
        }
        if (whole) {
          if (sum < kFewLost && top != -INFINITY) a.shares[blockIdx.x].again = 1;
          const int row = row0 + r, token = row / a.group, h = head * a.group + row - token * a.group;
          const float inv = sum == 0.f ? 0.f : kDenominators / sum;
          if (d < c.dim)
            *reinterpret_cast<uint2*>(a.out + (e.first + token) * a.ld_out + (int64_t)h * c.dim + d) =
                make_uint2(pack_bf16x2(y.x * inv, y.y * inv), pack_bf16x2(y.z * inv, y.w * inv));
          if (d == 0 && a.lse) a.lse[(e.first + token) * a.heads + h] = log_of(sum, top);
        } else {
          float* const to = a.parts + ((int64_t)slot * kMostRows + r) * (DIM + 2);
          to[d] = y.x; to[d + 1] = y.y; to[d + 2] = y.z; to[d + 3] = y.w;
          if (d == 0) { to[DIM] = top; to[DIM + 1] = sum; }
        }
      }
      first = false;
      pos = end;                                                         // (at or beyond hi: the loops end)
    }
    at += mine_all;
  }
}

// One query row by a warp, in two passes over its scores: the maximum first, then every weight in fp32 from it, and the denominator's terms without
// dv. For scales that no layer has.
template <int FMT>
__device__ __noinline__ void far_row(const RowsArgs& a, const Extent& e, int b, int head, int64_t row) {
  const CacheView& c = a.c;
  const int lane = threadIdx.x & 31;
  const int64_t token = row / a.group;
  const __nv_bfloat16* const q = a.q + (e.first + token) * a.ld_q + ((int64_t)head * a.group + row - token * a.group) * c.dim;
  const int end = min(e.reach, max(0, e.len - e.n + (int)token + 1));
  float top = 0.f;
  for (int d = lane; d < c.dim; d += 32) top = fmaxf(top, fabsf(__bfloat162float(q[d])));
  for (int x = 16; x; x /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
  const float scale = row_scale(top), factor = a.scale_log2 / scale;
  auto block_of = [&](int key) {                               // -1: none
    const int page = page_of(c, b, key >> c.shift);
    return page < 0 ? -1ll : (long long)page * c.kv_heads + head;
  };
  auto at = [&](long long block, int key) { return ((block << c.shift) + (key & ((1 << c.shift) - 1))) * c.dim; };
  // this lane's key's score to the base 2, and its values' scale
  auto score = [&](int key, float& dv) {
    const long long block = key < end ? block_of(key) : -1;
    dv = 0.f;
    if (key >= end) return -INFINITY;
    if (block < 0) return dv = __int_as_float(0x7fffffff);
    const uint32_t* const codes = reinterpret_cast<const uint32_t*>(c.k + at(block, key));
    float s = 0.f;
#pragma unroll 1
    for (int d = 0; d < c.dim; d += 4) {
      uint32_t h[2];
      half4_of<FMT>(__ldg(codes + d / 4), h[0], h[1]);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float2 k = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
        s = fmaf(__bfloat162float(q[d + 2 * i]) * scale, k.x, s);
        s = fmaf(__bfloat162float(q[d + 2 * i + 1]) * scale, k.y, s);
      }
    }
    dv = __ldg(c.dv + block);
    return s * (factor * key_scale(__ldg(c.dk + block)));
  };
  float most = -INFINITY, sum = 0.f;
  float4 y = make_float4(0.f, 0.f, 0.f, 0.f);                  // dims 4 lane ..
#pragma unroll 1
  for (int k0 = 0; k0 < end; k0 += 32) {
    float dv;
    const float x = score(k0 + lane, dv);
    most = fmaxf(most, x + weigh_of(dv));
  }
  for (int x = 16; x; x /= 2) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, x));
  const float from = most == -INFINITY ? 0.f : most - 14.f;
#pragma unroll 1
  for (int k0 = 0; k0 < end; k0 += 32) {
    float dv;
    const float x = score(k0 + lane, dv);
    sum += dv != dv ? dv : ex2(x - from + kLogDenominators);
    const float p = dv < kLeastScale ? 0.f : ex2(x + weigh_of(dv) - from);
#pragma unroll 1
    for (int i = 0; i < 32 && k0 + i < end; ++i) {
      const float w = __shfl_sync(0xffffffffu, p, i);
      const long long block = block_of(k0 + i);
      if (4 * lane >= c.dim || block < 0) continue;
      uint32_t h[2];
      half4_of<FMT>(__ldg(reinterpret_cast<const uint32_t*>(c.v + at(block, k0 + i)) + lane), h[0], h[1]);
      const float2 v0 = __half22float2(*reinterpret_cast<const __half2*>(&h[0])), v1 = __half22float2(*reinterpret_cast<const __half2*>(&h[1]));
      y.x = fmaf(w, v0.x, y.x); y.y = fmaf(w, v0.y, y.y); y.z = fmaf(w, v1.x, y.z); y.w = fmaf(w, v1.y, y.w);
    }
  }
  for (int x = 16; x; x /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, x);
  const int64_t h = (int64_t)head * a.group + row - token * a.group;
  const float inv = sum == 0.f ? 0.f : kDenominators / sum;
  if (4 * lane < c.dim)
    *reinterpret_cast<uint2*>(a.out + (e.first + token) * a.ld_out + h * c.dim + 4 * lane) =
        make_uint2(pack_bf16x2(y.x * inv, y.y * inv), pack_bf16x2(y.z * inv, y.w * inv));
  if (lane == 0 && a.lse) a.lse[(e.first + token) * a.heads + h] = log_of(sum, most);
}

// The rows whose keys several thread blocks have had, joined by the block whose share begins inside them first; and what has to be done again.  A row
// a thread block's quarter, or one of its warps.
template <int FMT, int DIM>
__global__ void __launch_bounds__(DIM) attention_join(const __grid_constant__ RowsArgs a, int grid) {
  pdl_prologue();
  const int i = blockIdx.x, warp = blockIdx.y * (DIM / 32) + (threadIdx.x >> 5), warps = gridDim.y * (DIM / 32);
  const CacheView& c = a.c;
  const Share s = a.shares[i];
  auto tiles_of = [&](const Extent& e) { return (int)(((int64_t)e.n * a.group + a.rows - 1) / a.rows); };
  auto item_again = [&](const Extent& e, int b, int item, int tiles) {
    const int head = item / tiles, row0 = (item - head * tiles) * a.rows;
    for (int r = warp; r < min(a.rows, e.n * a.group - row0); r += warps) far_row<FMT>(a, e, b, head, row0 + r);
  };
  if (*a.tiles_again) {                          // all rows of attention_tiles, by all warps
    int64_t next = (int64_t)i * warps + warp;
    for (int b = 0; b < c.batch; ++b) {
      const Extent e = extent_of(c, b);
      const int64_t rows = (int64_t)e.n * a.group, all = rows * c.kv_heads;
      if (rows < a.most_rows) continue;
      for (; next < all; next += (int64_t)gridDim.x * warps) far_row<FMT>(a, e, b, (int)(next / rows), next % rows);
      next -= all;
    }
  }
  if (s.again) {                                 // rows that it has had all of
    int64_t at = s.start - (int64_t)s.item * (s.end - s.start);
    int item = s.item;
    for (int b = s.b; at < s.hi; ++b, item = 0) {
      const Extent e = extent_of(c, b);
      const int64_t cells = cells_of(a, e, a.rows, a.cell);
      if (cells == 0) continue;
      const int tiles = tiles_of(e), per = (int)(cells / ((int64_t)c.kv_heads * tiles));
      for (; item < c.kv_heads * tiles && at + (int64_t)(item + 1) * per <= s.hi; ++item)
        if (at + (int64_t)item * per >= s.lo) item_again(e, b, item, tiles);
      at += cells;
    }
  }
  if (i == 0 || s.lo <= s.start || s.lo >= s.end || a.shares[i - 1].lo > s.start) return;
  const Extent e = extent_of(c, s.b);
  const int tiles = tiles_of(e), head = s.item / tiles, row0 = (s.item - head * tiles) * a.rows;
  const int rows = min(a.rows, e.n * a.group - row0), d = threadIdx.x;
  int last = i;
  while (last + 1 < grid && a.shares[last + 1].lo < s.end) ++last;
  for (int r = blockIdx.y; r < rows; r += gridDim.y) {
    float top = -INFINITY, sum = 0.f, y = 0.f;
    auto part = [&](int j) { return a.parts + ((int64_t)(2 * j + (j == i - 1 ? 1 : 0)) * kMostRows + r) * (DIM + 2); };
    for (int j = i - 1; j <= last; ++j) top = fmaxf(top, part(j)[DIM]);
#pragma unroll 4
    for (int j = i - 1; j <= last; ++j) {
      const float* const from = part(j);
      const float by = from[DIM] == top ? 1.f : ex2(from[DIM] - top);
      sum = fmaf(from[DIM + 1], by, sum);
      y = fmaf(from[d], by, y);
    }
    if (sum < kFewLost && top != -INFINITY) {    // (the same for all of the block's threads)
      if (threadIdx.x < 32) far_row<FMT>(a, e, s.b, head, row0 + r);
      continue;
    }
    const int row = row0 + r, token = row / a.group, h = head * a.group + row - token * a.group;
    if (d < c.dim) a.out[(e.first + token) * a.ld_out + (int64_t)h * c.dim + d] = __float2bfloat16_rn(sum == 0.f ? 0.f : y * (kDenominators / sum));
    if (d == 0 && a.lse) a.lse[(e.first + token) * a.heads + h] = log_of(sum, top);
  }
}

// ---------------------------------------------------------------- many rows
constexpr int kTileKeys = 32, kGroups = kTileKeys / 16;
// keys and values of a tile; bytes between tokens that put eight rows on distinct banks
template <int DIM> __host__ __device__ constexpr uint32_t tile_bytes() { return 2u * kTileKeys * (DIM * 2 + 16); }
template <int DIM> __host__ __device__ constexpr uint32_t tiles_smem(int mt) { return 2 * tile_bytes<DIM>() + 128 * mt * (DIM * 2 + 16); }

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_turned(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

// MT: times 16 rows a warp.  An operand of keys or values is 256 bytes of shared memory for a product of eight cycles a scheduler, which with 16 rows
// is all that shared memory gives; 32 rows use it twice.
template <int FMT, int DIM, int MT>
__global__ void __launch_bounds__(256, MT == 1 ? 2 : 1) attention_tiles(const RowsArgs a) {
  constexpr int kTileRows = 128 * MT, kPitch = DIM * 2 + 16, kSteps = DIM / 16, kOut = DIM / 8;
  static_assert(kTileKeys * DIM / 16 <= 256, "a 16-byte piece of the keys to a thread");
  extern __shared__ __align__(16) uint8_t tile_raw[];                          // [2 buffers][keys, values][kTileKeys][kPitch], queries [kTileRows][kPitch]
  __shared__ float scales[2][2][kGroups];                                         // [buffer][keys, values][16 tokens]
  pdl_prologue();
  const CacheView& c = a.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, cc = lane & 3;
  // All sequences' tiles in one line from its end: the last ones, which see most, come first.
  const int head = blockIdx.y;
  const Place at = place_of<256>(c.batch, blockIdx.x, [&](int i) {
    const int64_t rows = (int64_t)extent_of(c, c.batch - 1 - i).n * a.group;
    return rows < a.most_rows ? 0 : (int)((rows + kTileRows - 1) / kTileRows);
  });
  if (at.b < 0) return;
  const int b = c.batch - 1 - at.b;
  const Extent e = extent_of(c, b);
  const int64_t row0 = (int64_t)(at.n - 1 - ((int)blockIdx.x - at.begin)) * kTileRows, all = (int64_t)e.n * a.group;

  auto limit_of = [&](int64_t r) { return r < all ? min(e.reach, max(0, e.len - e.n + (int)(r / a.group) + 1)) : 0; };
  const int64_t first = row0 + 16 * MT * warp;                                 // of this warp; may be beyond the last
  const int rows = (int)min((int64_t)16 * MT, all - first);
  int limit[MT][2];
#pragma unroll
  for (int u = 0; u < MT; ++u)
#pragma unroll
    for (int r = 0; r < 2; ++r) limit[u][r] = limit_of(first + 16 * u + 8 * r + g);
  const int least = rows > 0 ? limit_of(first + 16 * MT - 1 < all ? first : all) : 0;      // (a row beyond the last sees nothing)
  const int most = rows > 0 ? limit_of(first + rows - 1) : 0;
  const int seen = limit_of(min(row0 + kTileRows, all) - 1), tiles = (seen + kTileKeys - 1) / kTileKeys;      // by the whole block

  const uint32_t smem = (uint32_t)__cvta_generic_to_shared(tile_raw), queries = smem + 2 * tile_bytes<DIM>() + warp * 16 * MT * kPitch;      // the warp's
  float factor[MT][2];
#pragma unroll
  for (int u = 0; u < MT; ++u)
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int in_warp = 16 * u + 8 * r + g;
      const int64_t row = first + in_warp, token = row / a.group;
      const bool in = in_warp < rows;
      const __nv_bfloat16* const from = a.q + (e.first + (in ? token : 0)) * a.ld_q + ((int64_t)head * a.group + (in ? row - token * a.group : 0)) * c.dim;
      uint32_t raw[kSteps][2];
      float top = 0.f;
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int d = 16 * s + 8 * i + 2 * cc;
          raw[s][i] = in && d < c.dim ? *reinterpret_cast<const uint32_t*>(from + d) : 0u;
          top = fmaxf(top, fmaxf(fabsf(bf16_lo(raw[s][i])), fabsf(bf16_hi(raw[s][i]))));
        }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const float by = row_scale(top);
      factor[u][r] = a.scale_log2 / by;
#pragma unroll
      for (int s = 0; s < kSteps; ++s)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          asm volatile("st.shared.b32 [%0], %1;" ::"r"(queries + in_warp * kPitch + s * 32 + i * 16 + cc * 4),
                       "r"(pack_half2(bf16_lo(raw[s][i]) * by, bf16_hi(raw[s][i]) * by)) : "memory");
    }
  __syncwarp();

  float m[MT][2], l[MT][2], o[MT][kOut][4];
#pragma unroll
  for (int u = 0; u < MT; ++u) {
    m[u][0] = m[u][1] = -INFINITY;
    l[u][0] = l[u][1] = 0.f;
#pragma unroll
    for (int t = 0; t < kOut; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[u][t][i] = 0.f;
  }

  // ---- a tile's codes: in registers, then as fp16 in shared memory
  Words<4> k, v;
  float scale = 0.f;
  int page, page_s = -1;
  const int token_in = tid / (DIM / 16), dim_in = tid % (DIM / 16) * 16;       // this thread's piece
  auto pages = [&](int tile) {
    const int token = tile * kTileKeys + token_in, group = tile * kTileKeys + 16 * (tid % kGroups);
    page = token_in < kTileKeys && token < seen ? page_of(c, b, token >> c.shift) : -1;
    page_s = tid < 2 * kGroups && group < seen ? page_of(c, b, group >> c.shift) : -1;
  };
  auto load = [&](int tile) {
    const int token = tile * kTileKeys + token_in;
    const bool in = page >= 0 && dim_in < c.dim;                               // (nothing behind the last key that is seen: its codes may be anything)
    const int64_t at = ((((int64_t)(in ? page : 0) * c.kv_heads + head) << c.shift) + (token & ((1 << c.shift) - 1))) * c.dim + dim_in;
    k = in ? load_words(c.k + at, Words<4>()) : Words<4>{};
    v = in ? load_words(c.v + at, Words<4>()) : Words<4>{};
    if (tid < 2 * kGroups) scale = page_s >= 0 ? __ldg((tid < kGroups ? c.dk : c.dv) + (int64_t)page_s * c.kv_heads + head) : __int_as_float(0x7fffffff);
  };
  auto store = [&](int buf) {
    const uint32_t at = smem + buf * tile_bytes<DIM>() + token_in * kPitch + dim_in * 2;
    if (token_in < kTileKeys)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const Words<4>& w = x ? v : k;
        uint32_t h[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) half4_of<FMT>(w.w[j], h[2 * j], h[2 * j + 1]);
#pragma unroll
        for (int j = 0; j < 2; ++j)
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at + x * kTileKeys * kPitch + 16 * j), "r"(h[4 * j]), "r"(h[4 * j + 1]),
                       "r"(h[4 * j + 2]), "r"(h[4 * j + 3]) : "memory");
      }
    if (tid < 2 * kGroups) scales[buf][tid / kGroups][tid % kGroups] = tid < kGroups ? key_scale(scale) : scale;
  };
  pages(0);
  load(0);
  pages(1);
  store(0);
  __syncthreads();
  const uint32_t at_q = queries + ((lane & 7) + ((lane >> 3) & 1) * 8) * kPitch + (lane >> 4) * 16;
  const uint32_t at_k = (lane & 7) * kPitch + (lane >> 4) * 8 * kPitch + ((lane >> 3) & 1) * 16;
  const uint32_t at_v = (lane & 7) * kPitch + ((lane >> 3) & 1) * 8 * kPitch + (lane >> 4) * 16;
  for (int tile = 0; tile < tiles; ++tile) {
    const int buf = tile & 1;
    if (tile + 1 < tiles) { load(tile + 1); pages(tile + 2); }
    if (tile * kTileKeys < most) {                                             // (uniform in the warp)
      const uint32_t keys = smem + buf * tile_bytes<DIM>(), values = keys + kTileKeys * kPitch;
      // (16 dims of all keys at a time: products that do not wait for one another)
      float s[MT][2 * kGroups][4];
#pragma unroll
      for (int u = 0; u < MT; ++u)
#pragma unroll
        for (int t = 0; t < 2 * kGroups; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[u][t][i] = 0.f;
#pragma unroll
      for (int d = 0; d < kSteps; ++d) {
        uint32_t q[MT][4], w[kGroups][4];
#pragma unroll
        for (int u = 0; u < MT; ++u) ldmatrix4(q[u], at_q + u * 16 * kPitch + d * 32);
#pragma unroll
        for (int t = 0; t < kGroups; ++t) ldmatrix4(w[t], keys + at_k + t * 16 * kPitch + d * 32);
#pragma unroll
        for (int t = 0; t < kGroups; ++t)
#pragma unroll
          for (int u = 0; u < MT; ++u) {
            mma16(s[u][2 * t], q[u], w[t][0], w[t][1]);
            mma16(s[u][2 * t + 1], q[u], w[t][2], w[t][3]);
          }
      }
      float weigh[kGroups];
#pragma unroll
      for (int i = 0; i < kGroups; ++i) weigh[i] = weigh_of(scales[buf][1][i]);
      const bool partial = (tile + 1) * kTileKeys > least;
      uint32_t p[MT][kGroups][4];
#pragma unroll
      for (int u = 0; u < MT; ++u) {
        float top[2] = {m[u][0], m[u][1]};
#pragma unroll
        for (int t = 0; t < 2 * kGroups; ++t) {
          const float ck = scales[buf][0][t >> 1];
#pragma unroll
          for (int i = 0; i < 4; ++i) s[u][t][i] = fmaf(s[u][t][i], factor[u][i >> 1] * ck, weigh[t >> 1]);
        }
        if (partial) {
#pragma unroll
          for (int t = 0; t < 2 * kGroups; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (tile * kTileKeys + 8 * t + 2 * cc + (i & 1) >= limit[u][i >> 1]) s[u][t][i] = -INFINITY;
        }
#pragma unroll
        for (int t = 0; t < 2 * kGroups; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) top[i >> 1] = fmaxf(top[i >> 1], s[u][t][i]);
        bool moved = false;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 1));
          top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 2));
          moved |= top[r] > m[u][r];
        }
        if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const float shrink = m[u][r] == top[r] ? 1.f : ex2(m[u][r] - top[r]);
            m[u][r] = top[r];
            l[u][r] *= shrink;
#pragma unroll
            for (int t = 0; t < kOut; ++t) { o[u][t][2 * r] *= shrink; o[u][t][2 * r + 1] *= shrink; }
          }
        }
        const float from[2] = {m[u][0] == -INFINITY ? 0.f : m[u][0] - 14.f, m[u][1] == -INFINITY ? 0.f : m[u][1] - 14.f};
#pragma unroll
        for (int i = 0; i < kGroups; ++i) {
          const bool none = weigh[i] < kNoValues;
          const float inverse = ex2(kLogDenominators - weigh[i]);
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const float e0 = ex2(s[u][2 * i][2 * r] - from[r]), e1 = ex2(s[u][2 * i][2 * r + 1] - from[r]);
            const float e2 = ex2(s[u][2 * i + 1][2 * r] - from[r]), e3 = ex2(s[u][2 * i + 1][2 * r + 1] - from[r]);
            const float sum = (e0 + e1) + (e2 + e3);
            if (sum != 0.f) l[u][r] = fmaf(sum, inverse, l[u][r]);
            p[u][i][r] = none ? 0u : pack_half2(e0, e1);
            p[u][i][2 + r] = none ? 0u : pack_half2(e2, e3);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < kGroups; ++i)                                        // 16 keys
#pragma unroll
        for (int h = 0; h < kOut / 4; ++h) {
          uint32_t w[2][4];
#pragma unroll
          for (int t = 0; t < 2; ++t) ldmatrix4_turned(w[t], values + at_v + i * 16 * kPitch + (2 * h + t) * 32);
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int u = 0; u < MT; ++u) {
              mma16(o[u][4 * h + 2 * t], p[u][i], w[t][0], w[t][1]);
              mma16(o[u][4 * h + 2 * t + 1], p[u][i], w[t][2], w[t][3]);
            }
        }
    }
    if (tile + 1 < tiles) store(buf ^ 1);                                      // (the tile before this one has been read by all: the barrier below)
    __syncthreads();
  }
#pragma unroll
  for (int u = 0; u < MT; ++u)
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      float sum = l[u][r];
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      const int in_warp = 16 * u + 8 * r + g;
      if (in_warp >= rows) continue;
      if (sum < kFewLost && m[u][r] != -INFINITY) *a.tiles_again = 1;
      const int64_t row = first + in_warp, token = row / a.group, h = (int64_t)head * a.group + row - token * a.group;
      const float inv = sum == 0.f ? 0.f : kDenominators / sum;
      __nv_bfloat16* const to = a.out + (e.first + token) * a.ld_out + h * c.dim;
#pragma unroll
      for (int t = 0; t < kOut; ++t)
        if (8 * t < c.dim) *reinterpret_cast<uint32_t*>(to + 8 * t + 2 * cc) = pack_bf16x2(o[u][t][2 * r] * inv, o[u][t][2 * r + 1] * inv);
      if (cc == 0 && a.lse) a.lse[(e.first + token) * a.heads + h] = log_of(sum, m[u][r]);
    }
}

constexpr size_t share_bytes() { return (kMaxBlocks * sizeof(Share) + sizeof(int) + 255) / 256 * 256; }

template <int FMT, int DIM, bool NARROW>
qm_status launch_rows(RowsArgs& a, int* grid, cudaStream_t s) {
  constexpr auto kern = attention_rows<FMT, DIM, NARROW>;
  constexpr size_t smem = (size_t)kWarps * (NARROW ? 8 : 16) * (DIM + 4) * 4;
  a.rows = NARROW ? 8 : 16;
  a.cell = cell_of(DIM, NARROW);
  static std::atomic<int> resident[kMaxDevices];
  const int dev = current_device();
  if (dev < 0) return QM_ERR_UNSUPPORTED;
  int most = resident[dev].load(std::memory_order_relaxed);
  if (most == 0) {
    QM_CUDA_OK(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    QM_CUDA_OK(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&most, kern, kWarps * 32, smem));
    most = std::min(kMaxBlocks, std::max(1, most) * sm_count());
    resident[dev].store(most, std::memory_order_relaxed);
  }
  QM_CUDA_OK(launch_pdl(kern, dim3((unsigned)most), dim3(kWarps * 32), smem, s, a));
  count_launch();
  *grid = most;
  return QM_OK;
}
template <int FMT, int DIM, int MT>
qm_status launch_tiles(const RowsArgs& a, cudaStream_t s) {
  constexpr auto kern = attention_tiles<FMT, DIM, MT>;
  static std::atomic<bool> ready[kMaxDevices];
  const int dev = current_device();
  if (dev < 0) return QM_ERR_UNSUPPORTED;
  if (!ready[dev].load(std::memory_order_relaxed)) {
    QM_CUDA_OK(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)tiles_smem<DIM>(MT)));
    ready[dev].store(true, std::memory_order_relaxed);
  }
  // at most (sequences' rows of the tokens do not overlap): every 128 MT rows, and one more for each sequence that has most_rows or more
  const int64_t rows = a.c.tokens * a.group, most = rows / (128 * MT) + std::min<int64_t>(a.c.batch, rows / a.most_rows);
  QM_CUDA_OK(launch_pdl(kern, dim3((unsigned)most, (unsigned)a.c.kv_heads), dim3(256), tiles_smem<DIM>(MT), s, a));
  count_launch();
  return QM_OK;
}

// Which sequences are whose: attention_tiles takes those with 64 query rows of a cached head or more, if the call has enough of them to give a third
// of the SMs 128 rows; its thread blocks do not share keys, attention_rows does, whatever the rows.  256 rows to a thread block where there are enough for all SMs.
// How many rows one sequence has only the device knows: all of the call's, at most, but where there are as many tokens as sequences a token of each is
// taken for granted. (Beside sequences without new tokens, us without attention_tiles / with it: 1000 tokens on 2000 among 1023, 32 heads on 8 of 128, 386 / 162;
// 300 on 2000 among 400, 64 heads of 64, 147 / 97; in vain: 512 single tokens on 500, 32 heads on 8 of 128, 162 / 169.)
template <int FMT, int DIM>
qm_status launch_both(RowsArgs a, cudaStream_t s) {
  const int64_t blocks = a.c.tokens * a.group / 128 * a.c.kv_heads;
  const int64_t most_tokens = a.c.tokens == a.c.batch ? 1 : a.c.tokens;
  const bool tiles = most_tokens * a.group >= 64 && blocks >= sm_count() / 3 && a.c.kv_heads < 65536;
  a.most_rows = tiles ? 64 : 0x7fffffff;
  // eight rows to a cell where a sequence has no more on the average
  int grid = 0;
  qm_status st = a.c.tokens * a.group <= 8ll * a.c.batch ? launch_rows<FMT, DIM, true>(a, &grid, s) : launch_rows<FMT, DIM, false>(a, &grid, s);
  if (st == QM_OK && tiles) st = blocks >= 2 * sm_count() ? launch_tiles<FMT, DIM, 2>(a, s) : launch_tiles<FMT, DIM, 1>(a, s);
  if (st != QM_OK) return st;
  QM_CUDA_OK(launch_pdl(attention_join<FMT, DIM>, dim3((unsigned)grid, 4), dim3(DIM), 0, s, a, grid));
  count_launch();
  return QM_OK;
}
template <int FMT>
qm_status launch_dim(const RowsArgs& a, cudaStream_t s) { return a.c.dim <= 64 ? launch_both<FMT, 64>(a, s) : launch_both<FMT, 128>(a, s); }

}  // namespace

size_t cache_attention_workspace(int dim) { return share_bytes() + (size_t)2 * kMaxBlocks * kMostRows * ((dim <= 64 ? 64 : 128) + 2) * 4; }

qm_status launch_cache_attention(const CacheArgs& c, const AttentionArgs& l, cudaStream_t s) {
  RowsArgs a{};
  a.c = view_of(c);
  a.q = static_cast<const __nv_bfloat16*>(l.q); a.ld_q = l.ld_q;
  a.heads = l.heads; a.group = l.heads / c.kv_heads;
  a.scale_log2 = l.scale * 1.44269504f;
  a.out = static_cast<__nv_bfloat16*>(l.out); a.ld_out = l.ld_out; a.lse = l.lse;
  a.shares = static_cast<Share*>(l.ws);
  a.tiles_again = reinterpret_cast<int*>(a.shares + kMaxBlocks);
  a.parts = reinterpret_cast<float*>(static_cast<char*>(l.ws) + share_bytes());
  return c.fmt == QM_FMT_INT8 ? launch_dim<QM_FMT_INT8>(a, s) : c.fmt == QM_FMT_E4M3 ? launch_dim<QM_FMT_E4M3>(a, s) : launch_dim<QM_FMT_E5M2>(a, s);
}

}  // namespace qm
