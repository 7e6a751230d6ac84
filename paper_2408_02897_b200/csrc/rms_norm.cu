// Root-mean-square norm with the residual's addition and an output in 8 bits (qm_rms_norm_quantize).
//
// Per row: z = x + residual, rounded to the stream's type; v = z w in fp32; Eq. 1 over v: d = max|v| / qmax,
// code = sat(RTNE(v / d)).  The norm's factor f = 1 / sqrt(mean(z^2) + eps) is the same positive number for the whole
// row, so it cancels in v f / (max|v f| / qmax) and goes into the scale alone: delta = d f.  The codes
// are therefore those of qm_quantize for v, independent of the order in which the squares are added.
//
// Bound by HBM: 7 bytes an element of a bf16 stream (x and residual read, z and codes written), so every element is touched once: a
// row's v stay in registers between its maximum and its codes, and persistent blocks have the next rows on their way meanwhile.
// 16384 x 4096 bf16 with a residual 75 us, 6.3 TB/s, 0.96 of a copy's 6.55 at its best (one of as many bytes, timed as this was, 73 us); rows that do not start on 16 bytes (4095
// elements) 105 us, where the instructions that move them into place are what it takes (247 a warp and 256 elements, 174 without).
#include <algorithm>
#include <atomic>

#include "quant_device.cuh"

namespace qm {
namespace {

struct NormArgs {
  const void* x; int64_t ld_x;
  const void* res; int64_t ld_res;        // null: nothing is added
  void* res_out; int64_t ld_out;
  const void* w; int w_bf16, w_vec;       // w_vec: on 16 bytes
  float eps;
  int64_t rows;
  int cols, ldc, fmt;
  uint8_t* codes;
  float* delta;
};

// Eight consecutive elements as they lie in memory, which need not be on 16 bytes: rows of any pitch are read and written in
// aligned 16-byte granules all the same, and moved into place in registers.
template <typename T>
struct Raw {
  static constexpr int kG = 16 / sizeof(T);               // elements of a granule
  static constexpr int kQ = 8 / kG;                       // granules of eight elements
  uint4 q[kQ];
  __device__ __forceinline__ uint32_t word(int i) const { const uint4& v = q[i >> 2]; return (i & 3) == 0 ? v.x : (i & 3) == 1 ? v.y : (i & 3) == 2 ? v.z : v.w; }
  __device__ __forceinline__ float at(int i) const {
    if (sizeof(T) == 4) return __uint_as_float(word(i));
    return i & 1 ? bf16_hi(word(i >> 1)) : bf16_lo(word(i >> 1));
  }
};

// A row's first granule and the place of its first element there.
template <typename T>
struct Row {
  const uint4* base;
  int off;
  __device__ __forceinline__ explicit Row(const T* p)
      : base(reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(p) & ~(uintptr_t)15)),
        off((int)((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T))) {}
};

// Asynchronous copies of 16 bytes past L1; every thread waits for its own.
__device__ __forceinline__ void copy16(uint32_t dst, const uint4* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }
__device__ __forceinline__ uint4 lds16(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}

__device__ __forceinline__ uint32_t lds4(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void sts16(uint32_t addr, const uint4& v) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// A lane's eight elements of a warp's piece in shared memory, the first of which is element `off` of the lane's first granule (the same
// for the whole row).  bf16 by words from there on, four lanes to a bank: less than moving two granules' words into place.
__device__ __forceinline__ void take(Raw<__nv_bfloat16>& r, uint32_t from, int off) {
  if (off == 0) { r.q[0] = lds16(from); return; }
  from += 4 * (off >> 1);
  uint32_t w[5];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = lds4(from + 4 * i);
  if (off & 1) {
    w[4] = lds4(from + 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
  }
  r.q[0] = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void take(Raw<float>& r, uint32_t from, int off) {
  r.q[0] = lds16(from); r.q[1] = lds16(from + 16);
  if (off == 0) return;
  const uint4 a = r.q[0], b = r.q[1], c = lds16(from + 32);
  r.q[0] = off == 1 ? make_uint4(a.y, a.z, a.w, b.x) : off == 2 ? make_uint4(a.z, a.w, b.x, b.y) : make_uint4(a.w, b.x, b.y, b.z);
  r.q[1] = off == 1 ? make_uint4(b.y, b.z, b.w, c.x) : off == 2 ? make_uint4(b.z, b.w, c.x, c.y) : make_uint4(b.w, c.x, c.y, c.z);
}

// Two fp32 values per register pair: one instruction for both.
__device__ __forceinline__ uint64_t pair_of(float lo, float hi) { uint64_t v; asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi)); return v; }
__device__ __forceinline__ void halves(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t mul2(uint64_t x, uint64_t y) { uint64_t d; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(x), "l"(y)); return d; }
__device__ __forceinline__ uint64_t fma2(uint64_t x, uint64_t y, uint64_t z) { uint64_t d; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(x), "l"(y), "l"(z)); return d; }

// x + r in the stream's type.  For bf16 the sum rounded once is the fp32 sum rounded to bf16: where the fp32 sum is not exact the
// smaller operand is below 2^-15 of the larger one, which is on bf16's grid, and both come out as that.
__device__ __forceinline__ uint32_t add_word(uint32_t x, uint32_t r, __nv_bfloat16) {
  uint32_t z;
  asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(z) : "r"(x), "r"(r));
  return z;
}
__device__ __forceinline__ uint32_t add_word(uint32_t x, uint32_t r, float) { return __float_as_uint(__fadd_rn(__uint_as_float(x), __uint_as_float(r))); }
template <typename T>
__device__ __forceinline__ void add(Raw<T>& x, const Raw<T>& r) {
#pragma unroll
  for (int i = 0; i < Raw<T>::kQ; ++i)
    x.q[i] = make_uint4(add_word(x.q[i].x, r.q[i].x, T()), add_word(x.q[i].y, r.q[i].y, T()), add_word(x.q[i].z, r.q[i].z, T()),
                        add_word(x.q[i].w, r.q[i].w, T()));
}
// zeros from element n on
template <typename T>
__device__ __forceinline__ void keep(Raw<T>& x, int n) {
  uint32_t w[4 * Raw<T>::kQ];
#pragma unroll
  for (int i = 0; i < 4 * Raw<T>::kQ; ++i) {
    w[i] = x.word(i);
    if (sizeof(T) == 4) w[i] = i < n ? w[i] : 0u;
    else w[i] = 2 * i + 1 < n ? w[i] : 2 * i < n ? w[i] & 0xffffu : 0u;
  }
#pragma unroll
  for (int i = 0; i < Raw<T>::kQ; ++i) x.q[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
}
// The warp's 256 consecutive elements z, eight a lane and the first lane's from element c0 on, to row p.  Rows that do not start on
// 16 bytes go through the warp's shared memory at `via`, an element per lane and store: whole sectors without regard to the row's place.
// (Granules that lanes pass on to their neighbours, with the piece's ends by themselves, took 200 instructions for these 30.)
template <typename T>
__device__ __forceinline__ void store_z(T* p, int c0, int lane, const Raw<T>& r, int cols, uint32_t via) {
  constexpr int kQ = Raw<T>::kQ;
  const int c = c0 + 8 * lane;
  if ((reinterpret_cast<uintptr_t>(p) & 15) == 0 && c0 + 256 <= cols) {
#pragma unroll
    for (int i = 0; i < kQ; ++i) reinterpret_cast<uint4*>(p + c)[i] = r.q[i];
    return;
  }
  __syncwarp();
#pragma unroll
  for (int i = 0; i < kQ; ++i) sts16(via + (lane * kQ + i) * 16, r.q[i]);
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int e = 32 * i + lane;
    if (c0 + e >= cols) continue;
    if (sizeof(T) == 4) reinterpret_cast<uint32_t*>(p)[c0 + e] = lds4(via + 4 * e);
    else {
      uint16_t v;
      asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(via + 2 * e) : "memory");
      reinterpret_cast<uint16_t*>(p)[c0 + e] = v;
    }
  }
}

// w[c .. c + 8), zeros from `cols` on, as pairs
__device__ __forceinline__ void load_w(const NormArgs& a, int c, uint64_t (&w)[4]) {
  float f[8];
  if (c + 8 <= a.cols && a.w_vec) {
    const Vec8 v = a.w_bf16 ? Loader<__nv_bfloat16>::load8(static_cast<const __nv_bfloat16*>(a.w) + c)
                            : Loader<float>::load8(static_cast<const float*>(a.w) + c);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = v.v[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      f[i] = c + i >= a.cols ? 0.f : a.w_bf16 ? Loader<__nv_bfloat16>::load1(a.w, c + i) : Loader<float>::load1(a.w, c + i);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = pair_of(f[2 * i], f[2 * i + 1]);
}

// the larger magnitude; a NaN stays
__device__ __forceinline__ float max_abs(float m, float v) {
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(m) : "f"(fabsf(v)));
  return m;
}
__device__ __forceinline__ float max_abs(float m, float v, float u) {
  asm("max.NaN.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(fabsf(v)), "f"(fabsf(u)));
  return m;
}

// top / qmax, correctly rounded (two residual corrections, as in Quotient) without a division's instructions for what is neither
// tiny nor infinite.
__device__ __forceinline__ float eq1_scale(float top, int fmt) {
  const float qmax = fmt_qmax(fmt);
  if (!(top >= 8.6736174e-19f && top <= 1.1529215e18f)) return top / qmax;
  const float r = fmt == QM_FMT_INT8 ? 1.f / 127.f : fmt == QM_FMT_E4M3 ? 1.f / 448.f : 1.f / 57344.f;
  const float q0 = top * r;
  const float q1 = fmaf(fmaf(-q0, qmax, top), r, q0);
  return fmaf(fmaf(-q1, qmax, top), r, q1);
}

template <int FMT>
__device__ __forceinline__ uint2 codes8(const uint64_t (&v)[4], const QuotientPair& quot) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float lo, hi;
    halves(v[i], lo, hi);
    w[i] = quant_bits_pair<FMT>(__float_as_uint(lo), __float_as_uint(hi), quot);
  }
  return make_uint2(__byte_perm(w[0], w[1], 0x5410), __byte_perm(w[2], w[3], 0x5410));
}
__device__ __forceinline__ uint2 codes8(const uint64_t (&v)[4], const QuotientPair& quot, int fmt) {
  return fmt == QM_FMT_INT8 ? codes8<QM_FMT_INT8>(v, quot) : fmt == QM_FMT_E4M3 ? codes8<QM_FMT_E4M3>(v, quot) : codes8<QM_FMT_E5M2>(v, quot);
}
// under scales outside QuotientPair's range
__device__ __noinline__ uint32_t code_far(float v, float own, int fmt) {
  const float t = Quotient(own)(v);
  return (fmt == QM_FMT_INT8 ? quant2<QM_FMT_INT8>(t, 0.f) : fmt == QM_FMT_E4M3 ? quant2<QM_FMT_E4M3>(t, 0.f) : quant2<QM_FMT_E5M2>(t, 0.f)) & 0xffu;
}

__host__ __device__ constexpr int block_threads(int tpr) { return tpr < 256 ? 256 : tpr; }

// What the threads of a row agree on: Eq. 1's scale of its v, and the row's delta (in the thread that stores it).  A scale that is 0 in
// fp32, though v is not, has no quotients: such a row counts as one of zeros.
__device__ __forceinline__ float row_delta(const NormArgs& a, float own, uint32_t top_bits, float sum, bool finite) {
  if (!finite) return __int_as_float(0x7fffffff);
  if (top_bits == 0 || own == 0.f) return 1.f;
  const float mean = sum / (float)a.cols, square = mean + a.eps;
  // (a quarter of either where their sum leaves fp32, which its root does not)
  return own * (square < INFINITY ? 1.f / sqrtf(square) : 0.5f / sqrtf(0.25f * mean + 0.25f * a.eps));
}

// Shared memory: a ring of rows on their way in.  A warp's piece is 256 elements: 32 x kQ granules and one more, for rows that do not
// start on 16 bytes.  Every warp copies what it reads itself, so the ring needs no barrier of the block.
template <typename T, int TPR, int N, bool RES>
struct Ring {
  static constexpr int kThreads = block_threads(TPR), kRows = kThreads / TPR;
  static constexpr uint32_t kPiece = (32 * Raw<T>::kQ + 1) * 16, kWarpStage = (RES ? 2 : 1) * N * kPiece;
  // two blocks of 256 threads to an SM, which is what their registers leave room for, up to four rows deep
  static constexpr int kFit = (kThreads >= 512 ? 208 * 1024 : 104 * 1024) / (kThreads / 32 * kWarpStage);
  static constexpr int kStages = kFit < 1 ? 1 : kFit > 4 ? 4 : kFit;
  static constexpr uint32_t kBytes = kStages * (kThreads / 32) * kWarpStage;
};

// TPR threads to a row, each with N pieces of eight consecutive elements, TPR pieces apart; persistent, the next rows on their way
// while a row is worked on.
template <typename T, int TPR, int N, bool RES>
__global__ void __launch_bounds__(block_threads(TPR)) rms_norm_rows(const NormArgs a) {
  extern __shared__ uint4 ring_raw[];
  using R = Ring<T, TPR, N, RES>;
  constexpr int kRows = R::kRows, kWarps = TPR / 32, kStages = R::kStages, kG = Raw<T>::kG, kQ = Raw<T>::kQ;
  __shared__ float sums[2][kRows][kWarps];
  __shared__ uint32_t tops[2][kRows][kWarps];
  pdl_prologue();
  const int t = threadIdx.x % TPR, slot = threadIdx.x / TPR, lane = threadIdx.x & 31;
  const uint32_t mine = (uint32_t)__cvta_generic_to_shared(ring_raw) + (threadIdx.x >> 5) * kStages * R::kWarpStage;
  const int64_t first = (int64_t)blockIdx.x * kRows + slot, step = (int64_t)gridDim.x * kRows;

  auto fetch = [&](const void* tensor, int64_t ld, int64_t row, uint32_t to) {
    const Row<T> src(static_cast<const T*>(tensor) + row * ld);
    const int end = src.off + a.cols;                      // in elements of granules from the row's first one on
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = (t + i * TPR) * 8;
#pragma unroll
      for (int k = 0; k < kQ; ++k)
        if (c + k * kG < end) copy16(to + i * R::kPiece + (lane * kQ + k) * 16, src.base + c / kG + k);
      if (lane == 31 && c + 8 < end) copy16(to + i * R::kPiece + 32 * kQ * 16, src.base + c / kG + kQ);
    }
  };
  auto prefetch = [&](int64_t row, int stage) {
    if (row < a.rows) {
      const uint32_t to = mine + stage * R::kWarpStage;
      fetch(a.x, a.ld_x, row, to);
      if (RES) fetch(a.res, a.ld_res, row, to + N * R::kPiece);
    }
    copies_commit();
  };
#pragma unroll
  for (int k = 0; k < kStages - 1; ++k) prefetch(first + k * step, k);
  uint64_t w[N][4];
#pragma unroll
  for (int i = 0; i < N; ++i) load_w(a, (t + i * TPR) * 8, w[i]);

  int stage = 0, ahead = kStages - 1, buf = 0;
  for (int64_t row = first; row < a.rows; row += step, buf ^= 1) {
    __syncwarp();                                            // the stage that is filled next has been read by all lanes
    prefetch(row + (kStages - 1) * step, ahead);
    copies_wait<kStages - 1>();
    __syncwarp();
    const int off_x = Row<T>(static_cast<const T*>(a.x) + row * a.ld_x).off, off_r = RES ? Row<T>(static_cast<const T*>(a.res) + row * a.ld_res).off : 0;
    T* const z = static_cast<T*>(a.res_out) + row * a.ld_out;
    const uint32_t from = mine + stage * R::kWarpStage + lane * kQ * 16;
    ahead = stage;
    stage = stage == kStages - 1 ? 0 : stage + 1;

    uint64_t v[N][4], sum2 = 0;
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = (t + i * TPR) * 8, n = a.cols - c;
      if (c - 8 * lane >= a.ldc) continue;                   // the whole warp beyond the row
      Raw<T> rx;
      take(rx, from + i * R::kPiece, off_x);
      if (RES) {
        Raw<T> rr;
        take(rr, from + (N + i) * R::kPiece, off_r);
        add(rx, rr);
      }
      if (n < 8) keep(rx, n);
      if (RES) store_z(z, c - 8 * lane, lane, rx, a.cols, from - lane * kQ * 16 + i * R::kPiece);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint64_t z2 = pair_of(rx.at(2 * j), rx.at(2 * j + 1));
        sum2 = fma2(z2, z2, sum2);
        v[i][j] = mul2(z2, w[i][j]);
        float lo, hi;
        halves(v[i][j], lo, hi);
        top = max_abs(top, lo, hi);
      }
    }
    float sum, sum_hi;
    halves(sum2, sum, sum_hi);
    sum += sum_hi;
    uint32_t bits = __reduce_max_sync(0xffffffffu, __float_as_uint(top));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (kWarps > 1) {
      // (two buffers: a warp that is a row ahead writes the other one)
      if (lane == 0) { sums[buf][slot][t >> 5] = sum; tops[buf][slot][t >> 5] = bits; }
      asm volatile("bar.sync %0, %1;" ::"r"(1 + slot), "n"(TPR) : "memory");
      sum = sums[buf][slot][lane % kWarps];
      bits = __reduce_max_sync(0xffffffffu, tops[buf][slot][lane % kWarps]);
#pragma unroll
      for (int o = kWarps / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    }
    const bool finite = bits < 0x7f800000u && sum < INFINITY;
    const float own = bits == 0 ? 1.f : eq1_scale(__uint_as_float(bits), a.fmt);
    if (t == 0) a.delta[row] = row_delta(a, own, bits, sum, finite);
    uint8_t* const codes = a.codes + row * a.ldc;
    if (finite && QuotientPair::serves(own)) {
      const QuotientPair quot(own);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int c = (t + i * TPR) * 8;
        if (c < a.ldc) *reinterpret_cast<uint2*>(codes + c) = codes8(v[i], quot, a.fmt);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int c = (t + i * TPR) * 8;
        if (c >= a.ldc) continue;
        uint32_t q[2] = {};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float lo, hi;
          halves(v[i][j], lo, hi);
          if (finite && own != 0.f) q[j >> 1] |= (code_far(lo, own, a.fmt) | code_far(hi, own, a.fmt) << 8) << (16 * (j & 1));
        }
        *reinterpret_cast<uint2*>(codes + c) = make_uint2(q[0], q[1]);
      }
    }
  }
}

// Rows that no block holds in registers: a block per row, v formed again for the codes from x or, with a residual, from z as this
// thread has left it.  A thread's squares may be a million, so its sum carries along what each addition has rounded off (Kahan): without that
// 2^24 equal elements were 5e-5 off, and a sum in 64 bits takes 433 us for 2048 x 32768 where this takes 289 and the plain one 278 (bf16 with a residual).
template <typename T>
__global__ void __launch_bounds__(1024) rms_norm_long(const NormArgs a) {
  pdl_prologue();
  const int64_t row = blockIdx.x;
  const T* const x = static_cast<const T*>(a.x) + row * a.ld_x;
  const T* const r = static_cast<const T*>(a.res) + row * a.ld_res;
  T* const z = static_cast<T*>(a.res_out) + row * a.ld_out;
  auto weight = [&](int c) { return a.w_bf16 ? Loader<__nv_bfloat16>::load1(a.w, c) : Loader<float>::load1(a.w, c); };
  float sum = 0.f, over = 0.f, top = 0.f;
  for (int c = threadIdx.x; c < a.cols; c += 1024) {
    float zf = (float)x[c];
    if (a.res) {
      const T rounded = (T)(zf + (float)r[c]);
      z[c] = rounded;
      zf = (float)rounded;
    }
    const float term = fmaf(zf, zf, -over), next = sum + term;
    over = (next - sum) - term;
    sum = next;
    top = max_abs(top, zf * weight(c));
  }
  __shared__ float sums[32];
  __shared__ uint32_t tops[32];
  uint32_t bits = __reduce_max_sync(0xffffffffu, __float_as_uint(top));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if ((threadIdx.x & 31) == 0) { sums[threadIdx.x >> 5] = sum; tops[threadIdx.x >> 5] = bits; }
  __syncthreads();
  sum = sums[threadIdx.x & 31];
  bits = __reduce_max_sync(0xffffffffu, tops[threadIdx.x & 31]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  const bool finite = bits < 0x7f800000u && sum < INFINITY;
  const float own = bits == 0 ? 1.f : eq1_scale(__uint_as_float(bits), a.fmt);
  if (threadIdx.x == 0) a.delta[row] = row_delta(a, own, bits, sum, finite);
  const T* const from = a.res ? z : x;
  uint8_t* const codes = a.codes + row * a.ldc;
  for (int c = threadIdx.x; c < a.ldc; c += 1024)
    codes[c] = finite && own != 0.f && c < a.cols ? (uint8_t)code_far((float)from[c] * weight(c), own, a.fmt) : (uint8_t)0;
}

template <typename T, int TPR, int N, bool RES>
qm_status launch_rows(const NormArgs& a, cudaStream_t s) {
  using R = Ring<T, TPR, N, RES>;
  constexpr auto kern = rms_norm_rows<T, TPR, N, RES>;
  static std::atomic<int> resident[kMaxDevices];             // blocks that a device holds at once; 0 = not yet asked
  const int dev = current_device();
  if (dev < 0) return QM_ERR_UNSUPPORTED;
  int most = resident[dev].load(std::memory_order_relaxed);
  if (most == 0) {
    QM_CUDA_OK(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)R::kBytes));
    QM_CUDA_OK(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&most, kern, R::kThreads, R::kBytes));
    most = std::max(1, most) * sm_count();
    resident[dev].store(most, std::memory_order_relaxed);
  }
  const int64_t blocks = (a.rows + R::kRows - 1) / R::kRows;
  QM_CUDA_OK(launch_pdl(kern, dim3((unsigned)std::min<int64_t>(blocks, most)), dim3(R::kThreads), R::kBytes, s, a));
  count_launch();
  return QM_OK;
}

// The shape for a row of ldc codes.  Two pieces a thread or more spread what a row costs as a whole (its reductions, quotients,
// addresses: as many instructions as a piece) while some 100 registers still leave two blocks to an SM; where the granules of fp32 rows are
// held beside a residual's, four pieces take 200.  us, (threads to a row, pieces a thread), bf16 with a residual if nothing is said:
//   16384 x 512 (32, 2) 12.8; 700 (32, 4) 20.1, (64, 2) 24.8; 900 24.9, 27.7; 1024 22.8, 22.8, fp32 with 42.3, 39.5, without 17.6, 20.3;
//   16384 x 1025 (64, 3) 37.0, (128, 2) 46.0; 2048 (128, 2) 40.8, (64, 4) 43.0; 4096 (256, 2) 75.3, (128, 4) 79.7, (512, 1) 95.4;
//   8192 x 5000 (256, 4) 55.9, (512, 2) 72.9; fp32 without 46.1, 80.9, with (256, 3) 92.7, (512, 2) 106, (256, 4) 153;
//   8192 x 8192 (256, 4) 80.7, (512, 2) 80.0; fp32 without 63.4, 95.0, with 199, 144.
// Rows that one SM each can hold are a matter of latency: one piece a thread (1 row of 1024 (128, 1) 1.9, (64, 2) 2.2; of 4096 (512, 1) 2.4,
// (256, 2) 2.5), and so, up to 1024, are some thousands (1000 rows of 1024 (64, 2) 3.2, (32, 4) 3.7).
template <typename T, bool RES>
qm_status launch_norm(const NormArgs& a, cudaStream_t s) {
  constexpr bool wide = sizeof(T) == 4 && RES;
  if (a.rows <= sm_count() && a.ldc <= 4096) {
    if (a.ldc <= 1024) return launch_rows<T, 128, 1, RES>(a, s);
    return a.ldc <= 2048 ? launch_rows<T, 256, 1, RES>(a, s) : launch_rows<T, 512, 1, RES>(a, s);
  }
  if (a.ldc <= 512) return launch_rows<T, 32, 2, RES>(a, s);
  if constexpr (!wide)
    if (a.ldc <= 1024 && a.rows >= 32 * sm_count()) return launch_rows<T, 32, 4, RES>(a, s);
  if (a.ldc <= 1024) return launch_rows<T, 64, 2, RES>(a, s);
  if (a.ldc <= 1536) return launch_rows<T, 64, 3, RES>(a, s);
  if (a.ldc <= 2048) return launch_rows<T, 128, 2, RES>(a, s);
  if (a.ldc <= 8 * 128 * 3) return launch_rows<T, 128, 3, RES>(a, s);
  if (a.ldc <= 4096) return launch_rows<T, 256, 2, RES>(a, s);
  if constexpr (wide) {
    if (a.ldc <= 8 * 256 * 3) return launch_rows<T, 256, 3, RES>(a, s);
    if (a.ldc <= 8192) return launch_rows<T, 512, 2, RES>(a, s);
  } else {
    if (a.ldc <= 8192) return launch_rows<T, 256, 4, RES>(a, s);
  }
  if (a.ldc <= 16384) return launch_rows<T, 1024, 2, RES>(a, s);
  QM_CUDA_OK(launch_pdl(rms_norm_long<T>, dim3((unsigned)a.rows), dim3(1024), 0, s, a));
  count_launch();
  return QM_OK;
}

}  // namespace

qm_status launch_rms_norm(const RowsView& x, const RowsView& residual, void* residual_out, int64_t ld_out,
                          const void* weight, int weight_dtype, float eps, int fmt, uint8_t* codes, float* delta,
                          cudaStream_t s) {
  NormArgs a{};
  a.x = x.data; a.ld_x = x.ld; a.res = residual.data; a.ld_res = residual.ld;
  a.res_out = residual_out; a.ld_out = ld_out;
  a.w = weight; a.w_bf16 = weight_dtype == QM_DT_BF16; a.w_vec = reinterpret_cast<uintptr_t>(weight) % 16 == 0;
  a.eps = eps; a.rows = x.rows; a.fmt = fmt;
  a.cols = (int)x.cols; a.ldc = (int)qm_code_ld(x.cols); a.codes = codes; a.delta = delta;
  if (x.dtype == QM_DT_BF16) return a.res ? launch_norm<__nv_bfloat16, true>(a, s) : launch_norm<__nv_bfloat16, false>(a, s);
  return a.res ? launch_norm<float, true>(a, s) : launch_norm<float, false>(a, s);
}

}  // namespace qm
