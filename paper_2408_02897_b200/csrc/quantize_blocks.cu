// FP8 codes with a scale for each 128 entries of the contraction, of one row or of 128 rows (qm_quantize_blocks).
//
// Eq. 1 over each block: delta = max|x| / qmax, codes = sat(RTNE(x / delta)).  Bound by HBM (3 bytes an element of bf16), so every
// element is read once and stays in registers between its block's maximum and its codes: 16384 x 4096 bf16, a scale per row and block, 35.6 us, 5.7 TB/s, 0.87 of
// the measured copy's rate (75 us with elements held as fp32 and each lane computing every block's scale).  Three shapes:
//   blocks_rows     contraction contiguous, a scale per row: eight lanes to a block, four blocks of a row on their way at once
//   blocks_squares  contraction contiguous, squares of 128: a thread block each
//   blocks_strided  contraction strided: a thread has two neighbouring rows of 16 contraction entries, the codes are turned in shared memory
#include "quant_device.cuh"

namespace qm {
namespace {

struct BlockArgs {
  const void* x;
  int64_t ld;                  // elements between rows, or between contraction entries where those are strided
  int64_t nc; int c, ldc;
  uint8_t* codes;
  float* delta;                // [blocks of the contraction][blocks of rows]
  int64_t delta_cols;
};

// A block's scale from the bits of its maximum.  One that holds a NaN or Inf gets NaN and codes 0; one so small that the quotient with
// qmax is 0 in fp32 counts as one of zeros.  `recip` is 0 where the two-wide quotient does not serve or the codes are all 0.
struct BlockScale { float delta, recip; };
template <int FMT>
__device__ __forceinline__ BlockScale block_scale(uint32_t top) {
  BlockScale s;
  const float x = __uint_as_float(top), qmax = fmt_qmax(FMT);
  if (top >= 0x26800000u && top < 0x58800000u) {                // 2^-50 .. 2^50: the division by two corrections (see Quotient)
    constexpr float r = FMT == QM_FMT_E4M3 ? 1.f / 448.f : 1.f / 57344.f;
    const float q0 = x * r, q1 = fmaf(fmaf(-q0, qmax, x), r, q0);
    s.delta = fmaf(fmaf(-q1, qmax, x), r, q1);
    s.recip = __frcp_rn(s.delta);
  } else {
    const float d = __fdiv_rn(x, qmax);
    s.delta = top >= 0x7f800000u ? __int_as_float(0x7fffffff) : d == 0.f ? 1.f : d;
    s.recip = QuotientPair::serves(s.delta) && (top == 0 || d != 0.f) ? __frcp_rn(s.delta) : 0.f;
  }
  return s;
}
// Two codes under a scale that the two-wide quotient does not serve, or of a block whose codes are all 0 (delta is 1 or NaN then).
template <int FMT>
__device__ __noinline__ uint32_t far_pair(float x0, float x1, float delta) {
  if (!(delta < INFINITY) || QuotientPair::serves(delta)) return 0u;
  const Quotient quot(delta);
  return quant2<FMT>(quot(x0), quot(x1)) & 0xffffu;
}
__device__ __forceinline__ QuotientPair quotient_of(const BlockScale& s) {
  uint64_t r, d;
  asm("mov.b64 %0, {%1, %1};" : "=l"(r) : "f"(s.recip));
  asm("mov.b64 %0, {%1, %1};" : "=l"(d) : "f"(-s.delta));
  return QuotientPair(r, d);
}
template <int FMT>
__device__ __forceinline__ uint32_t cvt_pair(uint64_t q) {
  float lo, hi;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(q));
  return quant2<FMT>(lo, hi);
}
__device__ __forceinline__ uint64_t pair_of_bits(uint32_t lo, uint32_t hi) {
  uint64_t v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "r"(lo), "r"(hi));
  return v;
}

// Eight consecutive elements of a row as they lie in memory, zeros beyond its end.
template <typename T> struct Eight;
template <> struct Eight<__nv_bfloat16> {
  uint4 q;
  __device__ __forceinline__ uint32_t top() const {               // as fp32's bits
    constexpr uint32_t k = 0x7fff7fffu;
    const uint32_t m = __vmaxu2(__vmaxu2(q.x & k, q.y & k), __vmaxu2(q.z & k, q.w & k));
    return max(m << 16, m & 0xffff0000u);
  }
  // the quotient of a zero loses its sign: all signs are put back, four at a time
  template <int FMT>
  static __device__ __forceinline__ uint32_t codes4(uint32_t a, uint32_t b, const QuotientPair& quot) {
    const uint32_t lo = cvt_pair<FMT>(quot(pair_of_bits(a << 16, a & 0xffff0000u))), hi = cvt_pair<FMT>(quot(pair_of_bits(b << 16, b & 0xffff0000u)));
    return __byte_perm(lo, hi, 0x5410) | (__byte_perm(a, b, 0x7531) & 0x80808080u);
  }
  template <int FMT>
  __device__ __forceinline__ uint2 codes(const BlockScale& s) const {
    if (s.recip != 0.f) {
      const QuotientPair quot = quotient_of(s);
      return make_uint2(codes4<FMT>(q.x, q.y, quot), codes4<FMT>(q.z, q.w, quot));
    }
    auto two = [&](uint32_t w) { return far_pair<FMT>(bf16_lo(w), bf16_hi(w), s.delta); };
    return make_uint2(two(q.x) | two(q.y) << 16, two(q.z) | two(q.w) << 16);
  }
  static __device__ __forceinline__ Eight load(const __nv_bfloat16* row, int c, int cols) {
    Eight v;
    if (c + 8 <= cols) {
      v.q = __ldg(reinterpret_cast<const uint4*>(row + c));
      return v;
    }
    uint32_t e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = c + i < cols ? __ldg(reinterpret_cast<const unsigned short*>(row) + c + i) : 0u;
    v.q = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
    return v;
  }
};
template <> struct Eight<float> {
  Vec8 v;
  __device__ __forceinline__ uint32_t top() const { return absmax8(v, 0u); }
  template <int FMT>
  __device__ __forceinline__ uint2 codes(const BlockScale& s) const {
    uint32_t w[4];
    if (s.recip != 0.f) {
      const QuotientPair quot = quotient_of(s);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = quant_pair_x2<FMT>(v.v[2 * i], v.v[2 * i + 1], quot);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = far_pair<FMT>(v.v[2 * i], v.v[2 * i + 1], s.delta);
    }
    return make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
  }
  static __device__ __forceinline__ Eight load(const float* row, int c, int cols) {
    Eight e;
    if (c + 8 <= cols) {
      e.v = Loader<float>::load8(row + c);
      return e;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) e.v.v[i] = c + i < cols ? __ldg(row + c + i) : 0.f;
    return e;
  }
};

// 32 rows x 512 contraction entries a thread block, eight lanes to a row's block of 128, four blocks of the row each.  What a block costs once (its
// scale and the reciprocal) is computed for all four at a time, one in two of the eight lanes.
template <typename T, int FMT>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? 4 : 3) blocks_rows(const BlockArgs a) {
  pdl_prologue();
  const int j = threadIdx.x & 7, kb0 = blockIdx.y * 4;
  const int64_t row = (int64_t)blockIdx.x * 32 + (threadIdx.x >> 3);
  const bool in = row < a.nc;
  const T* const x = static_cast<const T*>(a.x) + (in ? row : 0) * a.ld;
  Eight<T> v[4][2];
  uint32_t m[4];
#pragma unroll
  for (int b = 0; b < 4; ++b)
#pragma unroll
    for (int h = 0; h < 2; ++h) v[b][h] = Eight<T>::load(x, (kb0 + b) * kScaleBlock + 64 * h + 8 * j, a.c);
#pragma unroll
  for (int b = 0; b < 4; ++b) m[b] = max(v[b][0].top(), v[b][1].top());
  // the maxima of the eight lanes: lane j ends with that of block j / 2
  const bool b2 = j & 4, b1 = j & 2;
  uint32_t m0 = max(b2 ? m[2] : m[0], __shfl_xor_sync(0xffffffffu, b2 ? m[0] : m[2], 4));
  uint32_t m1 = max(b2 ? m[3] : m[1], __shfl_xor_sync(0xffffffffu, b2 ? m[1] : m[3], 4));
  m0 = max(b1 ? m1 : m0, __shfl_xor_sync(0xffffffffu, b1 ? m0 : m1, 2));
  m0 = max(m0, __shfl_xor_sync(0xffffffffu, m0, 1));
  const BlockScale mine = block_scale<FMT>(m0);
  if ((j & 1) == 0 && in && (kb0 + (j >> 1)) * kScaleBlock < a.c) a.delta[(int64_t)(kb0 + (j >> 1)) * a.delta_cols + row] = mine.delta;
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    const int from = (threadIdx.x & 24) + 2 * b;
    const BlockScale s{__shfl_sync(0xffffffffu, mine.delta, from), __shfl_sync(0xffffffffu, mine.recip, from)};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int c = (kb0 + b) * kScaleBlock + 64 * h + 8 * j;
      if (in && c < a.ldc) *reinterpret_cast<uint2*>(a.codes + row * a.ldc + c) = v[b][h].template codes<FMT>(s);
    }
  }
}

// A square of 128 a thread block: 16 lanes to a row, 16 rows at a time.
template <typename T, int FMT>
__global__ void __launch_bounds__(kThreads) blocks_squares(const BlockArgs a) {
  pdl_prologue();
  const int c = blockIdx.x * kScaleBlock + 8 * (threadIdx.x & 15);
  const int64_t row0 = (int64_t)blockIdx.y * 128 + (threadIdx.x >> 4);
  Eight<T> v[8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t row = row0 + 16 * i;
    v[i] = Eight<T>::load(static_cast<const T*>(a.x) + (row < a.nc ? row : 0) * a.ld, c, row < a.nc ? a.c : 0);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, v[i].top());
  __shared__ uint32_t tops[kThreads / 32];
  top = __reduce_max_sync(0xffffffffu, top);
  if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
  __syncthreads();
  const BlockScale s = block_scale<FMT>(__reduce_max_sync(0xffffffffu, tops[threadIdx.x & 7]));
  if (threadIdx.x == 0) a.delta[(int64_t)blockIdx.x * a.delta_cols + blockIdx.y] = s.delta;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t row = row0 + 16 * i;
    if (row < a.nc && c < a.ldc) *reinterpret_cast<uint2*>(a.codes + row * a.ldc + c) = v[i].template codes<FMT>(s);
  }
}

// 128 contraction entries x 64 SUB rows a thread block; warp w has entries 16 w ..., a lane rows 2 lane, 2 lane + 1 of each 64.  SUB = 2: one
// scale for all of it.
template <typename T, int FMT, int SUB>
__global__ void __launch_bounds__(kThreads) blocks_strided(const BlockArgs a) {
  constexpr int kPitch = 144;                                  // of a row of codes in shared memory
  __shared__ uint32_t tops[8][64];
  __shared__ __align__(16) uint8_t turned[64 * SUB][kPitch];
  pdl_prologue();
  const int w = threadIdx.x >> 5, lane = threadIdx.x & 31, k0 = blockIdx.y * kScaleBlock;
  const int64_t r0 = (int64_t)blockIdx.x * 64 * SUB;
  float v[SUB][16][2];
#pragma unroll
  for (int u = 0; u < SUB; ++u)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int k = k0 + 16 * w + i;
      const int64_t r = r0 + 64 * u + 2 * lane;
      const T* const p = static_cast<const T*>(a.x) + (int64_t)k * a.ld + r;
      v[u][i][0] = v[u][i][1] = 0.f;
      if (k < a.c && r + 1 < a.nc) {
        if (sizeof(T) == 2) {
          const uint32_t two = __ldg(reinterpret_cast<const uint32_t*>(p));
          v[u][i][0] = bf16_lo(two); v[u][i][1] = bf16_hi(two);
        } else {
          const float2 two = __ldg(reinterpret_cast<const float2*>(p));
          v[u][i][0] = two.x; v[u][i][1] = two.y;
        }
      } else if (k < a.c && r < a.nc) {
        v[u][i][0] = Loader<T>::load1(p, 0);
      }
    }
  uint32_t top[2] = {0u, 0u};
#pragma unroll
  for (int u = 0; u < SUB; ++u)
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) top[h] = max(top[h], absbits_f32(__float_as_uint(v[u][i][h])));
  if (SUB == 1) {
    *reinterpret_cast<uint2*>(&tops[w][2 * lane]) = make_uint2(top[0], top[1]);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint2 t = *reinterpret_cast<const uint2*>(&tops[i][2 * lane]);
      top[0] = max(top[0], t.x); top[1] = max(top[1], t.y);
    }
  } else {
    const uint32_t t = __reduce_max_sync(0xffffffffu, max(top[0], top[1]));
    if (lane == 0) tops[0][w] = t;
    __syncthreads();
    top[0] = top[1] = __reduce_max_sync(0xffffffffu, tops[0][lane & 7]);
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const BlockScale s = block_scale<FMT>(top[h]);
    const QuotientPair quot = quotient_of(s);
    if (SUB == 1) {
      const int64_t r = r0 + 2 * lane + h;
      if (w == 0 && r < a.nc) a.delta[(int64_t)blockIdx.y * a.delta_cols + r] = s.delta;
    } else if (threadIdx.x == 0 && h == 0) {
      a.delta[(int64_t)blockIdx.y * a.delta_cols + blockIdx.x] = s.delta;
    }
#pragma unroll
    for (int u = 0; u < SUB; ++u) {
      uint32_t c[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) c[i] = s.recip != 0.f ? quant_pair_x2<FMT>(v[u][2 * i][h], v[u][2 * i + 1][h], quot)
                                                             : far_pair<FMT>(v[u][2 * i][h], v[u][2 * i + 1][h], s.delta);
      *reinterpret_cast<uint4*>(&turned[64 * u + 2 * lane + h][16 * w]) =
          make_uint4(c[0] | c[1] << 16, c[2] | c[3] << 16, c[4] | c[5] << 16, c[6] | c[7] << 16);
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2 * SUB; ++i) {
    const int r = 32 * i + (threadIdx.x >> 3), c = 16 * (threadIdx.x & 7);
    if (r0 + r < a.nc && k0 + c < a.ldc)
      *reinterpret_cast<uint4*>(a.codes + (r0 + r) * a.ldc + k0 + c) = *reinterpret_cast<const uint4*>(&turned[r][c]);
  }
}

template <typename T, int FMT>
qm_status launch_typed(const BlockArgs& a, bool contiguous, int side, cudaStream_t s) {
  const unsigned kb = (unsigned)((a.c + kScaleBlock - 1) / kScaleBlock);
  auto tiles = [&](int64_t rows) { return (unsigned)((a.nc + rows - 1) / rows); };
  if (!contiguous) {
    if (side == 1) QM_CUDA_OK(launch_pdl(blocks_strided<T, FMT, 1>, dim3(tiles(64), kb), dim3(kThreads), 0, s, a));
    else QM_CUDA_OK(launch_pdl(blocks_strided<T, FMT, 2>, dim3(tiles(128), kb), dim3(kThreads), 0, s, a));
  } else if (side == 1) {
    QM_CUDA_OK(launch_pdl(blocks_rows<T, FMT>, dim3(tiles(32), (kb + 3) / 4), dim3(kThreads), 0, s, a));
  } else {
    QM_CUDA_OK(launch_pdl(blocks_squares<T, FMT>, dim3(kb, tiles(128)), dim3(kThreads), 0, s, a));
  }
  count_launch();
  return QM_OK;
}

}  // namespace

qm_status launch_quantize_blocks(const View& x, int fmt, int side, float* delta, uint8_t* codes, cudaStream_t s) {
  const bool contiguous = x.c_contig();
  BlockArgs a{x.data, contiguous ? x.s_nc : x.s_c, x.nc, (int)x.c, (int)qm_code_ld(x.c), codes, delta, (x.nc + side - 1) / side};
  // a grid's second extent
  if ((x.c + kScaleBlock - 1) / kScaleBlock > 65535 || (contiguous && side != 1 && a.delta_cols > 65535)) return QM_ERR_UNSUPPORTED;
  if (x.dtype == QM_DT_BF16)
    return fmt == QM_FMT_E4M3 ? launch_typed<__nv_bfloat16, QM_FMT_E4M3>(a, contiguous, side, s) : launch_typed<__nv_bfloat16, QM_FMT_E5M2>(a, contiguous, side, s);
  return fmt == QM_FMT_E4M3 ? launch_typed<float, QM_FMT_E4M3>(a, contiguous, side, s) : launch_typed<float, QM_FMT_E5M2>(a, contiguous, side, s);
}

}  // namespace qm
