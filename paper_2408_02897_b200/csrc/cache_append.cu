// New keys and values into the 8-bit cache (qm_cache_append).
//
// A block of tokens and a head have one scale, delta = max|x| / qmax over what the block has held; where new tokens raise it, the
// codes that are there already are rounded again under the new one.  One unit of work is a touched block, a head, and keys or values: it
// finds the new tokens' maximum, then writes codes.  Bound by HBM for prompts (the new tokens are read once from there and once
// from L1 or L2; 8 prompts of up to 1000 tokens, 16 heads of 64, 15.6 us), by latency for a token at a time (64 tokens, 8 heads of 128, 2.9 us).
#include "cache_device.cuh"

namespace qm {
namespace {

struct AppendArgs {
  CacheView c;
  const void *k, *v;
  int64_t ld_k, ld_v;              // elements between tokens
};

// The blocks that a sequence's new tokens touch, from `first` on; none if it has no tokens or they have no positions.
struct Touched { int first, n; };
__device__ __forceinline__ Touched touched_by(const CacheView& c, const Extent& e) {
  if (e.n == 0 || e.len == 0) return {0, 0};
  const int first = max(e.len - e.n, 0) >> c.shift;
  return {first, ((e.len - 1) >> c.shift) - first + 1};
}

template <int FMT>
__device__ __noinline__ uint32_t append_far(float x0, float x1, float delta) {
  const Quotient quot(delta);
  return quant2<FMT>(quot(x0), quot(x1));
}
// Two codes under a scale that covers both magnitudes.
template <int FMT>
__device__ __forceinline__ uint32_t append_pair(float x0, float x1, float delta, const QuotientPair& quot) {
  if (QuotientPair::serves(delta)) return quant_pair_x2<FMT>(x0, x1, quot);
  return delta > 0.f && delta < INFINITY ? append_far<FMT>(x0, x1, delta) & 0xffffu : 0u;
}
template <int FMT>
__device__ __forceinline__ uint2 append8(const Vec8& v, float delta, const QuotientPair& quot) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = append_pair<FMT>(v.v[2 * i], v.v[2 * i + 1], delta, quot);
  return make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
}
template <int FMT>
__device__ __forceinline__ uint32_t again4(uint32_t codes, float before, float after, const QuotientPair& quot) {
  uint32_t h[2];
  half4_of<FMT>(codes, h[0], h[1]);
  uint32_t r[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
    r[i] = append_pair<FMT>(f.x * before, f.y * before, after, quot);
  }
  return r[0] | r[1] << 16;
}

// THREADS: to a unit, 32 or 128 (of which a thread block has four, or one).
template <typename T, int FMT, int THREADS>
__global__ void __launch_bounds__(128) cache_append_kernel(const AppendArgs a) {
  pdl_prologue();
  const CacheView& c = a.c;
  const int tid = threadIdx.x % THREADS;
  auto units_of = [&](int b) { return touched_by(c, extent_of(c, b)).n * c.kv_heads; };
  // all sequences' units in one line; without `starts` a sequence has one block, or no position
  const int first = blockIdx.x * (128 / THREADS), unit = first + threadIdx.x / THREADS;
  Place at{unit / c.kv_heads, unit - unit % c.kv_heads, c.kv_heads};
  if (c.starts) {
    at = place_of<128>(c.batch, first, units_of);
    if (at.b < 0) return;
    while (unit >= at.begin + at.n && ++at.b < c.batch) { at.begin += at.n; at.n = units_of(at.b); }
  }
  if (at.b >= c.batch) return;
  const int head = (unit - at.begin) % c.kv_heads, b = at.b;
  const Extent e = extent_of(c, b);
  const Touched touched = touched_by(c, e);
  if (touched.n == 0) return;
  const int block = touched.first + (unit - at.begin) / c.kv_heads;
  const int64_t p0 = max((int64_t)e.len - e.n, (int64_t)0);                  // position of the first new token (those before 0 have none)
  const int64_t from = max(p0, (int64_t)block << c.shift), to = min((int64_t)e.len, ((int64_t)block + 1) << c.shift);
  const int page = page_of(c, b, block);
  if (page < 0) return;
  const int slot = (int)(from & ((1 << c.shift) - 1)), n = (int)(to - from);
  const int64_t token = e.first + (from - ((int64_t)e.len - e.n));

  const bool values = blockIdx.y;
  const T* const x = static_cast<const T*>(values ? a.v : a.k) + token * (values ? a.ld_v : a.ld_k) + (int64_t)head * c.dim;
  const int64_t ld = values ? a.ld_v : a.ld_k;
  const int64_t place = (int64_t)page * c.kv_heads + head;
  uint8_t* const codes = (values ? c.v : c.k) + (place << c.shift) * c.dim;
  float* const delta = (values ? c.dv : c.dk) + place;
  const int per = c.dim / 8, work = n * per;                                 // eight elements at a time

  uint32_t top = 0;
#pragma unroll 4
  for (int i = tid; i < work; i += THREADS) top = absmax8(Loader<T>::load8(x + (int64_t)(i / per) * ld + i % per * 8), top);
  const float before = slot ? *delta : 0.f;
  top = __reduce_max_sync(0xffffffffu, top);
  if (THREADS > 32) {
    __shared__ uint32_t tops[4];
    if ((tid & 31) == 0) tops[tid >> 5] = top;
    __syncthreads();                                                         // (and all have read the old scale)
    top = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
  }
  float after = top >= 0x7f800000u ? __int_as_float(0x7fffffff) : __fdiv_rn(__uint_as_float(top), fmt_qmax(FMT));
  if (after < kLeastScale) after = 0.f;
  after = before > after || before != before ? before : after;
  const QuotientPair quot(after);
  __syncwarp();
  if (tid == 0) *delta = after;
  if (slot && after > before) {
    for (int i = tid; i < slot * c.dim / 16; i += THREADS) {
      uint4 w = reinterpret_cast<uint4*>(codes)[i];
      w.x = again4<FMT>(w.x, before, after, quot); w.y = again4<FMT>(w.y, before, after, quot);
      w.z = again4<FMT>(w.z, before, after, quot); w.w = again4<FMT>(w.w, before, after, quot);
      reinterpret_cast<uint4*>(codes)[i] = w;
    }
  }
#pragma unroll 4
  for (int i = tid; i < work; i += THREADS)
    *reinterpret_cast<uint2*>(codes + (int64_t)slot * c.dim + i * 8) =
        append8<FMT>(Loader<T>::load8(x + (int64_t)(i / per) * ld + i % per * 8), after, quot);
}

template <typename T, int FMT>
qm_status launch_typed(const AppendArgs& a, int64_t units, cudaStream_t s) {
  // a warp where a unit has a token or two, as when one is generated at a time
  if (a.c.tokens <= 2ll * a.c.batch) {
    QM_CUDA_OK(launch_pdl(cache_append_kernel<T, FMT, 32>, dim3((unsigned)((units + 3) / 4), 2), dim3(128), 0, s, a));
  } else {
    QM_CUDA_OK(launch_pdl(cache_append_kernel<T, FMT, 128>, dim3((unsigned)units, 2), dim3(128), 0, s, a));
  }
  count_launch();
  return QM_OK;
}
template <typename T>
qm_status launch_format(const AppendArgs& a, int64_t units, int fmt, cudaStream_t s) {
  return fmt == QM_FMT_INT8 ? launch_typed<T, QM_FMT_INT8>(a, units, s) : fmt == QM_FMT_E4M3 ? launch_typed<T, QM_FMT_E4M3>(a, units, s) : launch_typed<T, QM_FMT_E5M2>(a, units, s);
}

}  // namespace

qm_status launch_cache_append(const CacheArgs& c, const void* k, int64_t ld_k, const void* v, int64_t ld_v, int dtype, cudaStream_t s) {
  AppendArgs a{};
  a.c = view_of(c);
  a.k = k; a.v = v; a.ld_k = ld_k; a.ld_v = ld_v;
  // at most (sequences' rows of the tokens do not overlap): a sequence's tokens touch a block for each block_tokens of them and two more
  const int64_t units = (c.starts ? (c.tokens >> a.c.shift) + 2 * c.batch : c.batch) * c.kv_heads;
  if (units >= (1ll << 31) - 4) return QM_ERR_UNSUPPORTED;
  return dtype == QM_DT_BF16 ? launch_format<__nv_bfloat16>(a, units, c.fmt, s) : launch_format<float>(a, units, c.fmt, s);
}

}  // namespace qm
