// The products of a layer whose codes are INT8 (qm_linear_int8, qm_gated_linear_int8):
//   y_ij = (sum_k x_ik w_jk) dx_i dw_j + bias_j          the sum in int32, exact
//   h_ij = act(g_ij) u_ij, g and u two such products     of the same x
// written in bf16 or fp32.  Two kernels, both on tcgen05.mma kind::i8 with operands staged by TMA in 128-byte-swizzled blocks
// 128 contraction entries deep; a tail of the contraction is what the tensor map fills with zeros.
//   linear_few_kernel   few rows of x.  A CTA takes 128 rows of the WEIGHT as the MMA's M and up to 128 rows of x as its N,
//                       so that a weight row is a lane of tensor memory and an output row is written by consecutive lanes.
//                       The contraction is split over the CTAs of a cluster.
//   linear_many_kernel  CTA pairs (cta_group::2) on tiles of 256 rows of x and 256 weight rows, two accumulator buffers.
// Integer sums are the same in any order, so an output does not depend on the kernel or the split.
//
// Every mbarrier wait is bounded (Waiter): a CTA that gives up leaves NaN in the outputs it cannot compute, waits for what it has
// in flight, frees tensor memory and returns.
#include "linear_shared.cuh"

namespace qm {
namespace {

struct Scales {
  const float* dx;
  const float* dw[2];
  const void* bias; int bias_bf16;
};

__device__ __forceinline__ float ex2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// One product.  The gated kernels are compiled for each activation: chosen in the epilogue's loop it is a branch for every output, under which no
// other output's exponential runs (8192 x 4096 x 1024 54 us instead of 50); chosen ahead of the loop, its three copies do not stay in the
// instruction cache (63 us).
constexpr int kNoAct = -1;

// act(g) in fp32.
//  GELU: g Phi(g), Phi(-|g|) = erfc(z) / 2 with z = |g| / sqrt 2 and erfc(z) = t exp(-z^2 + Q(t)), t = 1 / (1 + 0.39 z).  Q is log(erfc(z)
//    exp(z^2) / t) interpolated at Chebyshev points for z up to 10, degree 8.  To the base 2, with |g| for z.  What is off of |g| Phi(-|g|) is
//    at most 1.2 g^2 + 22 half steps of it (the exponent's roundings grow with g^2; the polynomial's, the fit's, ex2's 4 and the reciprocal's
//    are the 22), next to zero 11 half steps of |g| (4.2 seen).  1/2 g (1 + erff) has 3 there, in more instructions, and loses the
//    negative tail, which this keeps.
//  The others: g / (1 + exp(-t)), t = g or twice the tanh's argument: 1/2 (1 + tanh) is that quotient, and unlike 1 + tanh it keeps
//    its relative precision where g is negative.  1 / (1 + exp(-t)) is s / (s exp(-t) + s) with s = 2^-20, so that the exponential stays
//    inside fp32 and the approximate reciprocal, which gives 0 from 2^126 on, above 0 until g times the quotient is far below
//    fp32's normal numbers (t = -101).  g comes last: scaled by s a small gate would lose its bits.
//    The exponent's rounding and its constant's are |t| half steps of exp or, next to zero, 20: less than a bf16 output shows.  For fp32 outputs
//    the exponent's whole part is taken out exactly: 12 half steps at any g, for 8192 x 4096 x 1024 63 us instead of 59.
//  Two outputs at a time (8192 x 4096 x 1024 to bf16, SiLU 50.4 -> 49.4 us, GELU 58.5 -> 54.7, its tanh form 52.7 -> 50.7).
template <typename T, int ACT>
__device__ __forceinline__ void activate(float& g0, float& g1) {
  const uint64_t g = pair_of(g0, g1);
  if (ACT == QM_ACT_GELU) {
    const uint64_t t = pair_of(rcp_approx(fmaf(0.27577165f, fabsf(g0), 1.f)), rcp_approx(fmaf(0.27577165f, fabsf(g1), 1.f)));
    constexpr float kQ[] = {1.5611439f, -2.708909f, 2.1119456f, -1.0494819f, 0.6094263f, 0.5445073f, 1.4499226f, -2.1845343f};
    uint64_t q = both(-0.33402064f);
#pragma unroll
    for (int i = 0; i < 8; ++i) q = fma2(q, t, both(kQ[i]));
    float x0, x1, tail0, tail1;
    halves(fma2(mul2(g, g), both(-0.72134752f), q), x0, x1);
    halves(mul2(mul2(both(0.5f), g), mul2(t, pair_of(ex2_approx(x0), ex2_approx(x1)))), tail0, tail1);
    // (of an infinite gate the tail is Inf times 0; fmaxf makes 0 of a NaN)
    g0 = g0 < 0.f ? tail0 : g0 - fmaxf(tail0, 0.f);
    g1 = g1 < 0.f ? tail1 : g1 - fmaxf(tail1, 0.f);
    return;
  }
  constexpr float kS = 9.5367432e-7f;
  uint64_t t = g, e;
  if (ACT == QM_ACT_GELU_TANH) t = mul2(both(1.5957691f), fma2(mul2(mul2(both(0.044715f), g), g), g, g));
  float x0, x1;
  if (sizeof(T) == 4) {
    // s exp(-t) = 2^(n - 20) 2^r; beyond the limits it is nothing next to s, or the quotient nothing
    halves(t, x0, x1);
    const uint64_t u = pair_of(fmaxf(fminf(x0, 73.f), -102.f), fmaxf(fminf(x1, 73.f), -102.f));
    const uint64_t z = fma2(both(-1.442695f), u, both(12582912.f)), n = fma2(both(-1.f), z, both(12582912.f));   // n: -round(..)
    halves(fma2(both(-1.925963e-8f), u, fma2(both(-1.442695f), u, n)), x0, x1);
    const uint32_t z0 = (uint32_t)z, z1 = (uint32_t)(z >> 32);
    e = mul2(pair_of(ex2_approx(x0), ex2_approx(x1)), pair_of(__uint_as_float((z0 << 23) + (107u << 23)), __uint_as_float((z1 << 23) + (107u << 23))));
  } else {
    halves(fma2(both(-1.442695f), t, both(-20.f)), x0, x1);
    e = pair_of(ex2_approx(x0), ex2_approx(x1));
  }
  halves(add2(e, both(kS)), x0, x1);
  halves(mul2(g, mul2(both(kS), pair_of(rcp_approx(x0), rcp_approx(x1)))), g0, g1);
}

// An output of its sum, the same roundings in every epilogue (said here, so that the compiler makes the same instructions of it everywhere;
// with the sum as the first factor it gives one of the kernels 72 registers instead of 80, and 512 x 4096 x 1024 takes 6.5 us instead of 5.6).
__device__ __forceinline__ float output_of(uint32_t sum, float dx, float dw, float bias) { return fmaf(dx * dw, (float)(int)sum, bias); }
__device__ __forceinline__ float output_of(uint32_t sum, float dx, float dw) { return dx * dw * (float)(int)sum; }

__device__ __forceinline__ float load_bias(const Scales& s, int64_t n) {
  if (!s.bias) return 0.f;
  return s.bias_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(s.bias)[n]) : static_cast<const float*>(s.bias)[n];
}

// ------------------------------------------------------------------ few rows
// One tile of 128 weight rows x nt rows of x per CTA, or per cluster that splits the contraction.  Roles: warp 0 issues TMA loads into a
// ring, warp 1 holds tensor memory and issues the MMAs (weights as M, x as N), warps 2..9 are the epilogue.
// 128 contraction entries take a CTA 200 ns with 16 rows of x (18 KB) and 225 with 128 (32 KB): the round from a full block over four MMAs to
// its commit, more than the bytes from L2.  Weights that come from HBM bound by that: 64 x 8192 x 8192 streams its 67 MB in 9.2 of
// 13.9 us with three sets of weights in turn, part of which L2 still holds (hence more than a copy's rate), and takes 14.5 with 470 MB
// of sets.  All other times here are with weights in L2 as far as they fit; from HBM, 1 row of 4096 x 1024 takes 3.8 us instead of
// 2.8, of 4096 x 4096 5.5 instead of 4.3.  The rest, and most of a small
// call (1 x 4096 x 1024 3.1 us): 0.5 to 1.5 us to the first block, 0.2 from the last block to complete accumulators, 0.6 to hand the
// sums over, 0.4 for the cluster's barrier, 0.2 to 0.8 to finish the rows, 0.3 for the next kernel to start.  Tried: sums read
// from the peers instead of pushed (+0.7 us), the barrier of the next block asked ahead of this block's MMAs (no
// difference), half the ring and two CTAs to an SM for long parts (64 x 8192 x 8192 23 us: CTAs of one launch share SMs while others idle).
struct FewArgs {
  int64_t M, N;
  int num_kb, tiles_m, split, nt, stages;    // nt: rows of x per tile, 16 .. 128
  uint32_t sums_bytes;
  int prefetch;                              // weight blocks asked into L2 ahead of the kernel before this one
  int own_log2;                              // of a split contraction, rows of x that a CTA of the cluster finishes
  uint32_t idesc, tmem_cols;
  Scales sc;
  Waits waits;
  void* out; int64_t ld;
  int vec;                                   // four outputs at a multiple of four start on as many bytes
};
constexpr int kFewStages = 12;
constexpr int kMaxSplit = 8;
struct SharedFew {
  uint64_t full[kFewStages], empty[kFewStages], done, drain, read;
  uint32_t tmem_base, abort_flag, gave_up, pad;        // gave_up: some CTA of the cluster did
  float dx[256];
};

__device__ __forceinline__ void add4(int4& a, const int4& b) { a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w; }

template <typename T, int ACT>
__global__ void __launch_bounds__(kThreads, 2)
linear_few_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                  const __grid_constant__ CUtensorMap map_u, const FewArgs a) {
  constexpr bool GATED = ACT != kNoAct;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  constexpr int kW = GATED ? 2 : 1;
  const uint32_t stage_bytes = kW * kBlockBytes + (uint32_t)a.nt * kBlock;
  // behind the ring: of a split contraction the parts' sums of this CTA's rows, [part][product][row][weight row]
  int* const sums = reinterpret_cast<int*>(tiles + (size_t)a.stages * stage_bytes);
  SharedFew* sh = reinterpret_cast<SharedFew*>(reinterpret_cast<uint8_t*>(sums) + a.sums_bytes);
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const int tile = (int)blockIdx.x / a.split, part = (int)blockIdx.x - tile * a.split;
  const int n0 = tile / a.tiles_m * kBlock, m0 = tile % a.tiles_m * a.nt;
  const int kb0 = (int)((int64_t)a.num_kb * part / a.split), kb1 = (int)((int64_t)a.num_kb * (part + 1) / a.split);
  const Waiter w{&sh->abort_flag, nullptr, a.waits.limit_ns};

  if (warp == 0 && lane < 2 + (int)GATED) {
    const CUtensorMap* maps[3] = {&map_x, &map_w, &map_u};
    asm volatile("prefetch.tensormap [%0];" ::"l"(maps[lane]) : "memory");
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < a.stages; ++s) {
      mbar_init(smem_u32(&sh->full[s]), 1);
      mbar_init(smem_u32(&sh->empty[s]), 1);
    }
    mbar_init(smem_u32(&sh->done), 1);
    mbar_init(smem_u32(&sh->drain), 1);
    mbar_init(smem_u32(&sh->read), kEpiWarps);
    sh->abort_flag = 0; sh->gave_up = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  // Tensor memory is waited for where CTAs of other kernels on this SM hold it, and a CTA that holds some must not wait for one that waits
  // for some: a CTA tells its peers ahead of its allocation that its shared memory may be written, and gives its columns back ahead of
  // its wait for their sums.
  if (a.split > 1) cluster_arrive();
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem_base)), "r"(a.tmem_cols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  // The next kernel in the stream is let in when this one's loads are all on their way, so that its set-up runs under the epilogue here.
  // What it may do ahead of its wait is a prefetch into L2, which a later write cannot make stale: of large weights the first blocks.
  if (a.prefetch && warp == 0 && lane == 0)
    for (int k = 0; k < a.prefetch && kb0 + k < kb1; ++k) {
      prefetch_2d(&map_w, (kb0 + k) * kBlock, n0);
      if (GATED) prefetch_2d(&map_u, (kb0 + k) * kBlock, n0);
    }
  pdl_wait();
  tc_fence_after();
  const uint32_t tmem_base = sh->tmem_base;

  uint32_t loads = 0;
  if (warp == 0) {
    if (lane == 0) {
      uint32_t g = 0;
      int s = 0;
      uint32_t parity = 0;
      for (int kb = kb0; kb < kb1; ++kb, ++g) {
        if (g >= a.waits.stop_after) break;
        if (g >= (uint32_t)a.stages && !w.wait(smem_u32(&sh->empty[s]), parity ^ 1u)) break;
        const uint32_t bar = smem_u32(&sh->full[s]), base = smem_u32(tiles) + (uint32_t)s * stage_bytes;
        mbar_expect_tx(bar, stage_bytes);
        tma_load_2d_local(base, &map_w, bar, kb * kBlock, n0);
        if (GATED) tma_load_2d_local(base + kBlockBytes, &map_u, bar, kb * kBlock, n0);
        tma_load_2d_local(base + kW * kBlockBytes, &map_x, bar, kb * kBlock, m0);
        if (++s == a.stages) { s = 0; parity ^= 1u; }
      }
      pdl_launch_dependents();
      loads = g;
    }
    if (a.split > 1) { cluster_wait(); cluster_arrive(); }
  } else if (warp == 1) {
    const bool lead = elect_one();
    int s = 0;
    uint32_t parity = 0;
    bool ok = true;
    for (int kb = kb0; kb < kb1; ++kb) {
      if (!w.wait_warp(smem_u32(&sh->full[s]), parity)) { ok = false; break; }
      tc_fence_after();
      const uint32_t base = smem_u32(tiles) + (uint32_t)s * stage_bytes;
      const uint64_t dx = smem_desc(base + kW * kBlockBytes, 128);
      if (lead) {
#pragma unroll
        for (int p = 0; p < kW; ++p)
#pragma unroll
          for (int k = 0; k < 4; ++k)             // 32 codes per instruction
            mma_i8_one(tmem_base + (uint32_t)(p * a.nt), smem_desc(base + p * kBlockBytes, 128) + 2 * k, dx + 2 * k, a.idesc,
                       k ? 1u : (uint32_t)(kb > kb0));
        tc_commit_one(smem_u32(&sh->empty[s]));
      }
      if (++s == a.stages) { s = 0; parity ^= 1u; }
    }
    if (ok && lead) tc_commit_one(smem_u32(&sh->done));
    // the columns back when the epilogue has read them (or given up), ahead of the wait for the peers' sums
    if (a.split > 1) { cluster_wait(); cluster_arrive(); }
    wait_limited(smem_u32(&sh->read), 0, a.waits.limit_ns);
    // give-up path: MMAs that nobody has waited for.  The loading warp may flag the CTA at this moment: one decision for the warp
    if (__any_sync(0xffffffffu, *w.abort_flag)) {
      if (lead) tc_commit_one(smem_u32(&sh->drain));
      wait_limited(smem_u32(&sh->drain), 0, a.waits.limit_ns);
    }
    __syncwarp();
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(a.tmem_cols) : "memory");
  }

  // epilogue, warps 2..9: a warp may read the quarter warp % 4 of tensor memory's lanes; the two warps of a quarter take every
  // other chunk of 16 columns (rows of x).  Scales and biases are fetched ahead of the waits.
  const int et = (int)threadIdx.x - 64, q = warp & 3, h = (warp - 2) >> 2;
  const int live = (int)(a.M - m0 < a.nt ? a.M - m0 : a.nt);                 // rows of x in this tile
  // of a split contraction a CTA finishes `own` rows of x, a thread four neighbouring weight rows at a time
  const int own = 1 << a.own_log2;
  const int j = a.split == 1 ? q * 32 + lane : 4 * (et & (kBlock / 4 - 1));
  T* const out = static_cast<T*>(a.out);
  float dw[4], du[4], bias[4];
  if (warp >= 2) {
    if (et < live) sh->dx[et] = a.sc.dx[m0 + et];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int64_t n = (int64_t)n0 + j + k;
      const bool in = n < a.N && (k == 0 || a.split > 1);
      dw[k] = in ? a.sc.dw[0][n] : 0.f;
      du[k] = GATED && in ? a.sc.dw[1][n] : 0.f;
      bias[k] = !GATED && in ? load_bias(a.sc, n) : 0.f;
    }
    const bool ok = w.wait_warp(smem_u32(&sh->done), 0);
    tc_fence_after();
    asm volatile("bar.sync 1, 256;" ::: "memory");                            // dx is there, and every warp has waited
    const uint32_t lane_addr = tmem_base + ((uint32_t)(q * 32) << 16);
    if (a.split == 1) {
      const int64_t n = (int64_t)n0 + j;
      for (int c = h * 16; c < live; c += 32) {
        uint32_t r[16], u[16];
        if (ok) {
          tmem_ld16(lane_addr + c, r);
          if (GATED) tmem_ld16(lane_addr + a.nt + c, u);
          tmem_ld_wait();
        }
        float y[16], up[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float dxv = sh->dx[c + i];                                    // (rows beyond the last: not stored)
          y[i] = GATED ? output_of(r[i], dxv, dw[0]) : output_of(r[i], dxv, dw[0], bias[0]);
          if (GATED) up[i] = output_of(u[i], dxv, du[0]);
        }
        if (GATED)
#pragma unroll
          for (int i = 0; i < 16; i += 2) {
            activate<T, ACT>(y[i], y[i + 1]);
            y[i] *= up[i]; y[i + 1] *= up[i + 1];
          }
        T* p = out + (int64_t)(m0 + c) * a.ld + n;
#pragma unroll
        for (int i = 0; i < 16; ++i, p += a.ld)
          if (n < a.N && c + i < live) *p = (T)(ok ? y[i] : nan_f());
      }
    } else {
      // this part's sums to the CTAs that finish their rows: stores to another SM's shared memory are not waited for one by one,
      // as reads are (1 row of 4096 weight rows 0.7 us, 64 rows 1.4)
      cluster_wait();
      if (!ok && lane < a.split) sts_cluster(map_to_cta(smem_u32(&sh->gave_up), lane), 1u);
      for (int c = h * 16; ok && c < live; c += 32) {
#pragma unroll
        for (int p = 0; p < kW; ++p) {
          uint32_t r[16];
          tmem_ld16(lane_addr + p * a.nt + c, r);
          tmem_ld_wait();
          const uint32_t at = smem_u32(sums + (part * kW + p) * own * kBlock + q * 32 + lane);
          if (own >= 16) {                                                    // one CTA's rows, from c & (own - 1) on
            const uint32_t to = map_to_cta(at, c >> a.own_log2) + (uint32_t)((c & (own - 1)) * kBlock * 4);
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (c + i < live) sts_cluster(to + i * kBlock * 4, r[i]);
          } else {
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (c + i < live) sts_cluster(map_to_cta(at, (c + i) >> a.own_log2) + (uint32_t)((i & (own - 1)) * kBlock * 4), r[i]);
          }
        }
      }
    }
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&sh->read));
    if (a.split > 1) cluster_arrive();
  }
  if (a.split > 1) {
    cluster_wait();
    const int cols = (int)(a.N - n0 - j < 4 ? a.N - n0 - j : 4);
    if (warp >= 2 && cols > 0) {
      const bool ok = sh->gave_up == 0;
      const int rows = min(own, live - part * own);
      for (int i = et / (kBlock / 4); i < rows; i += 256 / (kBlock / 4)) {
        int4 g = make_int4(0, 0, 0, 0), u = g;
        const int4* from = reinterpret_cast<const int4*>(sums + i * kBlock + j);
        const int next = kW * own * (kBlock / 4);                             // from a part to the one behind it
#pragma unroll 2
        for (int p = 0; p < a.split; ++p, from += next) {
          add4(g, *from);
          if (GATED) add4(u, from[own * (kBlock / 4)]);
        }
        const int row = part * own + i;
        const float dxv = sh->dx[row];
        const int gs[4] = {g.x, g.y, g.z, g.w}, us[4] = {u.x, u.y, u.z, u.w};
        float y[4], up[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          y[k] = GATED ? output_of(gs[k], dxv, dw[k]) : output_of(gs[k], dxv, dw[k], bias[k]);
          if (GATED) up[k] = output_of(us[k], dxv, du[k]);
        }
        if (GATED)
#pragma unroll
          for (int k = 0; k < 4; k += 2) {
            activate<T, ACT>(y[k], y[k + 1]);
            y[k] *= up[k]; y[k + 1] *= up[k + 1];
          }
#pragma unroll
        for (int k = 0; k < 4; ++k) if (!ok) y[k] = nan_f();
        store4(out + (int64_t)(m0 + row) * a.ld + n0 + j, y, cols, a.vec);
      }
    }
  }
  __syncthreads();
  if (sh->abort_flag && threadIdx.x == 0) {        // give-up path: loads that nobody has waited for
    const uint32_t st = (uint32_t)a.stages;
    for (uint32_t g = loads > st ? loads - st : 0u; g < loads; ++g) wait_limited(smem_u32(&sh->full[g % st]), (g / st) & 1, a.waits.limit_ns);
  }
}

// ------------------------------------------------------------------ many rows
// Persistent CTA pairs on tiles of 256 rows of x and 256 weight rows (gated: 128 rows of either weight), a stage of 32 KB a CTA for 128
// contraction entries, five stages, two accumulator buffers, so that a tile's epilogue runs under the next one's MMAs.
// Bound by the tensor cores from contractions of 2048 on (8192 x 8192 x 4096 167 us, 3.3 POP/s; 531 cycles for 128 entries, 512 at the
// pipe's peak), below that by the output: 16384 x 4096 x 1024 takes 54 us, 44 without its stores, and 35 with a contraction
// of 128, which is what a fill of those 134 MB takes (34.8).  Bulk stores of the staged rows and plain ones measured the same; four stages
// 59, cache hints on the stores 53 to 54.  To fp32 the same product takes 69.5 us (268 MB of output); rows off 16 bytes go out 2 or 4 bytes a
// lane, one buffer at a time: 6000 x 2603 x 400 35 us.  The gated form's epilogue alone (contraction of 128) is 37 us for 8192 x 4096 outputs, half
// of it the activation, under 44 of MMAs.
struct ManyArgs {
  int64_t M, N;
  int num_kb, tiles_n, num_tiles;              // tiles of 256 rows of x and 256 weight rows (gated: 128 of each weight)
  Scales sc;
  Waits waits;
  void* out; int64_t ld;
  int vec;                                     // rows of the output start on 16 bytes
};
constexpr int kManyStages = 5;
constexpr uint32_t kManyStageBytes = 2 * kBlockBytes;
constexpr uint32_t kOutBytes = 32 * 128;       // of output on its way per epilogue warp: 32 rows of 128 bytes
struct SharedMany {
  uint64_t full[kManyStages], empty[kManyStages], tmem_full[2], tmem_empty[2], drain;
  uint32_t tmem_base, abort_flag, issued, peer_gave_up, peer_issued, pad[3];
  alignas(16) float dw[2][256], bias[2][256];
};

// 16 lanes x 32 columns of tensor memory: thread t gets, of every 8 columns i, columns 2 (t % 4) and one more in lanes t / 4 (words 4 i,
// 4 i + 1) and t / 4 + 8 (4 i + 2, 4 i + 3).
__device__ __forceinline__ void tmem_ld_16x32(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]),
        "=r"(r[15])
      : "r"(taddr)
      : "memory");
}

// 16 rows (from `row`) x 32 columns (from `col`) of output in that layout to the warp's staging buffer: rows of 128 bytes, 16-byte
// units permuted with the row.
__device__ __forceinline__ void stage_16x32(uint32_t stage, int lane, int row, int col, const float (&y)[16], float) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
      const int r = row + 8 * hh + (lane >> 2), unit = col / 4 + 2 * i + ((lane >> 1) & 1);
      asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(stage + r * 128 + ((unit ^ (r & 7)) << 4) + (lane & 1) * 8),
                   "f"(y[4 * i + 2 * hh]), "f"(y[4 * i + 2 * hh + 1]) : "memory");
    }
}
__device__ __forceinline__ void stage_16x32(uint32_t stage, int lane, int row, int col, const float (&y)[16], __nv_bfloat16) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    uint32_t w[4];                                          // two 8-column groups, the upper and lower 8 rows of each
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const int k = 4 * (2 * j + (m >> 1)) + 2 * (m & 1);
      const __nv_bfloat162 v = __floats2bfloat162_rn(y[k], y[k + 1]);
      w[m] = *reinterpret_cast<const uint32_t*>(&v);
    }
    const int m = lane >> 3, r = row + 8 * (m & 1) + (lane & 7), unit = col / 8 + 2 * j + (m >> 1);
    asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(stage + r * 128 + ((unit ^ (r & 7)) << 4)),
                 "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
  }
}

template <typename T, int ACT>
__global__ void __launch_bounds__(kThreads, 1)
linear_many_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
                   const __grid_constant__ CUtensorMap map_u, const __grid_constant__ CUtensorMap map_out, const ManyArgs a) {
  constexpr bool GATED = ACT != kNoAct;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* const staging = tiles + (size_t)kManyStages * kManyStageBytes;
  SharedMany* sh = reinterpret_cast<SharedMany*>(staging + kEpiWarps * kOutBytes);
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1, num_pairs = gridDim.x >> 1;
  const Waiter w{&sh->abort_flag, nullptr, a.waits.limit_ns};
  constexpr int kTileN = GATED ? 128 : 256;                                   // output columns of a tile

  if (warp == 0 && lane < 4) {
    const CUtensorMap* maps[4] = {&map_x, &map_w, &map_u, &map_out};
    asm volatile("prefetch.tensormap [%0];" ::"l"(maps[lane]) : "memory");
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < kManyStages; ++s) {
      mbar_init(smem_u32(&sh->full[s]), 1);
      mbar_init(smem_u32(&sh->empty[s]), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(smem_u32(&sh->tmem_full[b]), 1);
      mbar_init(smem_u32(&sh->tmem_empty[b]), 2 * kEpiWarps);
    }
    mbar_init(smem_u32(&sh->drain), 1);
    sh->abort_flag = 0; sh->issued = 0; sh->peer_gave_up = 0; sh->peer_issued = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem_base)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  pdl_prologue();
  tc_fence_after();
  const uint32_t tmem_base = sh->tmem_base;

  if (warp == 0) {
    // TMA producer (both CTAs): this CTA's 128 rows of x, and its half of the MMA's N: the tile's weight rows, or of the gated
    // form the gate's rows in the leader and up's in its peer, so that accumulator columns j and 128 + j are output column j's
    if (lane == 0) {
      const CUtensorMap* const mw = GATED && rank ? &map_u : &map_w;
      uint32_t g = 0;
      int s = 0;
      uint32_t parity = 0;
      bool ok = true;
      for (int t = pair; t < a.num_tiles && ok; t += num_pairs) {
        const int tm = t / a.tiles_n;
        const int r0 = tm * 256 + (int)rank * kBlock, c0 = (t - tm * a.tiles_n) * kTileN + (GATED ? 0 : (int)rank * kBlock);
        for (int kb = 0; kb < a.num_kb; ++kb, ++g) {
          if (g >= a.waits.stop_after || (g >= (uint32_t)kManyStages && !w.wait(smem_u32(&sh->empty[s]), parity ^ 1u))) { ok = false; break; }
          if (rank == 0) mbar_expect_tx(smem_u32(&sh->full[s]), 2 * kManyStageBytes);
          const uint32_t bar = map_to_cta(smem_u32(&sh->full[s]), 0), base = smem_u32(tiles) + (uint32_t)s * kManyStageBytes;
          tma_load_2d(base, &map_x, bar, kb * kBlock, r0);
          tma_load_2d(base + kBlockBytes, mw, bar, kb * kBlock, c0);
          if (++s == kManyStages) { s = 0; parity ^= 1u; }
        }
      }
      sh->issued = g;
    }
  } else if (warp == 1) {
    if (rank == 0) {
      const bool lead = elect_one();
      constexpr uint32_t idesc = make_idesc(2, 1, 1, 256, 256);               // s8 x s8 -> s32
      uint32_t it = 0;
      int s = 0;
      uint32_t parity = 0;
      bool ok = true;
      for (int t = pair; t < a.num_tiles && ok; t += num_pairs, ++it) {
        const uint32_t buf = it & 1;
        if (it >= 2 && !w.wait_warp(smem_u32(&sh->tmem_empty[buf]), ((it >> 1) - 1) & 1)) break;
        tc_fence_after();
        for (int kb = 0; kb < a.num_kb; ++kb) {
          if (!w.wait_warp(smem_u32(&sh->full[s]), parity)) { ok = false; break; }
          tc_fence_after();
          const uint32_t base = smem_u32(tiles) + (uint32_t)s * kManyStageBytes;
          const uint64_t da = smem_desc(base, 128), db = smem_desc(base + kBlockBytes, 128);
          if (lead) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              mma_pair<kKindI8>(tmem_base + buf * 256, da + 2 * k, db + 2 * k, idesc, k ? 1u : (uint32_t)(kb > 0), true);
            tc_commit_pair(smem_u32(&sh->empty[s]), true);
          }
          if (++s == kManyStages) { s = 0; parity ^= 1u; }
        }
        if (ok) tc_commit_pair(smem_u32(&sh->tmem_full[buf]), lead);
      }
    }
  } else {
    // epilogue, warps 2..9 of both CTAs; the two warps of a lane quarter (32 rows of x) take half of the columns each
    const int q = warp & 3, h = (warp - 2) >> 2, et = (int)threadIdx.x - 64;
    uint4* const stage = reinterpret_cast<uint4*>(staging + (warp - 2) * kOutBytes);
    T* const out = static_cast<T*>(a.out);
    constexpr int kChunk = 128 / sizeof(T);
    const bool has_bias = a.sc.bias != nullptr;
    bool ok = true;
    uint32_t it = 0;
    // A tile's scales are fetched while the tile before it is written (fetched when they are needed they are 2000 of 6300 cycles a
    // tile): by column of the accumulators (gated: gate's, then up's) one a thread, and those of rows lane / 4, + 8, + 16, + 24.
    float next_dw = 0.f, next_bias = 0.f, next_dx[4] = {};
    auto fetch = [&](int t) {
      if (t >= a.num_tiles) return;
      const int tm = t / a.tiles_n;
      const int64_t col = (int64_t)(t - tm * a.tiles_n) * kTileN + (GATED ? et & 127 : et);
      const bool in = col < a.N;
      next_dw = !in ? 0.f : GATED && et >= 128 ? a.sc.dw[1][col] : a.sc.dw[0][col];
      if (!GATED && has_bias) next_bias = in ? load_bias(a.sc, col) : 0.f;
      const int64_t row = (int64_t)tm * 256 + rank * kBlock + q * 32 + (lane >> 2);
#pragma unroll
      for (int k = 0; k < 4; ++k) next_dx[k] = row + 8 * k < a.M ? a.sc.dx[row + 8 * k] : 0.f;
    };
    fetch(pair);
    for (int t = pair; t < a.num_tiles; t += num_pairs, ++it) {
      const int tm = t / a.tiles_n;
      const uint32_t buf = it & 1;
      const int64_t c0 = (int64_t)(t - tm * a.tiles_n) * kTileN;
      sh->dw[buf][et] = next_dw;
      if (!GATED) sh->bias[buf][et] = next_bias;
      const float dx[4] = {next_dx[0], next_dx[1], next_dx[2], next_dx[3]};
      fetch(t + num_pairs);
      const int64_t row0 = (int64_t)tm * 256 + rank * kBlock + q * 32;
      const int rows = (int)(a.M - row0 < 32 ? a.M - row0 : 32);             // <= 0: none
      ok = ok && w.wait_warp(smem_u32(&sh->tmem_full[buf]), (it >> 1) & 1);
      asm volatile("bar.sync 1, 256;" ::: "memory");                          // publishes the scales
      tc_fence_after();
      const uint32_t acc = tmem_base + ((uint32_t)(q * 32) << 16) + buf * 256;
#pragma unroll 1
      for (int c = h * (kTileN / 2); c < (h + 1) * (kTileN / 2); c += kChunk) {
        if (c0 + c >= a.N) break;                                             // uniform across the warp
        const int cols = (int)(a.N - c0 - c < kChunk ? a.N - c0 - c : kChunk);
        if (a.vec) {                                                          // the last copy has read the buffer
          if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
          __syncwarp();
        }
#pragma unroll
        for (int part = 0; part < kChunk; part += 32) {
          uint32_t r[2][16], u[2][16];
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            tmem_ld_16x32(acc + (uint32_t)(hf * 16 << 16) + c + part, r[hf]);
            if (GATED) tmem_ld_16x32(acc + (uint32_t)(hf * 16 << 16) + 128 + c + part, u[hf]);
          }
          // a thread has eight columns of four rows: eight scales to load, where a row to a thread takes 32 and the epilogue the
          // shared memory's bandwidth from the MMAs (16384 x 4096 x 1024 61 us so)
          float2 d[4], e[4], b[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int k = c + part + 8 * i + 2 * (lane & 3);
            d[i] = *reinterpret_cast<const float2*>(&sh->dw[buf][k]);
            if (GATED) e[i] = *reinterpret_cast<const float2*>(&sh->dw[buf][128 + k]);
            b[i] = !GATED && has_bias ? *reinterpret_cast<const float2*>(&sh->bias[buf][k]) : make_float2(0.f, 0.f);
          }
          tmem_ld_wait();
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            float y[16], up[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              const int i = k >> 2;
              const float dxv = dx[2 * hf + ((k >> 1) & 1)], dwv = k & 1 ? d[i].y : d[i].x;
              y[k] = GATED ? output_of(r[hf][k], dxv, dwv) : output_of(r[hf][k], dxv, dwv, k & 1 ? b[i].y : b[i].x);
              if (GATED) up[k] = output_of(u[hf][k], dxv, k & 1 ? e[i].y : e[i].x);
            }
            if (GATED)
#pragma unroll
              for (int k = 0; k < 16; k += 2) {
                activate<T, ACT>(y[k], y[k + 1]);
                y[k] *= up[k]; y[k + 1] *= up[k + 1];
              }
#pragma unroll
            for (int k = 0; k < 16; ++k) if (!ok) y[k] = nan_f();
            stage_16x32(smem_u32(stage), lane, 16 * hf, part, y, T());
          }
        }
        if (a.vec) {
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) {
            if (rows > 0) tma_store_2d(&map_out, smem_u32(stage), (int)c0 + c, (int)row0);      // clipped to M x N
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
          }
        } else {
          __syncwarp();
          T* const to = out + row0 * a.ld + c0 + c;
          if (sizeof(T) == 2 && ((reinterpret_cast<uintptr_t>(to) & 3) | (a.ld & 1)) == 0) {
            store_rows(stage, lane, reinterpret_cast<uint32_t*>(to), a.ld >> 1, rows, cols >> 1);
            if ((cols & 1) && lane < rows) to[lane * a.ld + cols - 1] = reinterpret_cast<const T*>(stage)[lane * kChunk + (((cols - 1) / 8) ^ (lane & 7)) * 8 + (cols - 1) % 8];
          } else {
            store_rows(stage, lane, to, a.ld, rows, cols);
          }
          __syncwarp();
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0 && ok) mbar_arrive_cluster(map_to_cta(smem_u32(&sh->tmem_empty[buf]), 0));      // (as in linear_fp8_many: no arrival for what was not read)
    }
    if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  }

  tc_fence_before();
  __syncthreads();
  // Neither CTA loads from here on.  They go through the give-up path together, if either has given up.
  if (threadIdx.x == 0) {
    if (rank == 1) sts_cluster(map_to_cta(smem_u32(&sh->peer_issued), 0), sh->issued);
    if (sh->abort_flag) sts_cluster(map_to_cta(smem_u32(&sh->peer_gave_up), rank ^ 1u), 1u);
  }
  cluster_sync();
  if (sh->abort_flag | sh->peer_gave_up) {
    // loads (both CTAs' complete on the leader's barriers) and MMAs that nobody has waited for.  A commit that came as the leader gave up may
    // have let the peer load further: bytes that the leader has yet to expect
    if (threadIdx.x == 0 && rank == 0) {
      const uint32_t n = sh->issued, most = max(n, sh->peer_issued);
      for (uint32_t g = n; g < most; ++g) mbar_expect_tx(smem_u32(&sh->full[g % kManyStages]), kManyStageBytes);
      for (uint32_t g = most > (uint32_t)kManyStages ? most - kManyStages : 0u; g < most; ++g)
        wait_limited(smem_u32(&sh->full[g % kManyStages]), (g / kManyStages) & 1, a.waits.limit_ns);
    }
    if (warp == 1 && rank == 0) {
      if (elect_one())
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(&sh->drain)) : "memory");
      wait_limited(smem_u32(&sh->drain), 0, a.waits.limit_ns);
    }
    cluster_sync();
  }
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
  }
}

// ------------------------------------------------------------------ host side
bool rows_on_16(const LinearArgs& l) {
  return (reinterpret_cast<uintptr_t>(l.out) & 15) == 0 && l.ld_out * (l.out_dtype == QM_DT_BF16 ? 2 : 4) % 16 == 0;
}

Scales scales_of(const LinearArgs& l) {
  return {l.dx, {l.dw[0], l.dw[1]}, l.bias, l.bias_dtype == QM_DT_BF16};
}

// Which kernel, and how the few rows' one is cut, by the time that it takes: rows of x per tile (nt), parts of the contraction (split),
// in ns by what was measured on 148 SMs at 1 to 1024 rows, 1024 to 8192 weight rows and contractions of 1024 to 8192:
//   a CTA of the few rows' kernel: kBase, kDepth for each 128 contraction entries (the MMA warp's round, so that more
//   rows cost little), kSplit where sums are exchanged; as often as the CTAs, one to an SM, fill the GPU;
//   the many rows' kernel: 5000, and for each round of its tiles 310 for 128 contraction entries or the epilogue's 2500, where the output's
//   rows do not start on 16 bytes 5000 in bf16, 6000 in fp32 and 3600 of the gated form's narrower tiles.
// Those times are with weights in L2; there is no term for HBM, so that calls that read 60 MB of weights take 3 to 5 us more than it says,
// whichever cut they get.
// What it settles (us, product of 4096 x 4096 weights): 64 rows (nt 64, split 4) 6.0, (64, 2) 7.0, (64, 1) 9.3, many 13.2; 256 rows (64, 1) 9.9,
// which it takes, (128, 2) 9.6, (128, 1) 10.5, (64, 2) 15.4, many 13.7; 1024 rows many 15.0, (128, 1) 21.8.
struct Plan { int nt, split; };            // nt 0: the many rows' kernel
Plan make_plan(const LinearArgs& l, bool gated, bool aligned) {
  static constexpr int kNt[4] = {16, 32, 64, 128};
  static constexpr int64_t kBase[2][4] = {{2200, 2500, 3100, 4100}, {2300, 2800, 3700, 5200}};
  static constexpr int64_t kDepth[2][4] = {{200, 200, 205, 225}, {300, 310, 330, 390}};
  static constexpr int64_t kSplit[2][4] = {{600, 800, 1100, 2200}, {800, 1000, 1700, 6000}};
  const int64_t sms = sm_count(), num_kb = (l.K + kBlock - 1) / kBlock, tiles_n = (l.N + kBlock - 1) / kBlock;
  const int64_t pairs = sms / 2, tiles = (l.M + 255) / 256 * ((l.N + (gated ? 127 : 255)) / (gated ? 128 : 256));
  int64_t best = 5000 + (tiles + pairs - 1) / pairs * std::max<int64_t>(310 * num_kb, aligned ? 2500 : gated ? 3600 : l.out_dtype == QM_DT_BF16 ? 5000 : 6000);
  Plan plan{0, 1};
  for (int i = 0; i < 4 && (i == 0 || kNt[i - 1] < l.M); ++i) {
    const int64_t ctas = tiles_n * ((l.M + kNt[i] - 1) / kNt[i]);
    if (ctas > 64 * sms) continue;
    // (a cluster lies inside one of the GPU's eight groups of SMs, so not every SM is in one of four or eight)
    for (int split = 1; split <= kMaxSplit && split <= num_kb && (split == 1 || ctas * split <= sms - 4 * split); split *= 2) {
      const int64_t one = kBase[gated][i] + (num_kb + split - 1) / split * kDepth[gated][i] + (split > 1 ? kSplit[gated][i] + 50 * split : 0);
      const int64_t t = 900 + (ctas * split + sms - 1) / sms * (one - 900);
      if (t < best) { best = t; plan = {kNt[i], split}; }
    }
  }
  return plan;
}

constexpr size_t kFewRing = 200 * 1024;
constexpr size_t kFewSmem = 1024 + kFewRing + sizeof(SharedFew);

template <typename T, int ACT>
qm_status launch_few(const LinearArgs& l, const Plan& plan, cudaStream_t s) {
  constexpr bool GATED = ACT != kNoAct;
  static std::atomic<bool> ready[kMaxDevices];
  FewArgs a{};
  a.M = l.M; a.N = l.N;
  a.num_kb = (int)((l.K + kBlock - 1) / kBlock);
  a.nt = plan.nt; a.split = plan.split;
  const int64_t tiles_m = (l.M + a.nt - 1) / a.nt, tiles = (l.N + kBlock - 1) / kBlock * tiles_m;
  const size_t stage = (GATED ? 2 : 1) * kBlockBytes + (size_t)a.nt * kBlock;
  const int own = (int)((std::min<int64_t>(l.M, a.nt) + a.split - 1) / a.split);
  while ((1 << a.own_log2) < own) ++a.own_log2;
  a.sums_bytes = a.split > 1 ? (uint32_t)((GATED ? 2 : 1) * a.split << a.own_log2) * kBlock * 4 : 0u;
  // A part of the contraction that is on its way at once anyhow gets half an SM's shared memory, so that the next kernel's CTAs find room
  // beside it (1 x 4096 x 4096 5.3 -> 4.5 us); longer ones get it all: CTAs of one kernel two to an SM leave others without (64 x 8192 x
  // 8192 14.7 us, 23 in half rings).
  const size_t blocks = (size_t)((a.num_kb + a.split - 1) / a.split), ring = blocks * stage;
  const bool shortly = ring <= 160 * 1024;
  a.stages = (int)std::min<size_t>({(size_t)kFewStages, blocks, (shortly ? kFewRing / 2 - std::min<size_t>(a.sums_bytes, kFewRing / 4) : kFewRing - a.sums_bytes) / stage});
  // Weights that do not stay in L2 between the calls of one layer: 24 x 8192 x 4096 gated 14.5 -> 14.0 us.  Smaller ones, when they are there, lose
  // by it (0.1 to 0.3 us, small calls); when they come from HBM, as those of a deep stack do, they would gain up to 0.7 (1 row of gated 4096 x
  // 1024 4.8 us, 4.1 with four blocks; of 4096 x 4096 none).
  a.prefetch = (GATED ? 2 : 1) * l.N * l.K >= (32ll << 20) ? 4 : 0;
  a.tiles_m = (int)tiles_m;
  a.idesc = make_idesc(2, 1, 1, kBlock, (uint32_t)a.nt);                      // s8 x s8 -> s32
  a.tmem_cols = std::max(32, a.nt * (GATED ? 2 : 1));
  a.sc = scales_of(l); a.out = l.out; a.ld = l.ld_out;
  a.vec = (reinterpret_cast<uintptr_t>(l.out) & (4 * sizeof(T) - 1)) == 0 && l.ld_out % 4 == 0;
  wait_settings(&a.waits.limit_ns, &a.waits.stop_after);
  CUtensorMap maps[3];
  if (!code_map(&maps[0], l.x, l.K, l.M, l.ld_x, a.nt) || !code_map(&maps[1], l.w[0], l.K, l.N, l.ld_w[0], kBlock)) return QM_ERR_CUDA;
  if (!GATED) maps[2] = maps[1];
  else if (!code_map(&maps[2], l.w[1], l.K, l.N, l.ld_w[1], kBlock)) return QM_ERR_CUDA;
  const size_t smem = 1024 + a.stages * stage + a.sums_bytes + sizeof(SharedFew);
  return launch_cluster(linear_few_kernel<T, ACT>, ready, smem, kFewSmem,
                        (unsigned)(tiles * a.split), kThreads, (unsigned)a.split, s, maps[0], maps[1], maps[2], a);
}

template <typename T, int ACT>
qm_status launch_many(const LinearArgs& l, cudaStream_t s) {
  constexpr bool GATED = ACT != kNoAct;
  static std::atomic<bool> ready[kMaxDevices];
  // all of an SM's shared memory: a CTA that holds tensor memory waits for its peer here, so neither may have to wait for another kernel's
  constexpr size_t smem = 232448;
  static_assert(1024 + (size_t)kManyStages * kManyStageBytes + kEpiWarps * kOutBytes + sizeof(SharedMany) <= smem, "shared memory of a CTA");
  ManyArgs a{};
  a.M = l.M; a.N = l.N;
  a.num_kb = (int)((l.K + kBlock - 1) / kBlock);
  a.tiles_n = (int)((l.N + (GATED ? 127 : 255)) / (GATED ? 128 : 256));
  const int64_t tiles = (l.M + 255) / 256 * a.tiles_n;
  if (tiles >= (1ll << 31) - 1024) return QM_ERR_UNSUPPORTED;                 // the walk adds the grid to an index
  a.num_tiles = (int)tiles;
  a.sc = scales_of(l); a.out = l.out; a.ld = l.ld_out;
  a.vec = rows_on_16(l);
  wait_settings(&a.waits.limit_ns, &a.waits.stop_after);
  CUtensorMap maps[4];
  if (!code_map(&maps[0], l.x, l.K, l.M, l.ld_x, kBlock) || !code_map(&maps[1], l.w[0], l.K, l.N, l.ld_w[0], kBlock)) return QM_ERR_CUDA;
  if (!GATED) maps[2] = maps[1];
  else if (!code_map(&maps[2], l.w[1], l.K, l.N, l.ld_w[1], kBlock)) return QM_ERR_CUDA;
  if (!a.vec) maps[3] = maps[0];                                              // not used
  else if (!out_map(&maps[3], l.out, l.out_dtype, l.M, l.N, l.ld_out)) return QM_ERR_CUDA;
  const int pairs = sm_count() / 2;
  return launch_cluster(linear_many_kernel<T, ACT>, ready, smem, smem, (unsigned)(2 * (tiles < pairs ? tiles : pairs)), kThreads, 2u, s, maps[0], maps[1],
                        maps[2], maps[3], a);
}

template <typename T, int ACT>
qm_status launch_sized(const LinearArgs& l, cudaStream_t s) {
  const Plan plan = make_plan(l, ACT != kNoAct, rows_on_16(l));
  return plan.nt ? launch_few<T, ACT>(l, plan, s) : launch_many<T, ACT>(l, s);
}

template <typename T>
qm_status launch_typed(const LinearArgs& l, cudaStream_t s) {
  if (!l.w[1]) return launch_sized<T, kNoAct>(l, s);
  if (l.act == QM_ACT_SILU) return launch_sized<T, QM_ACT_SILU>(l, s);
  return l.act == QM_ACT_GELU ? launch_sized<T, QM_ACT_GELU>(l, s) : launch_sized<T, QM_ACT_GELU_TANH>(l, s);
}

}  // namespace

qm_status launch_linear_int8(const LinearArgs& l, cudaStream_t s) {
  return l.out_dtype == QM_DT_BF16 ? launch_typed<__nv_bfloat16>(l, s) : launch_typed<float>(l, s);
}

}  // namespace qm
