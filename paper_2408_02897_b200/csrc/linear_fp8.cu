// The product of FP8 codes with a scale for each 128 entries of the contraction (qm_linear_fp8):
//   y_ij = sum_c dx[c][i] dw[c][j / side] S_c + bias_j,   S_c = sum of x_ik w_jk over the 128 k of block c
// S_c is what the tensor cores add up in tensor memory (tcgen05.mma kind::f8f6f4); the scales change with c, so every block's sums are
// taken out of there, scaled and added in fp32 registers, under the MMAs of the next block.  Written in bf16 or fp32.
//   linear_fp8_few    few rows of x: 128 rows of the WEIGHT as the MMA's M, up to 128 rows of x as its N, the contraction split over the CTAs
//                     of a cluster, whose sums are added in the order of the parts.
//   linear_fp8_many   CTA pairs (cta_group::2) on tiles of 256 rows of x and 256 weight rows, two blocks' sums in tensor memory.
//
// What the scales cost: 128 entries of a 256 x 256 tile take the CTA pair 610 to 720 ns (16384 x 4096 x 1024 90 to 97 us, 102 to 112 with a bias), 505 with the sums left unread. The multiply-adds
// are 257 cycles of it, under the MMAs; a buffer's round (MMA, commit, sums to registers, arrival at the leader, next MMA) is longer than two MMA times, and two
// buffers are all of tensor memory. A scale per weight row too is a second multiplication: 1000 to 1300 ns.
//
// Every mbarrier wait is bounded (Waiter): a CTA that gives up leaves NaN in the outputs it cannot compute, waits for what it has
// in flight, frees tensor memory and returns.
#include "linear_shared.cuh"

namespace qm {
namespace {

struct BlockScales {
  const float* dx;                             // [blocks of the contraction][M]
  const float* dw; int64_t dw_cols; int side;  // [blocks of the contraction][dw_cols], a column for `side` weight rows
  const void* bias; int bias_bf16;
};

__device__ __forceinline__ float load_bias(const BlockScales& s, int64_t n) {
  if (!s.bias) return 0.f;
  return s.bias_bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(s.bias)[n]) : static_cast<const float*>(s.bias)[n];
}
// acc += scale * (two sums out of tensor memory). Volatile, so that it stays behind the wait for them.
__device__ __forceinline__ void add_scaled(uint64_t& acc, uint32_t lo, uint32_t hi, uint64_t scale) {
  asm volatile("{\n\t.reg .b64 v;\n\tmov.b64 v, {%1, %2};\n\tfma.rn.f32x2 %0, v, %3, %0;\n\t}" : "+l"(acc) : "r"(lo), "r"(hi), "l"(scale));
}
__device__ __forceinline__ void add_scaled(uint64_t& acc, uint32_t lo, uint32_t hi, uint64_t column, uint64_t scale) {
  asm volatile("{\n\t.reg .b64 v;\n\tmov.b64 v, {%1, %2};\n\tmul.rn.f32x2 v, v, %3;\n\tfma.rn.f32x2 %0, v, %4, %0;\n\t}"
               : "+l"(acc) : "r"(lo), "r"(hi), "l"(column), "l"(scale));
}
// Scales on their way to shared memory, four bytes a copy (0 where there is none): a block's are asked for several blocks ahead, which registers
// that are handed on from round to round would wait for a round later.
__device__ __forceinline__ void copy4(uint32_t dst, const float* src, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4u : 0u) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }
constexpr int kAhead = 6;                      // blocks whose scales are in shared memory or on their way there

__device__ __forceinline__ void add4(float4& a, const float4& b) { a.x += b.x; a.y += b.y; a.z += b.z; a.w += b.w; }

// ------------------------------------------------------------------ few rows
// One tile of 128 weight rows x NT rows of x per CTA, or per cluster that splits the contraction.  Roles: warp 0 issues TMA loads into a
// ring, warp 1 holds tensor memory and issues the MMAs, warps 2..9 add the blocks' sums up: the two warps of a lane quarter take half
// of the NT columns each (of 16, one of them takes all).  1 x 4096 x 1024 3.2 us, a chain of latencies; 64 x 8192 x 8192 19.2, weights from HBM (10.5 for their
// bytes): 300 to 550 ns for each 128 entries, 15.7 us with the sums left unread.
struct FewArgs {
  int64_t M, N;
  int num_kb, tiles_m, split, stages;
  uint32_t sums_bytes;
  int prefetch;                              // weight blocks asked into L2 ahead of the kernel before this one
  int own_log2;                              // of a split contraction, rows of x that a CTA of the cluster finishes
  uint32_t idesc;
  BlockScales sc;
  Waits waits;
  void* out; int64_t ld;
  int vec;                                   // four outputs at a multiple of four start on as many bytes
};
constexpr int kFewStages = 12;
constexpr int kMaxSplit = 8;
__host__ __device__ constexpr int few_cols(int nt) { return nt < 32 ? nt : nt / 2; }            // columns of a thread
__host__ __device__ constexpr int few_bufs(int nt) { return nt < 128 ? 4 : 2; }                 // blocks' sums in tensor memory
__host__ __device__ constexpr uint32_t few_scale_bytes(int nt) { return kEpiWarps * kAhead * (few_cols(nt) + 32) * 4; }
struct SharedFew {
  uint64_t full[kFewStages], empty[kFewStages], sum_full[4], sum_empty[4], drain, read;
  uint32_t tmem_base, abort_flag, gave_up, pad;        // gave_up: some CTA of the cluster did
};

template <typename T, int NT>
__global__ void __launch_bounds__(kThreads, NT == 128 ? 1 : 2)
linear_fp8_few(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const FewArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  constexpr int kCols = few_cols(NT), kBufs = few_bufs(NT);
  constexpr uint32_t kStage = kBlockBytes + (uint32_t)NT * kBlock, kTmemCols = NT * kBufs;
  // behind the ring: of a split contraction the parts' sums of this CTA's rows, [part][row][weight row]
  float* const sums = reinterpret_cast<float*>(tiles + (size_t)a.stages * kStage);
  // (16-byte aligned, as everything here)
  float* const scales = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(sums) + a.sums_bytes);
  SharedFew* sh = reinterpret_cast<SharedFew*>(reinterpret_cast<uint8_t*>(scales) + few_scale_bytes(NT));
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const int tile = (int)blockIdx.x / a.split, part = (int)blockIdx.x - tile * a.split;
  const int n0 = tile / a.tiles_m * kBlock, m0 = tile % a.tiles_m * NT;
  const int kb0 = (int)((int64_t)a.num_kb * part / a.split), kb1 = (int)((int64_t)a.num_kb * (part + 1) / a.split);
  const Waiter w{&sh->abort_flag, nullptr, a.waits.limit_ns};

  if (warp == 0 && lane < 2) {
    const CUtensorMap* maps[2] = {&map_x, &map_w};
    asm volatile("prefetch.tensormap [%0];" ::"l"(maps[lane]) : "memory");
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < a.stages; ++s) {
      mbar_init(smem_u32(&sh->full[s]), 1);
      mbar_init(smem_u32(&sh->empty[s]), 1);
    }
    for (int b = 0; b < kBufs; ++b) {
      mbar_init(smem_u32(&sh->sum_full[b]), 1);
      mbar_init(smem_u32(&sh->sum_empty[b]), NT < 32 ? kEpiWarps / 2 : kEpiWarps);
    }
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
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh->tmem_base)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  // The next kernel in the stream is let in when this one's loads are all on their way.  What this one does ahead of its own wait is a
  // prefetch into L2, which a later write cannot make stale: of large weights the first blocks.
  if (a.prefetch && warp == 0 && lane == 0)
    for (int k = 0; k < a.prefetch && kb0 + k < kb1; ++k) prefetch_2d(&map_w, (kb0 + k) * kBlock, n0);
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
        const uint32_t bar = smem_u32(&sh->full[s]), base = smem_u32(tiles) + (uint32_t)s * kStage;
        mbar_expect_tx(bar, kStage);
        tma_load_2d_local(base, &map_w, bar, kb * kBlock, n0);
        tma_load_2d_local(base + kBlockBytes, &map_x, bar, kb * kBlock, m0);
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
    for (int kb = kb0, g = 0; kb < kb1; ++kb, ++g) {
      const int buf = g % kBufs;
      if (g >= kBufs && !w.wait_warp(smem_u32(&sh->sum_empty[buf]), (uint32_t)(g / kBufs - 1) & 1u)) break;
      if (!w.wait_warp(smem_u32(&sh->full[s]), parity)) break;
      tc_fence_after();
      const uint32_t base = smem_u32(tiles) + (uint32_t)s * kStage;
      const uint64_t dw = smem_desc(base, 128), dx = smem_desc(base + kBlockBytes, 128);
      if (lead) {
#pragma unroll
        for (int k = 0; k < 4; ++k)                 // 32 codes per instruction
          mma_f8_one(tmem_base + (uint32_t)(buf * NT), dw + 2 * k, dx + 2 * k, a.idesc, k ? 1u : 0u);
        tc_commit_one(smem_u32(&sh->sum_full[buf]));
        tc_commit_one(smem_u32(&sh->empty[s]));
      }
      if (++s == a.stages) { s = 0; parity ^= 1u; }
    }
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
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(kTmemCols) : "memory");
  }

  // warps 2..9: lanes 32 (warp % 4) .. of tensor memory, columns (rows of x) kCols h ..
  const int et = (int)threadIdx.x - 64, q = warp & 3, h = (warp - 2) >> 2;
  const int live = (int)(a.M - m0 < NT ? a.M - m0 : NT);                     // rows of x in this tile
  const int own = 1 << a.own_log2;
  T* const out = static_cast<T*>(a.out);
  if (warp >= 2) {
    bool ok = true;
    uint64_t acc[kCols / 2];
#pragma unroll
    for (int i = 0; i < kCols / 2; ++i) acc[i] = 0;
    const int c0 = h * kCols;
    if (NT >= 32 || h == 0) {
      const int64_t n = (int64_t)n0 + q * 32 + lane;
      const int64_t wcol = a.sc.side == 1 ? (n < a.N ? n : a.N - 1) : n0 / kBlock;
      // a block's scales: of x for the thread's columns, then of the weights for the warp's 32 lanes (or one for all)
      constexpr int kSlot = kCols + 32;
      float* const ring = scales + (warp - 2) * kAhead * kSlot;
      const float* px[(kCols + 31) / 32];
      bool there[(kCols + 31) / 32];
#pragma unroll
      for (int i = 0; i < (kCols + 31) / 32; ++i) {
        there[i] = c0 + 32 * i + lane < live;
        px[i] = a.sc.dx + (int64_t)kb0 * a.M + m0 + (there[i] ? c0 + 32 * i + lane : 0);
      }
      const float* pw = a.sc.dw + (int64_t)kb0 * a.sc.dw_cols + wcol;
      uint32_t put = smem_u32(ring + lane);
      const uint32_t put_end = put + kAhead * kSlot * 4;
      int left = kb1 - kb0;
      // (addresses and conditions are handed on from block to block: 256 x 4096 x 4096 18.7 -> 18.0 us, where no copies at all would leave 14.7)
      auto fetch = [&]() {
        if (left-- > 0) {
#pragma unroll
          for (int i = 0; i < (kCols + 31) / 32; ++i) {
            if (kCols >= 32 || lane < kCols) copy4(put + 128 * i, px[i], there[i]);
            px[i] += a.M;
          }
          copy4(put + kCols * 4, pw, true);
          pw += a.sc.dw_cols;
        }
        copies_commit();
        put += kSlot * 4;
        if (put == put_end) put -= kAhead * kSlot * 4;
      };
      for (int d = 0; d < kAhead - 1; ++d) fetch();
      const uint32_t lane_addr = tmem_base + ((uint32_t)(q * 32) << 16) + c0;
      int slot = 0;
      for (int kb = kb0, g = 0; kb < kb1; ++kb, ++g) {
        const int buf = g % kBufs;
        copies_wait<kAhead - 2>();
        __syncwarp();                                                        // (and the slot that is filled next has been read by all lanes)
        fetch();
        const float* const dx = ring + slot * kSlot;
        const uint64_t dw = both(dx[kCols + lane]);
        slot = slot == kAhead - 1 ? 0 : slot + 1;
        ok = w.wait_warp(smem_u32(&sh->sum_full[buf]), (uint32_t)(g / kBufs) & 1u);
        if (!ok) break;
        tc_fence_after();
#pragma unroll
        for (int c = 0; c < kCols; c += 16) {
          uint32_t r[16];
          tmem_ld16(lane_addr + buf * NT + c, r);
          float4 d[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) d[i] = *reinterpret_cast<const float4*>(dx + c + 4 * i);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            add_scaled(acc[c / 2 + 2 * i], r[4 * i], r[4 * i + 1], mul2(pair_of(d[i].x, d[i].y), dw));
            add_scaled(acc[c / 2 + 2 * i + 1], r[4 * i + 2], r[4 * i + 3], mul2(pair_of(d[i].z, d[i].w), dw));
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sh->sum_empty[buf]));
      }
    }
    copies_wait<0>();                                                         // (of scales that a kernel which gives up has not used)
    if (lane == 0) mbar_arrive(smem_u32(&sh->read));
    if (a.split == 1) {
      const int64_t n = (int64_t)n0 + q * 32 + lane;
      const float bias = n < a.N ? load_bias(a.sc, n) : 0.f;
      T* p = out + (int64_t)(m0 + c0) * a.ld + n;
#pragma unroll
      for (int i = 0; i < kCols; ++i, p += a.ld) {
        float y[2];
        halves(acc[i / 2], y[0], y[1]);
        if (n < a.N && c0 + i < live && (NT >= 32 || h == 0)) *p = (T)(ok ? y[i & 1] + bias : nan_f());
      }
    } else {
      // this part's sums to the CTAs that finish their rows
      cluster_wait();
      if (!ok && lane < a.split) sts_cluster(map_to_cta(smem_u32(&sh->gave_up), lane), 1u);
      if (ok && (NT >= 32 || h == 0)) {
        const uint32_t at = smem_u32(sums + part * own * kBlock + q * 32 + lane);
#pragma unroll
        for (int i = 0; i < kCols; ++i) {
          float y[2];
          halves(acc[i / 2], y[0], y[1]);
          const int c = c0 + i;
          if (c < live) sts_cluster(map_to_cta(at, c >> a.own_log2) + (uint32_t)((c & (own - 1)) * kBlock * 4), __float_as_uint(y[i & 1]));
        }
      }
      cluster_arrive();
    }
  }
  if (a.split > 1) {
    cluster_wait();
    const int j = 4 * (et & (kBlock / 4 - 1));                                // a thread finishes four neighbouring weight rows at a time
    const int cols = (int)(a.N - n0 - j < 4 ? a.N - n0 - j : 4);
    if (warp >= 2 && cols > 0) {
      float bias[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) bias[k] = k < cols ? load_bias(a.sc, (int64_t)n0 + j + k) : 0.f;
      const bool ok = sh->gave_up == 0;
      const int rows = min(own, live - part * own);
      for (int i = et / (kBlock / 4); i < rows; i += 256 / (kBlock / 4)) {
        float4 g = make_float4(0.f, 0.f, 0.f, 0.f);
        const float4* from = reinterpret_cast<const float4*>(sums + i * kBlock + j);
#pragma unroll 2
        for (int p = 0; p < a.split; ++p, from += own * (kBlock / 4)) add4(g, *from);
        float y[4] = {g.x + bias[0], g.y + bias[1], g.z + bias[2], g.w + bias[3]};
#pragma unroll
        for (int k = 0; k < 4; ++k) if (!ok) y[k] = nan_f();
        store4(out + (int64_t)(m0 + part * own + i) * a.ld + n0 + j, y, cols, a.vec);
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
// Persistent CTA pairs on tiles of 256 rows of x and 256 weight rows, a stage of 32 KB a CTA for 128 contraction entries, five stages, the
// sums of two blocks in tensor memory (all of its 512 columns).  Eight warps add up: a thread keeps half a row of the tile in 128 registers.
struct ManyArgs {
  int64_t M, N;
  int num_kb, tiles_n, num_tiles;
  uint32_t idesc;
  BlockScales sc;
  Waits waits;
  void* out; int64_t ld;
  int vec;                                     // rows of the output start on 16 bytes
};
constexpr int kManyStages = 5;
// Warps 0 and 1 as above, 2 and 3 idle (registers are handed out by four warps), 4..11 add up.
constexpr int kManyThreads = 384, kManyRegs = 168, kRegsFew = 40, kRegsMany = 232;
static_assert(kRegsFew + 2 * kRegsMany <= 3 * kManyRegs, "an increase that the block's registers cannot serve waits for ever");
template <int N> __device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
constexpr uint32_t kManyStageBytes = 2 * kBlockBytes;
constexpr uint32_t kOutBytes = 32 * 128;       // of output on its way per epilogue warp: 32 rows of 128 bytes
// floats of a block's scales in a warp's ring: 32 rows, and 128 columns or one
__host__ __device__ constexpr int many_slot(bool side1) { return side1 ? 160 : 36; }
__host__ __device__ constexpr uint32_t many_scale_bytes(bool side1) { return kEpiWarps * kAhead * many_slot(side1) * 4; }
struct SharedMany {
  uint64_t full[kManyStages], empty[kManyStages], sum_full[2], sum_empty[2], drain;
  uint32_t tmem_base, abort_flag, issued, peer_gave_up, peer_issued, pad[3];
  alignas(16) float bias[256];
};

// 32 (fp32) or 64 (bf16) columns of a thread's row to the warp's staging buffer: rows of 128 bytes, 16-byte units permuted with the row.
__device__ __forceinline__ void stage_row(uint32_t stage, int lane, const float (&y)[32]) {
#pragma unroll
  for (int u = 0; u < 8; ++u)
    asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(stage + lane * 128 + ((u ^ (lane & 7)) << 4)), "f"(y[4 * u]), "f"(y[4 * u + 1]),
                 "f"(y[4 * u + 2]), "f"(y[4 * u + 3]) : "memory");
}
__device__ __forceinline__ void stage_row(uint32_t stage, int lane, const float (&y)[64]) {
#pragma unroll
  for (int u = 0; u < 8; ++u) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 v = __floats2bfloat162_rn(y[8 * u + 2 * i], y[8 * u + 2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(stage + lane * 128 + ((u ^ (lane & 7)) << 4)), "r"(w[0]), "r"(w[1]), "r"(w[2]),
                 "r"(w[3]) : "memory");
  }
}

// SIDE1: the weight has a scale per row too, not one for 128.
template <typename T, bool SIDE1>
__global__ void __launch_bounds__(kManyThreads, 1)
linear_fp8_many(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_out,
                const ManyArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* const staging = tiles + (size_t)kManyStages * kManyStageBytes;
  float* const scales = reinterpret_cast<float*>(staging + kEpiWarps * kOutBytes);
  SharedMany* sh = reinterpret_cast<SharedMany*>(reinterpret_cast<uint8_t*>(scales) + many_scale_bytes(SIDE1));
  const int warp = __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1, num_pairs = gridDim.x >> 1;
  const Waiter w{&sh->abort_flag, nullptr, a.waits.limit_ns};

  if (warp == 0 && lane < 3) {
    const CUtensorMap* maps[3] = {&map_x, &map_w, &map_out};
    asm volatile("prefetch.tensormap [%0];" ::"l"(maps[lane]) : "memory");
  }
  if (threadIdx.x == 0) {
    for (int s = 0; s < kManyStages; ++s) {
      mbar_init(smem_u32(&sh->full[s]), 1);
      mbar_init(smem_u32(&sh->empty[s]), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(smem_u32(&sh->sum_full[b]), 1);
      mbar_init(smem_u32(&sh->sum_empty[b]), 2 * kEpiWarps);
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
    regs_down<kRegsFew>();
    // TMA producer (both CTAs): this CTA's 128 rows of x, and its half of the tile's weight rows
    if (lane == 0) {
      uint32_t g = 0;
      int s = 0;
      uint32_t parity = 0;
      bool ok = true;
      for (int t = pair; t < a.num_tiles && ok; t += num_pairs) {
        const int tm = t / a.tiles_n;
        const int r0 = tm * 256 + (int)rank * kBlock, c0 = (t - tm * a.tiles_n) * 256 + (int)rank * kBlock;
        for (int kb = 0; kb < a.num_kb; ++kb, ++g) {
          if (g >= a.waits.stop_after || (g >= (uint32_t)kManyStages && !w.wait(smem_u32(&sh->empty[s]), parity ^ 1u))) { ok = false; break; }
          if (rank == 0) mbar_expect_tx(smem_u32(&sh->full[s]), 2 * kManyStageBytes);
          const uint32_t bar = map_to_cta(smem_u32(&sh->full[s]), 0), base = smem_u32(tiles) + (uint32_t)s * kManyStageBytes;
          tma_load_2d(base, &map_x, bar, kb * kBlock, r0);
          tma_load_2d(base + kBlockBytes, &map_w, bar, kb * kBlock, c0);
          if (++s == kManyStages) { s = 0; parity ^= 1u; }
        }
      }
      sh->issued = g;
    }
  } else if (warp == 1) {
    regs_down<kRegsFew>();
    if (rank == 0) {
      const bool lead = elect_one();
      uint32_t it = 0;
      int s = 0;
      uint32_t parity = 0;
      bool ok = true;
      for (int t = pair; t < a.num_tiles && ok; t += num_pairs) {
        for (int kb = 0; kb < a.num_kb; ++kb, ++it) {
          const uint32_t buf = it & 1;
          if (!w.wait_warp(smem_u32(&sh->full[s]), parity)) { ok = false; break; }
          const uint32_t base = smem_u32(tiles) + (uint32_t)s * kManyStageBytes;
          const uint64_t da = smem_desc(base, 128), db = smem_desc(base + kBlockBytes, 128);
          if (it >= 2 && !w.wait_warp(smem_u32(&sh->sum_empty[buf]), ((it >> 1) - 1) & 1)) { ok = false; break; }
          tc_fence_after();
          if (lead) {
#pragma unroll
            for (int k = 0; k < 4; ++k) mma_pair<kKindF8>(tmem_base + buf * 256, da + 2 * k, db + 2 * k, a.idesc, k ? 1u : 0u, true);
            tc_commit_pair(smem_u32(&sh->sum_full[buf]), true);
            tc_commit_pair(smem_u32(&sh->empty[s]), true);
          }
          if (++s == kManyStages) { s = 0; parity ^= 1u; }
        }
      }
    }
  } else if (warp < 4) {
    regs_down<kRegsFew>();
  } else {
    regs_up<kRegsMany>();
    // warps 4..11 of both CTAs: rows 32 (warp % 4) .. of the CTA's 128, columns 128 h ..
    const int q = warp & 3, h = (warp - 4) >> 2, et = (int)threadIdx.x - 128;
    uint4* const stage = reinterpret_cast<uint4*>(staging + (warp - 4) * kOutBytes);
    T* const out = static_cast<T*>(a.out);
    constexpr int kChunk = 128 / sizeof(T);
    const bool has_bias = a.sc.bias != nullptr;
    bool ok = true;
    uint32_t it = 0;
    // A block's scales: of x for the warp's 32 rows, then of the weight for its 128 columns.  They are asked for across the ends of tiles.
    constexpr int kSlot = many_slot(SIDE1);
    float* const ring = scales + (warp - 4) * kAhead * kSlot;
    int ft = pair, left = 0, put = 0, slot = 0, in_w = 0;
    const float *px = nullptr, *pw = nullptr;
    bool in_x = false;
    auto fetch = [&]() {
      if (left == 0 && ft < a.num_tiles) {
        const int tm = ft / a.tiles_n;
        const int64_t row = (int64_t)tm * 256 + rank * kBlock + q * 32 + lane, c = (int64_t)(ft - tm * a.tiles_n) * 256 + h * 128;
        const int64_t col = SIDE1 ? c + lane : c / kBlock;
        in_x = row < a.M;
        in_w = col < a.sc.dw_cols ? (int)(a.sc.dw_cols - col < 128 ? a.sc.dw_cols - col : 128) : 0;         // columns from this lane's on
        px = a.sc.dx + (in_x ? row : 0); pw = a.sc.dw + (in_w ? col : 0);
        left = a.num_kb;
      }
      if (left > 0) {
        const uint32_t to = smem_u32(ring + put * kSlot + lane);
        copy4(to, px, in_x);
        if (SIDE1) {
#pragma unroll
          for (int i = 0; i < 4; ++i) copy4(to + 128 * (i + 1), in_w > 32 * i ? pw + 32 * i : a.sc.dw, in_w > 32 * i);
        } else if (lane == 0) {
          copy4(to + 128, pw, in_w > 0);
        }
        px += a.M; pw += a.sc.dw_cols;
        if (--left == 0) ft += num_pairs;
      }
      copies_commit();
      put = put == kAhead - 1 ? 0 : put + 1;
    };
    for (int d = 0; d < kAhead - 1; ++d) fetch();
    for (int t = pair; t < a.num_tiles; t += num_pairs) {
      const int tm = t / a.tiles_n;
      const int64_t c0 = (int64_t)(t - tm * a.tiles_n) * 256;
      const int64_t row0 = (int64_t)tm * 256 + rank * kBlock + q * 32;
      const int rows = (int)(a.M - row0 < 32 ? a.M - row0 : 32);             // <= 0: none
      if (has_bias) {                                                         // (the barriers: all have read the last tile's, all are written)
        asm volatile("bar.sync 1, 256;" ::: "memory");
        sh->bias[et] = c0 + et < a.N ? load_bias(a.sc, c0 + et) : 0.f;
        asm volatile("bar.sync 1, 256;" ::: "memory");
      }
      uint64_t acc[64];
#pragma unroll
      for (int i = 0; i < 64; ++i) acc[i] = 0;
      for (int kb = 0; kb < a.num_kb && ok; ++kb, ++it) {
        const uint32_t buf = it & 1, from = tmem_base + ((uint32_t)(q * 32) << 16) + buf * 256 + h * 128;
        copies_wait<kAhead - 2>();
        __syncwarp();                                                         // (and the slot that is filled next has been read by all lanes)
        fetch();
        const float* const sc = ring + slot * kSlot;
        const uint64_t scale = both(SIDE1 ? sc[lane] : sc[lane] * sc[32]);
        slot = slot == kAhead - 1 ? 0 : slot + 1;
        float4 d[2][SIDE1 ? 4 : 1];
        auto columns = [&](int c) {
#pragma unroll
          for (int i = 0; i < 4; ++i) d[c & 1][SIDE1 ? i : 0] = *reinterpret_cast<const float4*>(sc + 32 + 16 * c + 4 * i);
        };
        if (SIDE1) columns(0);
        // (a warp that gives up arrives no more: an arrival for sums that it has not read would let others be overwritten that a peer yet reads)
        ok = w.wait_warp(smem_u32(&sh->sum_full[buf]), (it >> 1) & 1);
        if (!ok) break;
        tc_fence_after();
        uint32_t r[2][16];
        tmem_ld16(from, r[0]);
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          tmem_ld_wait();
          if (c < 7) {
            if (SIDE1) columns(c + 1);
            tmem_ld16(from + 16 * (c + 1), r[(c + 1) & 1]);
          } else {                                                            // all of it is in registers
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(map_to_cta(smem_u32(&sh->sum_empty[buf]), 0));
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float4& e = d[c & 1][SIDE1 ? i / 2 : 0];
            if (SIDE1) add_scaled(acc[8 * c + i], r[c & 1][2 * i], r[c & 1][2 * i + 1], i & 1 ? pair_of(e.z, e.w) : pair_of(e.x, e.y), scale);
            else add_scaled(acc[8 * c + i], r[c & 1][2 * i], r[c & 1][2 * i + 1], scale);
          }
        }
      }
#pragma unroll
      for (int ch = 0; ch < 128 / kChunk; ++ch) {
        const int64_t col = c0 + h * 128 + ch * kChunk;
        if (col < a.N) {                                                      // uniform across the warp
          const int cols = (int)(a.N - col < kChunk ? a.N - col : kChunk);
          if (a.vec) {                                                        // the last copy has read the buffer
            if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
            __syncwarp();
          }
          float y[kChunk];
#pragma unroll
          for (int i = 0; i < kChunk; i += 2) {
            halves(acc[(ch * kChunk + i) / 2], y[i], y[i + 1]);
            if (has_bias) {
              const float2 b = *reinterpret_cast<const float2*>(&sh->bias[h * 128 + ch * kChunk + i]);
              y[i] += b.x; y[i + 1] += b.y;
            }
            if (!ok) y[i] = y[i + 1] = nan_f();
          }
          stage_row(smem_u32(stage), lane, y);
          if (a.vec) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
              if (rows > 0) tma_store_2d(&map_out, smem_u32(stage), (int)col, (int)row0);         // clipped to M x N
              asm volatile("cp.async.bulk.commit_group;" ::: "memory");
            }
          } else {
            __syncwarp();
            T* const to = out + row0 * a.ld + col;
            if (sizeof(T) == 2 && ((reinterpret_cast<uintptr_t>(to) & 3) | (a.ld & 1)) == 0) {
              store_rows(stage, lane, reinterpret_cast<uint32_t*>(to), a.ld >> 1, rows, cols >> 1);
              if ((cols & 1) && lane < rows) to[lane * a.ld + cols - 1] = reinterpret_cast<const T*>(stage)[lane * kChunk + (((cols - 1) / 8) ^ (lane & 7)) * 8 + (cols - 1) % 8];
            } else {
              store_rows(stage, lane, to, a.ld, rows, cols);
            }
            __syncwarp();
          }
        }
      }
    }
    copies_wait<0>();                                                         // (of scales that a kernel which gives up has not used)
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
bool rows_on_16(const LinearFp8Args& l) {
  return (reinterpret_cast<uintptr_t>(l.out) & 15) == 0 && l.ld_out * (l.out_dtype == QM_DT_BF16 ? 2 : 4) % 16 == 0;
}

BlockScales scales_of(const LinearFp8Args& l) {
  return {l.dx, l.dw, (l.N + l.side_w - 1) / l.side_w, l.side_w, l.bias, l.bias_dtype == QM_DT_BF16};
}

// D in fp32, E4M3 is 0 and E5M2 is 1
uint32_t idesc_of(int fmt_a, int fmt_b, uint32_t m, uint32_t n) {
  return make_idesc(1, fmt_a == QM_FMT_E5M2, fmt_b == QM_FMT_E5M2, m, n);
}

// Which kernel, and how the few rows' one is cut (rows of x per tile, parts of the contraction): by the time that it takes, in ns, as measured back to back
// over 538 shapes and scales (M 1 to 16384, N 256 to 8192, K 256 to 16384) in all cuts that each has: a part of the contraction costs kBase and kDepth
// for each 128 entries, one that is joined kSplit, further rounds of CTAs what is above kFirst. A scale for each weight row is no more work for the few rows' kernel (less: its scales' copies
// are not of one address), the many rows' takes 950 ns instead of 570. Predicted within 15 % for 535 of them; what is chosen is 0.3 % slower on the average than
// the best, 10 % at most. Examples (us; a tile's rows and parts): 1024 x 1024 x 4096 (128, 2) 15.0, (64, 1) 17.8, many 22.1; 4096 x 1024 x 16384 with a
// scale for each weight row many 124, (128, 1) 130; 1536 x 4096 x 4096 so (128, 1) 57, many 66, with one for 128 66 and 42.
struct Plan { int nt, split; };            // nt 0: the many rows' kernel
Plan make_plan(const LinearFp8Args& l, bool aligned) {
  static constexpr int kNt[4] = {16, 32, 64, 128};
  static constexpr int64_t kFirst[4] = {1600, 1450, 1300, 150};
  static constexpr int64_t kBase[2][4] = {{2100, 2400, 2850, 3900}, {2100, 2200, 2850, 3950}};
  static constexpr int64_t kDepth[2][4] = {{310, 355, 480, 545}, {310, 330, 400, 470}};
  static constexpr int64_t kSplit[2][4] = {{890, 980, 1420, 2270}, {890, 1100, 1480, 2320}};
  const int64_t sms = sm_count(), num_kb = (l.K + kBlock - 1) / kBlock, tiles_n = (l.N + kBlock - 1) / kBlock;
  const int64_t pairs = sms / 2, tiles = (l.M + 255) / 256 * ((l.N + 255) / 256), written = !aligned ? 5500 : l.out_dtype == QM_DT_BF16 ? 1600 : 2600;
  const bool side1 = l.side_w == 1;
  int64_t best = (side1 ? 3700 : 3200) + (tiles + pairs - 1) / pairs * ((side1 ? 950 : 570) * num_kb + written);
  Plan plan{0, 1};
  for (int i = 0; i < 4 && (i == 0 || kNt[i - 1] < l.M); ++i) {
    const int64_t ctas = tiles_n * ((l.M + kNt[i] - 1) / kNt[i]);
    if (ctas > 64 * sms) continue;
    // (a cluster lies inside one of the GPU's eight groups of SMs, so not every SM is in one of four or eight)
    for (int split = 1; split <= kMaxSplit && split <= num_kb && (split == 1 || ctas * split <= sms - 4 * split); split *= 2) {
      const int64_t one = kBase[side1][i] + (num_kb + split - 1) / split * kDepth[side1][i] + (split > 1 ? kSplit[side1][i] : 0);
      const int64_t t = kFirst[i] + (ctas * split + sms - 1) / sms * (one - kFirst[i]);
      if (t < best) { best = t; plan = {kNt[i], split}; }
    }
  }
  return plan;
}

constexpr size_t kFewRing = 200 * 1024;
constexpr size_t kFewSmem = 1024 + kFewRing + few_scale_bytes(128) + sizeof(SharedFew);

template <typename T, int NT>
qm_status launch_few(const LinearFp8Args& l, int split, cudaStream_t s) {
  static std::atomic<bool> ready[kMaxDevices];
  FewArgs a{};
  a.M = l.M; a.N = l.N;
  a.num_kb = (int)((l.K + kBlock - 1) / kBlock);
  a.split = split;
  const int64_t tiles_m = (l.M + NT - 1) / NT, tiles = (l.N + kBlock - 1) / kBlock * tiles_m;
  const size_t stage = kBlockBytes + (size_t)NT * kBlock;
  const int own = (int)((std::min<int64_t>(l.M, NT) + split - 1) / split);
  while ((1 << a.own_log2) < own) ++a.own_log2;
  a.sums_bytes = split > 1 ? (uint32_t)(split << a.own_log2) * kBlock * 4 : 0u;
  // as in the INT8 product: half an SM's shared memory for a part that is on its way at once anyhow
  const size_t blocks = (size_t)((a.num_kb + split - 1) / split), ring = blocks * stage;
  const bool shortly = ring <= 160 * 1024;
  a.stages = (int)std::min<size_t>({(size_t)kFewStages, blocks, (shortly ? kFewRing / 2 - 10240 - std::min<size_t>(a.sums_bytes, kFewRing / 4) : kFewRing - a.sums_bytes) / stage});
  a.prefetch = l.N * l.K >= (32ll << 20) ? 4 : 0;
  a.tiles_m = (int)tiles_m;
  a.idesc = idesc_of(l.fmt_w, l.fmt_x, kBlock, NT);
  a.sc = scales_of(l); a.out = l.out; a.ld = l.ld_out;
  a.vec = (reinterpret_cast<uintptr_t>(l.out) & (4 * sizeof(T) - 1)) == 0 && l.ld_out % 4 == 0;
  wait_settings(&a.waits.limit_ns, &a.waits.stop_after);
  CUtensorMap maps[2];
  if (!code_map(&maps[0], l.x, l.K, l.M, l.ld_x, NT) || !code_map(&maps[1], l.w, l.K, l.N, l.ld_w, kBlock)) return QM_ERR_CUDA;
  const size_t smem = 1024 + a.stages * stage + a.sums_bytes + few_scale_bytes(NT) + sizeof(SharedFew);
  return launch_cluster(linear_fp8_few<T, NT>, ready, smem, kFewSmem, (unsigned)(tiles * split), kThreads, (unsigned)split, s, maps[0], maps[1], a);
}

template <typename T, bool SIDE1>
qm_status launch_many(const LinearFp8Args& l, cudaStream_t s) {
  static std::atomic<bool> ready[kMaxDevices];
  // all of an SM's shared memory: a CTA that holds tensor memory waits for its peer here, so neither may have to wait for another kernel's
  constexpr size_t smem = 232448;
  static_assert(1024 + (size_t)kManyStages * kManyStageBytes + kEpiWarps * kOutBytes + many_scale_bytes(SIDE1) + sizeof(SharedMany) <= smem, "shared memory of a CTA");
  ManyArgs a{};
  a.M = l.M; a.N = l.N;
  a.num_kb = (int)((l.K + kBlock - 1) / kBlock);
  a.tiles_n = (int)((l.N + 255) / 256);
  const int64_t tiles = (l.M + 255) / 256 * a.tiles_n;
  if (tiles >= (1ll << 31) - 1024) return QM_ERR_UNSUPPORTED;                 // the walk adds the grid to an index
  a.num_tiles = (int)tiles;
  a.idesc = idesc_of(l.fmt_x, l.fmt_w, 256, 256);
  a.sc = scales_of(l); a.out = l.out; a.ld = l.ld_out;
  a.vec = rows_on_16(l);
  wait_settings(&a.waits.limit_ns, &a.waits.stop_after);
  CUtensorMap maps[3];
  if (!code_map(&maps[0], l.x, l.K, l.M, l.ld_x, kBlock) || !code_map(&maps[1], l.w, l.K, l.N, l.ld_w, kBlock)) return QM_ERR_CUDA;
  if (!a.vec) maps[2] = maps[0];                                              // not used
  else if (!out_map(&maps[2], l.out, l.out_dtype, l.M, l.N, l.ld_out)) return QM_ERR_CUDA;
  static std::atomic<bool> split[kMaxDevices];                                // whether the registers are known to be there
  const int dev = current_device();
  if (dev < 0) return QM_ERR_UNSUPPORTED;
  if (!split[dev].load(std::memory_order_relaxed)) {
    cudaFuncAttributes fa{};
    QM_CUDA_OK(cudaFuncGetAttributes(&fa, linear_fp8_many<T, SIDE1>));
    if (fa.numRegs < kManyRegs) return QM_ERR_UNSUPPORTED;
    split[dev].store(true, std::memory_order_relaxed);
  }
  const int pairs = sm_count() / 2;
  return launch_cluster(linear_fp8_many<T, SIDE1>, ready, smem, smem, (unsigned)(2 * (tiles < pairs ? tiles : pairs)), kManyThreads, 2u, s, maps[0], maps[1], maps[2], a);
}

template <typename T>
qm_status launch_typed(const LinearFp8Args& l, cudaStream_t s) {
  const Plan plan = make_plan(l, rows_on_16(l));
  switch (plan.nt) {
    case 0: return l.side_w == 1 ? launch_many<T, true>(l, s) : launch_many<T, false>(l, s);
    case 16: return launch_few<T, 16>(l, plan.split, s);
    case 32: return launch_few<T, 32>(l, plan.split, s);
    case 64: return launch_few<T, 64>(l, plan.split, s);
    default: return launch_few<T, 128>(l, plan.split, s);
  }
}

}  // namespace

qm_status launch_linear_fp8(const LinearFp8Args& l, cudaStream_t s) {
  return l.out_dtype == QM_DT_BF16 ? launch_typed<__nv_bfloat16>(l, s) : launch_typed<float>(l, s);
}

}  // namespace qm
