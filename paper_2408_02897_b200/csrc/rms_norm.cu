// Root-mean-square norm with the residual's addition and an output in 8 bits (qm_rms_norm_quantize).
//
// Per row: z = x + residual, rounded to the stream's type; v = z w in fp32; Eq. 1 over v: d = max|v| / qmax,
// code = sat(RTNE(v / d)).  The norm's factor f = 1 / sqrt(mean(z^2) + eps) is the same positive number for the whole
// row, so it cancels in v f / (max|v f| / qmax) and goes into the scale alone: delta = d f.  The codes
// are therefore those of qm_quantize for v, independent of the order in which the squares are added.
#include "quant_device.cuh"

namespace qm {
namespace {

struct NormArgs {
  const void* x; int64_t ld_x;
  const void* res; int64_t ld_res;        // null: nothing is added
  void* res_out; int64_t ld_out;
  const void* w;
  float eps;
  int cols, ldc;
  uint8_t* codes;
  float* delta;
};

template <typename T> __device__ __forceinline__ float load_f(const T* p) { return (float)*p; }
template <typename T> __device__ __forceinline__ T round_to(float v) { return (T)v; }

template <typename T, typename W, int FMT>
__global__ void __launch_bounds__(kThreads) rms_norm_rows(const NormArgs a) {
  pdl_prologue();
  const int64_t row = blockIdx.x;
  const T* x = static_cast<const T*>(a.x) + row * a.ld_x;
  const T* r = static_cast<const T*>(a.res) + row * a.ld_res;
  T* z = static_cast<T*>(a.res_out) + row * a.ld_out;
  const W* w = static_cast<const W*>(a.w);
  float sum = 0.f;
  uint32_t top = 0;
  for (int c = threadIdx.x; c < a.cols; c += kThreads) {
    float s = load_f(x + c);
    if (a.res) {
      const T t = round_to<T>(s + load_f(r + c));
      z[c] = t;
      s = load_f(&t);
    }
    sum = fmaf(s, s, sum);
    top = max(top, absbits_f32(__float_as_uint(s * load_f(w + c))));
  }
  __shared__ float sums[kThreads / 32];
  __shared__ uint32_t tops[kThreads / 32];
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  top = __reduce_max_sync(0xffffffffu, top);
  if ((threadIdx.x & 31) == 0) { sums[threadIdx.x >> 5] = sum; tops[threadIdx.x >> 5] = top; }
  __syncthreads();
  sum = 0.f; top = 0;
  for (int i = 0; i < kThreads / 32; ++i) { sum += sums[i]; top = max(top, tops[i]); }
  const float own = top == 0 ? 1.f : __uint_as_float(top) / fmt_qmax(FMT);
  const float mean = sum / (float)a.cols;
  const bool finite = top < 0x7f800000u && mean < INFINITY;
  if (threadIdx.x == 0)
    a.delta[row] = !finite ? __int_as_float(0x7fffffff) : top == 0 ? 1.f : own * (1.f / sqrtf(mean + a.eps));
  const Quotient quot(own);
  const T* from = a.res ? z : x;
  uint8_t* codes = a.codes + row * a.ldc;
  for (int c = threadIdx.x; c < a.ldc; c += kThreads)
    codes[c] = c < a.cols && finite ? (uint8_t)quant2<FMT>(quot(load_f(from + c) * load_f(w + c)), 0.f) : (uint8_t)0;
}

template <typename T, typename W>
qm_status launch_fmt(const NormArgs& a, int64_t rows, int fmt, cudaStream_t s) {
  auto kern = fmt == QM_FMT_INT8 ? rms_norm_rows<T, W, QM_FMT_INT8>
            : fmt == QM_FMT_E4M3 ? rms_norm_rows<T, W, QM_FMT_E4M3> : rms_norm_rows<T, W, QM_FMT_E5M2>;
  QM_CUDA_OK(launch_pdl(kern, dim3((unsigned)rows), dim3(kThreads), 0, s, a));
  count_launch();
  return QM_OK;
}

}  // namespace

qm_status launch_rms_norm(const RowsView& x, const RowsView& residual, void* residual_out, int64_t ld_out,
                          const void* weight, int weight_dtype, float eps, int fmt, uint8_t* codes, float* delta,
                          cudaStream_t s) {
  NormArgs a{};
  a.x = x.data; a.ld_x = x.ld; a.res = residual.data; a.ld_res = residual.ld;
  a.res_out = residual_out; a.ld_out = ld_out; a.w = weight; a.eps = eps;
  a.cols = (int)x.cols; a.ldc = (int)qm_code_ld(x.cols); a.codes = codes; a.delta = delta;
  if (x.dtype == QM_DT_BF16)
    return weight_dtype == QM_DT_BF16 ? launch_fmt<__nv_bfloat16, __nv_bfloat16>(a, x.rows, fmt, s)
                                      : launch_fmt<__nv_bfloat16, float>(a, x.rows, fmt, s);
  return weight_dtype == QM_DT_BF16 ? launch_fmt<float, __nv_bfloat16>(a, x.rows, fmt, s)
                                    : launch_fmt<float, float>(a, x.rows, fmt, s);
}

}  // namespace qm
