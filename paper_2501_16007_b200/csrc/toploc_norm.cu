// The residual addition with the RMS norm behind it, in 16, 32 or 8 bits.
#include "model_common.cuh"

#include <cuda_fp8.h>

namespace {

using namespace toploc_model;

constexpr float kE4m3Max = 448.0f;
constexpr float kSmallestScale = 1.17549435e-38f;  // 2^-126: a zero group divides by it and stores zeros

struct NormParams {
  const void* x;
  const void* residual;  // or NULL
  const void* weight;
  void* residual_out;  // or NULL
  void* y;
  float* scales;
  long long rows, x_stride, residual_stride, residual_out_stride, y_stride;
  float eps;
  int hidden, group, groups;
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, off);
  return v;
}

// max that keeps a NaN: a row with one gets a NaN scale, as the formula has it
__device__ __forceinline__ float max_nan(float a, float b) { return (a > b || a != a) ? a : b; }

__device__ __forceinline__ float warp_max_nan(float v) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v = max_nan(v, __shfl_xor_sync(0xFFFFFFFFu, v, off));
  return v;
}

__device__ __forceinline__ float scale_of(float amax) {
  const float s = __fdiv_rn(amax, kE4m3Max);
  return s < kSmallestScale ? kSmallestScale : s;
}

// A block per row, the row's h in shared memory between the two passes.
template <typename T, bool QUANT>
__global__ void __launch_bounds__(256) toploc_rmsnorm_residual_kernel(const NormParams p) {
  extern __shared__ float h[];
  __shared__ float partial[8];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long row = blockIdx.x;
  const T* x = static_cast<const T*>(p.x) + row * p.x_stride;
  const T* r = p.residual ? static_cast<const T*>(p.residual) + row * p.residual_stride : nullptr;
  T* ro = p.residual_out ? static_cast<T*>(p.residual_out) + row * p.residual_out_stride : nullptr;
  const T* w = static_cast<const T*>(p.weight);
  float ss = 0.f;
  for (int c = tid; c < p.hidden; c += 256) {
    float v = to_float(x[c]);
    if (r) v += to_float(r[c]);
    if (ro) store_as(ro + c, v);
    h[c] = v;
    ss = fmaf(v, v, ss);
  }
  ss = warp_sum(ss);
  if (lane == 0) partial[warp] = ss;
  __syncthreads();
  float total = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) total += partial[i];
  const float scale = rsqrtf(total / (float)p.hidden + p.eps);
  if constexpr (!QUANT) {
    T* y = static_cast<T*>(p.y) + row * p.y_stride;
    for (int c = tid; c < p.hidden; c += 256) store_as(y + c, h[c] * scale * to_float(w[c]));
  } else {
    __nv_fp8_e4m3* y = static_cast<__nv_fp8_e4m3*>(p.y) + row * p.y_stride;
    for (int g = warp; g < p.groups; g += 8) {  // a warp per group of channels
      const int begin = g * p.group, end = min(begin + p.group, p.hidden);
      float amax = 0.f;
      for (int c = begin + lane; c < end; c += 32) {
        const float v = h[c] * scale * to_float(w[c]);
        h[c] = v;
        amax = max_nan(fabsf(v), amax);
      }
      const float s = scale_of(warp_max_nan(amax));
      for (int c = begin + lane; c < end; c += 32) y[c] = __nv_fp8_e4m3(__fdiv_rn(h[c], s));
      if (lane == 0) p.scales[row * p.groups + g] = s;
    }
  }
}

template <typename T, bool QUANT>
int launch(const NormParams& p, cudaStream_t stream) {
  const size_t bytes = (size_t)p.hidden * 4;
  if (bytes > 40 * 1024 && cudaFuncSetAttribute(toploc_rmsnorm_residual_kernel<T, QUANT>,
                                                cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != cudaSuccess)
    return TOPLOC_ERR_CUDA;
  toploc_rmsnorm_residual_kernel<T, QUANT><<<(unsigned)p.rows, 256, bytes, stream>>>(p);
  return launched();
}

}  // namespace

extern "C" int toploc_rmsnorm_residual(const void* d_x, const void* d_residual_opt, const void* d_weight, float eps,
                                       const toploc_norm_layout* lay, void* d_residual_out_opt, void* d_y,
                                       float* d_scales_opt, void* cuda_stream) {
  if (!lay || lay->hidden <= 0 || lay->rows < 0 || lay->group < 0 || !(eps >= 0.f)) return TOPLOC_ERR_INVALID_ARGUMENT;
  const int size = element_bytes(lay->dtype);
  const bool quant = lay->out_kind == TOPLOC_NORM_OUT_E4M3;
  if (size == 0 || (!quant && lay->out_kind != TOPLOC_NORM_OUT_SAME) || lay->hidden > 49152 || lay->rows > 0x7FFFFFFF)
    return TOPLOC_ERR_UNSUPPORTED;
  if (lay->rows == 0) return TOPLOC_OK;
  if (!d_x || !d_weight || !d_y || (quant && !d_scales_opt)) return TOPLOC_ERR_INVALID_ARGUMENT;
  if (lay->x_stride < lay->hidden || lay->y_stride < lay->hidden ||
      (d_residual_opt && lay->residual_stride < lay->hidden) ||
      (d_residual_out_opt && lay->residual_out_stride < lay->hidden))
    return TOPLOC_ERR_INVALID_ARGUMENT;
  for (const void* q : {d_x, d_residual_opt, d_weight, (const void*)d_residual_out_opt})
    if (!aligned(q, size)) return TOPLOC_ERR_INVALID_ARGUMENT;
  if (!aligned(d_y, quant ? 1 : size) || (quant && !aligned(d_scales_opt, 4))) return TOPLOC_ERR_INVALID_ARGUMENT;
  if (const int rc = check_device()) return rc;
  NormParams p = {d_x, d_residual_opt, d_weight, d_residual_out_opt, d_y, d_scales_opt, lay->rows, lay->x_stride,
                  lay->residual_stride, lay->residual_out_stride, lay->y_stride, eps, lay->hidden, lay->group, 0};
  if (p.group == 0 || p.group > p.hidden) p.group = p.hidden;
  p.groups = (p.hidden + p.group - 1) / p.group;
  const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  if (lay->dtype == TOPLOC_DTYPE_BF16)
    return quant ? launch<__nv_bfloat16, true>(p, stream) : launch<__nv_bfloat16, false>(p, stream);
  return quant ? launch<float, true>(p, stream) : launch<float, false>(p, stream);
}
