// The residual addition with the RMS norm behind it, in 16, 32 or 8 bits.
#include "model_common.cuh"

#include <cuda_fp8.h>

namespace {

using namespace toploc_model;

constexpr int kMostHidden = 49152;  // channels of a row (its fp32 values fit shared memory)
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
  float eps, per_channel;  // 1 / hidden
  int hidden, group, groups;
  int group_shift;         // group = 2^group_shift accesses (groups of neighbouring lanes)
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, off);
  return v;
}

// max that keeps a NaN: a row with one gets a NaN scale, as the formula has it
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

__device__ __forceinline__ float warp_max_nan(float v) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v = max_nan(v, __shfl_xor_sync(0xFFFFFFFFu, v, off));
  return v;
}

__device__ __forceinline__ float reciprocal(float s) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
  return r;
}

__device__ __forceinline__ float scale_of(float amax) {
  const float s = amax * (1.0f / kE4m3Max);
  return s < kSmallestScale ? kSmallestScale : s;
}

// Bound by memory: x and residual are read once, residual_out and y written once.  A block takes a row and keeps it in
// registers between the two passes, 16 bytes an access where rows allow it.  What has to be in flight on an SM (50 KB and
// more) comes from its many threads, not from many values a thread: 16 values a thread and 32 registers (2048 threads an
// SM) take 618 to 633 us for 65536 x 8192 bf16 with e4m3 groups of 128 (6.0 to 6.1 TB/s; 663 on inputs that change from
// pass to pass), 32 values 715 us.  Rows that begin
// anywhere (an odd hidden size) move as vectors too where all tensors share the odd place (4095 x 5001 fp32: 62 us, 5.3
// TB/s; element by element 78 us, with 32 values a thread 135 us).  Where they do not (or 8 bits come out), single elements:
// 4096 x 12289 in fp32 154 us, 5.2 TB/s, to e4m3 152, bf16 133 and 154 (2.3 to 3.0 TB/s).
//
// kVec elements an access, kPer accesses a thread, access v of a row to thread v % threads.
enum Mode { kSame, kRowScale, kGroupScale };

template <typename T, int kVec>
__device__ __forceinline__ void load_values(const T* p, float* v) {
  if constexpr (kVec == 1) {
    v[0] = to_float(p[0]);
  } else {
    const uint4 q = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[2 * i] = bf16_low(w[i]), v[2 * i + 1] = bf16_high(w[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
    }
  }
}

template <typename T, int kVec>
__device__ __forceinline__ void store_values(T* p, const float* v) {
  if constexpr (kVec == 1) {
    store_as(p, v[0]);
  } else if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint4*>(p) =
        make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
  } else {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  }
}

template <int kVec>
__device__ __forceinline__ void store_e4m3(uint8_t* p, const float* v) {
  if constexpr (kVec == 1) {
    *p = __nv_cvt_float_to_fp8(v[0], __NV_SATFINITE, __NV_E4M3);
  } else {
    uint32_t w[kVec / 4];
#pragma unroll
    for (int i = 0; i < kVec / 4; ++i)
      w[i] = __nv_cvt_float2_to_fp8x2(make_float2(v[4 * i], v[4 * i + 1]), __NV_SATFINITE, __NV_E4M3) |
             (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(v[4 * i + 2], v[4 * i + 3]), __NV_SATFINITE, __NV_E4M3) << 16;
    if constexpr (kVec == 4)
      *reinterpret_cast<uint32_t*>(p) = w[0];
    else
      *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  }
}

// Access of kVec elements from c on of a row of `hidden`, which may begin in front of the row or end behind it (kShift).
template <typename T, int kVec, bool kShift>
__device__ __forceinline__ void load_part(const T* p, int c, int hidden, float* v) {
  if (!kShift || (c >= 0 && c + kVec <= hidden)) {
    load_values<T, kVec>(p + c, v);
  } else {
#pragma unroll
    for (int e = 0; e < kVec; ++e) v[e] = c + e >= 0 && c + e < hidden ? to_float(p[c + e]) : 0.f;
  }
}

template <typename T, int kVec, bool kShift>
__device__ __forceinline__ void store_part(T* p, int c, int hidden, const float* v) {
  if (!kShift || (c >= 0 && c + kVec <= hidden)) {
    store_values<T, kVec>(p + c, v);
  } else {
#pragma unroll
    for (int e = 0; e < kVec; ++e)
      if (c + e >= 0 && c + e < hidden) store_as(p + c + e, v[e]);
  }
}

// kShift: rows that do not begin at a vector's place, but all tensors' rows at the same distance from one: the accesses
// are laid from that place on, the first and the last partly outside (the weights, whose rows begin elsewhere, are read
// element by element).
template <typename T, int kVec, int kPer, Mode kMode, bool kShift>
__global__ void __launch_bounds__(kVec > 1 ? 512 : 1024,
                                  kVec * kPer > 16 ? 1 : kShift ? 2 : kVec > 1 ? 4 : kPer <= 5 ? 2 : 1)
    toploc_rmsnorm_rows_kernel(const NormParams p) {
  __shared__ float partial[32], partial_max[32];
  // (a constant where a thread has many accesses: their places then differ by constants, and nothing spills)
  const int threads = kPer > 8 ? 1024 : blockDim.x;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = threads >> 5;
  const long long row = blockIdx.x;
  const T* x = static_cast<const T*>(p.x) + row * p.x_stride;
  const T* r = static_cast<const T*>(p.residual) + row * p.residual_stride;
  T* ro = static_cast<T*>(p.residual_out) + row * p.residual_out_stride;
  const T* w = static_cast<const T*>(p.weight);
  // elements in front of the row in its first access
  const int shift = kShift ? (int)((reinterpret_cast<uintptr_t>(x) / sizeof(T)) % kVec) : 0;
  float h[kPer][kVec];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int c = (tid + i * threads) * kVec - shift;
#pragma unroll
    for (int e = 0; e < kVec; ++e) h[i][e] = 0.f;
    if (c < p.hidden) load_part<T, kVec, kShift>(x, c, p.hidden, h[i]);
  }
  if (p.residual) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int c = (tid + i * threads) * kVec - shift;
      if (c < p.hidden) {
        float v[kVec];
        load_part<T, kVec, kShift>(r, c, p.hidden, v);
#pragma unroll
        for (int e = 0; e < kVec; ++e) h[i][e] += v[e];
      }
    }
  }
  float ss = 0.f;
#pragma unroll
  for (int i = 0; i < kPer; ++i)
#pragma unroll
    for (int e = 0; e < kVec; ++e) ss = fmaf(h[i][e], h[i][e], ss);
  ss = warp_sum(ss);
  if (lane == 0) partial[warp] = ss;
  if (p.residual_out) {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int c = (tid + i * threads) * kVec - shift;
      if (c < p.hidden) store_part<T, kVec, kShift>(ro, c, p.hidden, h[i]);
    }
  }
  __syncthreads();
  float total = warp_sum(lane < warps ? partial[lane] : 0.f);
  const float scale = rsqrtf(fmaf(total, p.per_channel, p.eps));
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int c = (tid + i * threads) * kVec - shift;
    if (c < p.hidden) {
      float v[kVec];
      if constexpr (kShift) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) v[e] = c + e >= 0 && c + e < p.hidden ? to_float(w[c + e]) : 0.f;
      } else {
        load_values<T, kVec>(w + c, v);
      }
#pragma unroll
      for (int e = 0; e < kVec; ++e) h[i][e] = h[i][e] * scale * v[e];
    }
  }
  if constexpr (kMode == kSame) {
    T* y = static_cast<T*>(p.y) + row * p.y_stride;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int c = (tid + i * threads) * kVec - shift;
      if (c < p.hidden) store_part<T, kVec, kShift>(y, c, p.hidden, h[i]);
    }
  } else {
    uint8_t* y = static_cast<uint8_t*>(p.y) + row * p.y_stride;
    float amax[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      amax[i] = 0.f;
#pragma unroll
      for (int e = 0; e < kVec; ++e) amax[i] = max_nan(fabsf(h[i][e]), amax[i]);
    }
    float row_scale = 0.f;
    if constexpr (kMode == kRowScale) {
      float top = amax[0];
#pragma unroll
      for (int i = 1; i < kPer; ++i) top = max_nan(amax[i], top);
      top = warp_max_nan(top);
      if (lane == 0) partial_max[warp] = top;
      __syncthreads();
      row_scale = scale_of(warp_max_nan(lane < warps ? partial_max[lane] : 0.f));
      if (tid == 0) p.scales[row] = row_scale;
    }
    if constexpr (kMode == kGroupScale) {  // a group is the accesses of neighbouring lanes (2^n of them)
      for (int off = 1 << p.group_shift >> 1; off > 0; off >>= 1) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) amax[i] = max_nan(amax[i], __shfl_xor_sync(0xFFFFFFFFu, amax[i], off));
      }
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int v = tid + i * threads, c = v * kVec;
      float s = row_scale;
      if constexpr (kMode == kGroupScale) {
        s = scale_of(amax[i]);
        if (c < p.hidden && (v & ((1 << p.group_shift) - 1)) == 0) p.scales[row * p.groups + (v >> p.group_shift)] = s;
      }
      // y / s as y * (1 / s): off by an fp32 rounding or two, which moves an e4m3 result only next to the middle of two (17 of
      // a million, by the same arithmetic on the CPU; y's own roundings move as many, whichever way it is divided)
      const float inv = reciprocal(s);
#pragma unroll
      for (int e = 0; e < kVec; ++e) h[i][e] *= inv;
      if (c < p.hidden) store_e4m3<kVec>(y + c, h[i]);
    }
  }
}

// Any hidden size, layout and group: a block per row, the row's h in shared memory between the two passes.
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
  const float scale = rsqrtf(fmaf(total, p.per_channel, p.eps));
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
      const float s = scale_of(warp_max_nan(amax)), inv = reciprocal(s);
      for (int c = begin + lane; c < end; c += 32) y[c] = __nv_fp8_e4m3(h[c] * inv);
      if (lane == 0) p.scales[row * p.groups + g] = s;
    }
  }
}

template <typename T, bool QUANT>
int launch_any(const NormParams& p, cudaStream_t stream) {
  const size_t bytes = (size_t)p.hidden * 4;
  static std::atomic<uint64_t> allowed{0};
  if (const int rc = allow_shared(reinterpret_cast<const void*>(toploc_rmsnorm_residual_kernel<T, QUANT>), kMostHidden * 4,
                                  allowed))
    return rc;
  toploc_rmsnorm_residual_kernel<T, QUANT><<<(unsigned)p.rows, 256, bytes, stream>>>(p);
  return launched();
}

template <typename T, int kVec, int kPer>
int launch_rows(const NormParams& p, Mode mode, bool shifted, int threads, cudaStream_t stream) {
  const unsigned rows = (unsigned)p.rows;
  if (kVec > 1 && shifted)
    toploc_rmsnorm_rows_kernel<T, kVec, kPer, kSame, (kVec > 1)><<<rows, threads, 0, stream>>>(p);
  else if (mode == kSame)
    toploc_rmsnorm_rows_kernel<T, kVec, kPer, kSame, false><<<rows, threads, 0, stream>>>(p);
  else if (mode == kRowScale)
    toploc_rmsnorm_rows_kernel<T, kVec, kPer, kRowScale, false><<<rows, threads, 0, stream>>>(p);
  else
    toploc_rmsnorm_rows_kernel<T, kVec, kPer, kGroupScale, false><<<rows, threads, 0, stream>>>(p);
  return launched();
}

// The row in registers where it fits 512 threads of 32 values, or 1024 of 16 single ones (and a group's lanes are
// neighbours), else in shared memory.
template <typename T>
int launch(NormParams& p, bool quant, bool vectors, bool shifted, cudaStream_t stream) {
  constexpr int kWide = 16 / sizeof(T);
  const int vec = vectors || shifted ? kWide : 1, accesses = (p.hidden + (shifted ? vec - 1 : 0) + vec - 1) / vec;
  const Mode mode = !quant ? kSame : p.groups == 1 ? kRowScale : kGroupScale;
  const int lanes = p.group / vec;  // of a group
  const bool fits = accesses <= 512 * (32 / vec) &&
                    (mode != kGroupScale || (p.group % vec == 0 && lanes <= 32 && (lanes & (lanes - 1)) == 0));
  if (!fits) return quant ? launch_any<T, true>(p, stream) : launch_any<T, false>(p, stream);
  while (1 << p.group_shift < lanes && p.group_shift < 5) ++p.group_shift;
  int per = 1;
  if (vec > 1) {
    while (per * 512 < accesses) per *= 2;
  } else {
    for (const int more : {2, 3, 5, 8, 16})
      if (per * 1024 < accesses) per = more;
  }
  const int threads = per > 8 ? 1024 : ((accesses + per - 1) / per + 31) / 32 * 32;
  if (vec > 1) {
    switch (per) {
      case 1: return launch_rows<T, kWide, 1>(p, mode, shifted, threads, stream);
      case 2: return launch_rows<T, kWide, 2>(p, mode, shifted, threads, stream);
      case 4: return launch_rows<T, kWide, 4>(p, mode, shifted, threads, stream);
      default: return launch_rows<T, kWide, 32 / kWide>(p, mode, shifted, threads, stream);
    }
  }
  switch (per) {
    case 1: return launch_rows<T, 1, 1>(p, mode, shifted, threads, stream);
    case 2: return launch_rows<T, 1, 2>(p, mode, shifted, threads, stream);
    case 3: return launch_rows<T, 1, 3>(p, mode, shifted, threads, stream);
    case 5: return launch_rows<T, 1, 5>(p, mode, shifted, threads, stream);
    case 8: return launch_rows<T, 1, 8>(p, mode, shifted, threads, stream);
    default: return launch_rows<T, 1, 16>(p, mode, shifted, threads, stream);
  }
}

}  // namespace

extern "C" int toploc_rmsnorm_residual(const void* d_x, const void* d_residual_opt, const void* d_weight, float eps,
                                       const toploc_norm_layout* lay, void* d_residual_out_opt, void* d_y,
                                       float* d_scales_opt, void* cuda_stream) {
  if (!lay || lay->hidden <= 0 || lay->rows < 0 || lay->group < 0 || !(eps >= 0.f)) return TOPLOC_ERR_INVALID_ARGUMENT;
  const int size = element_bytes(lay->dtype);
  const bool quant = lay->out_kind == TOPLOC_NORM_OUT_E4M3;
  if (size == 0 || (!quant && lay->out_kind != TOPLOC_NORM_OUT_SAME) || lay->hidden > kMostHidden || lay->rows > 0x7FFFFFFF)
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
                  lay->residual_stride, lay->residual_out_stride, lay->y_stride, eps, 1.0f / (float)lay->hidden, lay->hidden,
                  lay->group, 0, 0};
  if (p.group == 0 || p.group > p.hidden) p.group = p.hidden;
  p.groups = (p.hidden + p.group - 1) / p.group;
  const int64_t per = 16 / size;
  bool vectors = p.hidden % per == 0 && p.x_stride % per == 0 && aligned(d_x, 16) && aligned(d_weight, 16) &&
                 p.y_stride % per == 0 && aligned(d_y, quant ? per : 16);
  if (d_residual_opt) vectors = vectors && p.residual_stride % per == 0 && aligned(d_residual_opt, 16);
  if (d_residual_out_opt) vectors = vectors && p.residual_out_stride % per == 0 && aligned(d_residual_out_opt, 16);
  const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  // rows that begin anywhere, but all tensors' rows at the same distance from a vector's place (one unaligned stride)
  const auto away = [&](const void* at, int64_t stride) {
    return !at || (reinterpret_cast<uintptr_t>(at) % 16 == reinterpret_cast<uintptr_t>(d_x) % 16 &&
                   (stride - p.x_stride) % per == 0);
  };
  const bool shifted = !vectors && !quant && p.hidden >= 256 && away(d_residual_opt, p.residual_stride) &&
                       away(d_residual_out_opt, p.residual_out_stride) && away(d_y, p.y_stride);
  return lay->dtype == TOPLOC_DTYPE_BF16 ? launch<__nv_bfloat16>(p, quant, vectors, shifted, stream)
                                         : launch<float>(p, quant, vectors, shifted, stream);
}
