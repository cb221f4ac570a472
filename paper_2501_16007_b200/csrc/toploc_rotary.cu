// Queries and keys between projection and attention: the RMS norm of every head and the rotation by position in one
// pass, keys and values straight to the paged cache.
#include "model_common.cuh"

namespace {

using namespace toploc_model;

constexpr int kWarps = 4;             // of a block
constexpr int kMostHeadDim = 256;
constexpr int kMostHalf = kMostHeadDim / 2;

struct Heads {  // one of queries, keys, values: where it is read and written
  const void* in;
  const void* weight;  // of its norm, or NULL
  void* out;
  long long in_token, in_head;
  long long out_page, out_token, out_head;  // (no pages: out_token counts tokens)
};

struct RotaryParams {
  Heads part[3];
  const int32_t* positions;
  const int64_t* slots;  // of keys and values, NULL: rows like the queries'
  const float* inv_freq;
  long long num_tokens, num_slots;
  float eps, per_channel;  // 1 / head_dim
  int head_dim, half;      // channels, turned pairs
  int q_heads, qk_heads, heads;  // ends of queries, of keys, of all
  int page_size;
  int lane_shift, lanes;   // a head is 2^lane_shift lanes, the first `lanes` of which have channels
  int steps, steps_per_warp;
};

// cos and sin of position * freq.  The angle is taken in turns and brought into one turn in 64 bits (position and frequency
// have 31 and 24 bits: nothing is lost before the product), so what remains in 32 is below 2^-25 turns off wherever the
// position is.
__device__ __forceinline__ float2 turn_of(int position, float freq) {
  double t = (double)position * (double)freq * 0.15915494309189533577;  // 1 / 2 pi
  t -= rint(t);
  float2 r;
  sincospif(2.f * (float)t, &r.y, &r.x);
  return r;
}

// Where a token's keys and values go: page and place in it.  false: nowhere.
__device__ __forceinline__ bool place_of(const RotaryParams& p, long long token, long long* page, long long* at) {
  if (!p.slots) {
    *page = 0, *at = token;
    return true;
  }
  const long long slot = p.slots[token];
  if (slot < 0 || slot >= p.num_slots) return false;
  if (slot <= 0xFFFFFFFFll) {  // a 32-bit division is several times as short
    *page = (unsigned)slot / (unsigned)p.page_size;
    *at = (unsigned)slot % (unsigned)p.page_size;
  } else {
    *page = slot / p.page_size;
    *at = slot - *page * p.page_size;
  }
  return true;
}

template <int kBytes>
struct Word;
template <>
struct Word<16> { using type = uint4; };
template <>
struct Word<8> { using type = uint2; };

template <typename T, int kVec>
using Packed = typename Word<sizeof(T) * kVec>::type;

template <typename T, int kVec>
__device__ __forceinline__ void unpack(const Packed<T, kVec>& q, float* v) {
  constexpr int kWords = sizeof(T) * kVec / 4;
  const uint32_t* w = reinterpret_cast<const uint32_t*>(&q);
#pragma unroll
  for (int i = 0; i < kWords; ++i) {
    if constexpr (sizeof(T) == 2)
      v[2 * i] = bf16_low(w[i]), v[2 * i + 1] = bf16_high(w[i]);
    else
      v[i] = __uint_as_float(w[i]);
  }
}

template <typename T, int kVec>
__device__ __forceinline__ Packed<T, kVec> pack(const float* v) {
  constexpr int kWords = sizeof(T) * kVec / 4;
  Packed<T, kVec> q;
  uint32_t* w = reinterpret_cast<uint32_t*>(&q);
#pragma unroll
  for (int i = 0; i < kWords; ++i) {
    if constexpr (sizeof(T) == 2)
      w[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
    else
      w[i] = __float_as_uint(v[i]);
  }
  return q;
}

// Bound by memory: every head is read once and written once.  A warp takes one token and some of its heads, 32 >> lane_shift
// heads a step.  A lane holds two vectors of a head, chosen so that turned channels meet in one lane: vector l and the one
// half the turned channels further on, or two neighbours; so the rotation needs no exchange, and the norm's sum a few
// shuffles.  The turns of a token are the same for all its heads: the warp works them out once (two a lane for 128
// channels) and every lane keeps its own in registers.
template <typename T, int kVec, bool kNeighbours, int kUnroll>
__global__ void __launch_bounds__(kWarps * 32) toploc_norm_rotary_kernel(const __grid_constant__ RotaryParams p) {
  __shared__ float2 turns[kWarps][kMostHalf];
  using Vector = Packed<T, kVec>;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long token = (long long)blockIdx.x * kWarps + warp;
  if (token >= p.num_tokens) return;
  const int width = 1 << p.lane_shift, l = lane & (width - 1);
  const int per_step = 32 >> p.lane_shift, sub = lane >> p.lane_shift;
  const bool has = l < p.lanes;
  const int half_vectors = p.half / kVec, turned_vectors = 2 * p.half / kVec;
  // the lane's two vectors of a head, and which of them turn
  int a, b;
  bool turn_a, turn_b;
  if constexpr (kNeighbours) {
    a = 2 * l, b = a + 1;
    turn_a = a < turned_vectors, turn_b = b < turned_vectors;
  } else {
    turn_a = turn_b = l < half_vectors;
    a = turn_a ? l : 2 * l;
    b = turn_a ? l + half_vectors : a + 1;
  }
  const int end = min(((int)blockIdx.y + 1) * p.steps_per_warp, p.steps);
  float cs[kVec], sn[kVec];
  bool turned = false;
  long long page = 0, at = 0;
  bool placed = false;
  for (int s0 = blockIdx.y * p.steps_per_warp; s0 < end; s0 += kUnroll) {
    Vector in_a[kUnroll], in_b[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int h = (s0 + u) * per_step + sub;
      in_a[u] = Vector{}, in_b[u] = Vector{};
      if (s0 + u < end && h < p.heads && has) {
        const Heads& w = p.part[h < p.q_heads ? 0 : h < p.qk_heads ? 1 : 2];
        const int first = h < p.q_heads ? 0 : h < p.qk_heads ? p.q_heads : p.qk_heads;
        const Vector* at_in =
            reinterpret_cast<const Vector*>(static_cast<const T*>(w.in) + token * w.in_token + (h - first) * w.in_head);
        in_a[u] = at_in[a], in_b[u] = at_in[b];
      }
    }
    if (!turned) {  // behind the first loads, in front of their use
      turned = true;
      const int position = p.half ? p.positions[token] : 0;
      for (int j = lane; j < p.half; j += 32) turns[warp][j] = turn_of(position, p.inv_freq[j]);
      placed = place_of(p, token, &page, &at);
      __syncwarp();
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const int j = l * kVec + e;
        const float2 t = j < p.half ? turns[warp][j] : make_float2(1.f, 0.f);
        cs[e] = t.x, sn[e] = t.y;
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (s0 + u >= end) break;
      const int h = (s0 + u) * per_step + sub;
      const int which = h < p.q_heads ? 0 : h < p.qk_heads ? 1 : 2;
      const int first = which == 0 ? 0 : which == 1 ? p.q_heads : p.qk_heads;
      const Heads& w = p.part[which];
      float x[kVec], y[kVec];
      unpack<T, kVec>(in_a[u], x);
      unpack<T, kVec>(in_b[u], y);
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < kVec; ++e) ss = fmaf(x[e], x[e], ss), ss = fmaf(y[e], y[e], ss);
      for (int off = width >> 1; off > 0; off >>= 1) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, off);
      if (h >= p.heads || !has) continue;
      if (which != 2) {
        if (w.weight) {
          const float r = rsqrtf(fmaf(ss, p.per_channel, p.eps));
          const Vector* weight = static_cast<const Vector*>(w.weight);
          float g[kVec];
          unpack<T, kVec>(__ldg(weight + a), g);
#pragma unroll
          for (int e = 0; e < kVec; ++e) x[e] = x[e] * r * g[e];
          unpack<T, kVec>(__ldg(weight + b), g);
#pragma unroll
          for (int e = 0; e < kVec; ++e) y[e] = y[e] * r * g[e];
        }
        if constexpr (kNeighbours) {
#pragma unroll
          for (int e = 0; e < kVec / 2; ++e) {
            const float u0 = x[2 * e], u1 = x[2 * e + 1], v0 = y[2 * e], v1 = y[2 * e + 1];
            const float c0 = cs[e], s0_ = sn[e], c1 = cs[kVec / 2 + e], s1 = sn[kVec / 2 + e];
            if (turn_a) x[2 * e] = u0 * c0 - u1 * s0_, x[2 * e + 1] = u0 * s0_ + u1 * c0;
            if (turn_b) y[2 * e] = v0 * c1 - v1 * s1, y[2 * e + 1] = v0 * s1 + v1 * c1;
          }
        } else if (turn_a) {
#pragma unroll
          for (int e = 0; e < kVec; ++e) {
            const float u0 = x[e], v0 = y[e];
            x[e] = u0 * cs[e] - v0 * sn[e];
            y[e] = u0 * sn[e] + v0 * cs[e];
          }
        }
        in_a[u] = pack<T, kVec>(x), in_b[u] = pack<T, kVec>(y);
      }
      if (which == 0 || placed) {
        T* out = static_cast<T*>(w.out) + (h - first) * w.out_head;
        out += which == 0 ? token * w.out_token : page * w.out_page + at * w.out_token;
        reinterpret_cast<Vector*>(out)[a] = in_a[u];
        reinterpret_cast<Vector*>(out)[b] = in_b[u];
      }
    }
  }
}

// Any layout: a warp per token and head, element by element, the head in shared memory between the passes.
template <typename T>
__global__ void __launch_bounds__(kWarps * 32) toploc_norm_rotary_any_kernel(const __grid_constant__ RotaryParams p,
                                                                            bool neighbours) {
  __shared__ float head[kWarps][kMostHeadDim];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long token = (long long)blockIdx.x * kWarps + warp;
  if (token >= p.num_tokens) return;
  const int h = blockIdx.y;
  const int which = h < p.q_heads ? 0 : h < p.qk_heads ? 1 : 2;
  const int first = which == 0 ? 0 : which == 1 ? p.q_heads : p.qk_heads;
  const Heads& w = p.part[which];
  const T* in = static_cast<const T*>(w.in) + token * w.in_token + (h - first) * w.in_head;
  T* out = static_cast<T*>(w.out) + (h - first) * w.out_head;
  if (which == 0) {
    out += token * w.out_token;
  } else {
    long long page, at;
    if (!place_of(p, token, &page, &at)) return;
    out += page * w.out_page + at * w.out_token;
  }
  if (which == 2) {
    for (int c = lane; c < p.head_dim; c += 32) out[c] = in[c];
    return;
  }
  float ss = 0.f;
  for (int c = lane; c < p.head_dim; c += 32) {
    const float v = to_float(in[c]);
    head[warp][c] = v;
    ss = fmaf(v, v, ss);
  }
  __syncwarp();
  if (w.weight) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, off);
    const float r = rsqrtf(fmaf(ss, p.per_channel, p.eps));
    for (int c = lane; c < p.head_dim; c += 32)
      head[warp][c] = head[warp][c] * r * to_float(static_cast<const T*>(w.weight)[c]);
    __syncwarp();
  }
  const int position = p.half ? p.positions[token] : 0;
  for (int c = lane; c < p.head_dim; c += 32) {
    float y = head[warp][c];
    if (c < 2 * p.half) {
      const bool second = neighbours ? c & 1 : c >= p.half;
      const int pair = neighbours ? c >> 1 : second ? c - p.half : c;
      const float other = head[warp][neighbours ? c ^ 1 : second ? c - p.half : c + p.half];
      const float2 t = turn_of(position, p.inv_freq[pair]);
      y = second ? other * t.y + y * t.x : y * t.x - other * t.y;
    }
    store_as(out + c, y);
  }
}

template <typename T, int kVec>
void launch_vectors(const RotaryParams& p, bool neighbours, dim3 grid, cudaStream_t stream) {
  constexpr int kUnroll = 4;
  if (neighbours)
    toploc_norm_rotary_kernel<T, kVec, true, kUnroll><<<grid, kWarps * 32, 0, stream>>>(p);
  else
    toploc_norm_rotary_kernel<T, kVec, false, kUnroll><<<grid, kWarps * 32, 0, stream>>>(p);
}

// Shape of the heads, the same for both entries.
int check_layout(const toploc_rotary_layout* lay) {
  if (!lay || lay->head_dim <= 0 || lay->q_heads <= 0 || lay->kv_heads <= 0 || lay->rotary_dim < 0 ||
      lay->rotary_dim > lay->head_dim || lay->rotary_dim % 2 != 0 || lay->num_tokens < 0 || !(lay->eps >= 0.f) ||
      (lay->pairing != TOPLOC_ROTARY_HALVES && lay->pairing != TOPLOC_ROTARY_NEIGHBOURS))
    return TOPLOC_ERR_INVALID_ARGUMENT;
  if (element_bytes(lay->dtype) == 0 || lay->head_dim > kMostHeadDim || lay->num_tokens > 0x7FFFFFFF ||
      lay->q_heads > 16384 || lay->kv_heads > 16384)
    return TOPLOC_ERR_UNSUPPORTED;
  return TOPLOC_OK;
}

// p.part, p.slots and the page fields are the caller's.
int run(RotaryParams& p, const toploc_rotary_layout* lay, const int32_t* positions, const float* inv_freq, int parts,
        cudaStream_t stream) {
  const int size = element_bytes(lay->dtype);
  if (lay->rotary_dim > 0 && (!positions || !inv_freq || !aligned(positions, 4) || !aligned(inv_freq, 4)))
    return TOPLOC_ERR_INVALID_ARGUMENT;
  for (int i = 0; i < parts; ++i) {
    const Heads& w = p.part[i];
    if (!w.in || !w.out || !aligned(w.in, size) || !aligned(w.out, size) || !aligned(w.weight, size) || w.in_token < 0 ||
        w.in_head < 0 || w.out_page < 0 || w.out_token < 0 || w.out_head < 0)
      return TOPLOC_ERR_INVALID_ARGUMENT;
  }
  int sms = 0;
  if (const int rc = check_device(&sms)) return rc;
  p.positions = positions;
  p.inv_freq = inv_freq;
  p.num_tokens = lay->num_tokens;
  p.eps = lay->eps;
  p.per_channel = 1.0f / (float)lay->head_dim;
  p.head_dim = lay->head_dim;
  p.half = lay->rotary_dim / 2;
  p.q_heads = lay->q_heads;
  p.qk_heads = lay->q_heads + lay->kv_heads;
  p.heads = parts == 3 ? p.qk_heads + lay->kv_heads : p.qk_heads;
  const bool neighbours = lay->pairing == TOPLOC_ROTARY_NEIGHBOURS;

  // whole vectors of `vec` elements everywhere: two a lane, turned channels in whole vectors
  const auto fits = [&](int vec) {
    const int bytes = vec * size;
    if (p.head_dim % (2 * vec) != 0 || (neighbours ? lay->rotary_dim : p.half) % vec != 0 || p.head_dim / (2 * vec) > 32)
      return false;
    for (int i = 0; i < parts; ++i) {
      const Heads& w = p.part[i];
      if (!aligned(w.in, bytes) || !aligned(w.out, bytes) || !aligned(w.weight, bytes)) return false;
      for (const long long s : {w.in_token, w.in_head, w.out_page, w.out_token, w.out_head})
        if (s % vec != 0) return false;
    }
    return true;
  };
  const int wide = 16 / size, vec = fits(wide) ? wide : size == 2 && fits(4) ? 4 : 0;
  const unsigned blocks = (unsigned)((p.num_tokens + kWarps - 1) / kWarps);
  if (vec == 0) {
    const dim3 grid(blocks, (unsigned)p.heads);
    if (size == 2)
      toploc_norm_rotary_any_kernel<__nv_bfloat16><<<grid, kWarps * 32, 0, stream>>>(p, neighbours);
    else
      toploc_norm_rotary_any_kernel<float><<<grid, kWarps * 32, 0, stream>>>(p, neighbours);
    return launched();
  }
  p.lanes = p.head_dim / (2 * vec);
  while (1 << p.lane_shift < p.lanes) ++p.lane_shift;
  const int per_step = 32 >> p.lane_shift;
  p.steps = (p.heads + per_step - 1) / per_step;
  // As many heads a warp as leave the SMs enough warps (48 each), so that few of them work the same turns out again.
  const long long split = min((long long)p.steps, max(1ll, 48ll * sms / p.num_tokens));
  p.steps_per_warp = (int)((p.steps + split - 1) / split);
  const dim3 grid(blocks, (unsigned)((p.steps + p.steps_per_warp - 1) / p.steps_per_warp));
  if (size == 4)
    launch_vectors<float, 4>(p, neighbours, grid, stream);
  else if (vec == 8)
    launch_vectors<__nv_bfloat16, 8>(p, neighbours, grid, stream);
  else
    launch_vectors<__nv_bfloat16, 4>(p, neighbours, grid, stream);
  return launched();
}

}  // namespace

extern "C" int toploc_norm_rotary_prompt(const void* d_q, const void* d_k, const int32_t* d_positions,
                                         const float* d_inv_freq, const void* d_q_weight_opt, const void* d_k_weight_opt,
                                         const toploc_rotary_layout* lay, void* d_q_out, void* d_k_out,
                                         void* cuda_stream) {
  if (const int rc = check_layout(lay)) return rc;
  if (lay->num_tokens == 0) return TOPLOC_OK;
  RotaryParams p = {};
  p.part[0] = {d_q, d_q_weight_opt, d_q_out, lay->q_token_stride, lay->q_head_stride, 0, lay->q_out_token_stride,
               lay->q_out_head_stride};
  p.part[1] = {d_k, d_k_weight_opt, d_k_out, lay->k_token_stride, lay->k_head_stride, 0, lay->k_out_token_stride,
               lay->k_out_head_stride};
  return run(p, lay, d_positions, d_inv_freq, 2, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" int toploc_norm_rotary_paged(const void* d_q, const void* d_k, const void* d_v, const int32_t* d_positions,
                                        const int64_t* d_slots, const float* d_inv_freq, const void* d_q_weight_opt,
                                        const void* d_k_weight_opt, const toploc_rotary_layout* lay, void* d_q_out,
                                        void* d_k_cache, void* d_v_cache, const toploc_kv_layout* kv,
                                        void* cuda_stream) {
  if (const int rc = check_layout(lay)) return rc;
  if (!kv || kv->page_size <= 0 || kv->num_pages < 0) return TOPLOC_ERR_INVALID_ARGUMENT;
  if (lay->num_tokens == 0) return TOPLOC_OK;
  if (!d_slots || !aligned(d_slots, 8)) return TOPLOC_ERR_INVALID_ARGUMENT;
  RotaryParams p = {};
  p.part[0] = {d_q, d_q_weight_opt, d_q_out, lay->q_token_stride, lay->q_head_stride, 0, lay->q_out_token_stride,
               lay->q_out_head_stride};
  p.part[1] = {d_k, d_k_weight_opt, d_k_cache, lay->k_token_stride, lay->k_head_stride, kv->k_page_stride,
               kv->k_token_stride, kv->k_head_stride};
  p.part[2] = {d_v, nullptr, d_v_cache, lay->v_token_stride, lay->v_head_stride, kv->v_page_stride, kv->v_token_stride,
               kv->v_head_stride};
  p.slots = d_slots;
  p.num_slots = (long long)kv->num_pages * kv->page_size;
  p.page_size = kv->page_size;
  return run(p, lay, d_positions, d_inv_freq, 3, static_cast<cudaStream_t>(cuda_stream));
}
