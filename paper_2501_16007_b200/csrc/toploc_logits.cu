// Rows of logits: log probability of a given token, entropy, the likeliest alternatives, in one pass over them.
//
// The sums are kept in base 2 against a reference c that follows the maximum loosely: with y_j = x_j log2 e - c,
//   s = sum 2^y_j,  w = sum 2^y_j y_j;  lse = (c + log2 s) ln 2,  entropy = (log2 s - w / s) ln 2.
// c is renewed only when a value passes it by 2^8, so a few times a thread and not with every new maximum (it costs precision
// too: y_j is off by half a step, 2^-22 just below 2^3).
//
// Bound by memory (one pass), with the powers, 16 a cycle and SM, not far behind: 4097 x 128000 bf16 takes 162 us without
// alternatives (6.5 TB/s; the powers alone 130) and 171 with five; in long runs, where the board's power brings the clock down
// to 1.6 GHz, 189.  What counts is many warps with many independent operations each: 40 warps an SM (48 registers) and four
// vectors a thread at a time.  Copies ahead through shared memory or registers, which cost warps, took 205 to 255 us.
//
// Alternatives: while it streams, a block leaves the largest of every four vectors (32 or 16 logits) in shared memory.  The
// four largest of each warp's threads' maxima give a bound that at least `top` logits reach; behind the row only the vectors
// that reach it are read again, a few dozen, and their logits ranked by (value, index).  Where fewer than top / 4 warps have any
// candidates there is no bound, and with more than 256 of them one warp takes them in order (best_in_order).
#include "model_common.cuh"

#include <cooperative_groups.h>

#include <cfloat>
#include <utility>

namespace {

using namespace toploc_model;
namespace cg = cooperative_groups;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
// Of an SM: with fp32 there is half as much to compute a byte, and 64 registers a thread do more for it than a fifth block
// (1000 x 50257, on one board: 35.6 us against 37.9; bf16, 4097 x 128000: 188 against 172).
template <typename T>
constexpr int kBlocksPerSm = sizeof(T) == 2 ? 5 : 4;
constexpr int kMostVocab = 1 << 20;
constexpr int kMostTop = TOPLOC_MAX_ALTERNATIVES;
constexpr int kMostCluster = 8;       // blocks that share a row
constexpr int kMaximaBytes = 32768;   // of shared memory that the maxima of a block take, as a rule (five blocks fit an SM)
constexpr int kBatch = 4;             // vectors of a thread that are loaded together, and whose largest logit is kept
constexpr int kMostBatches = 256;     // threads' batches, and logits in them, that reach the bound; more take the ordered way
constexpr int kMostKeys = 256;
static_assert(kMostKeys >= kThreads && kMostCluster * kMostTop <= kThreads, "a thread for each of a row's candidates");
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kSlack = 8.f;         // powers of 2 that a value may pass the reference by
constexpr float kNothing = 60.f;      // powers of 2 below the reference: 2^20 such logits are nothing in a sum of 24 bits
// The reference is off its logit by half a step of its own, a power of 2 at kSums and more than fp32 has powers a little further
// on.  So rows whose maximum is out of +-kFar are summed again by differences from it.  In other rows nothing below -kSums has
// any weight: such parts' sums are left out, and logits below kTiny count as kTiny.
constexpr float kFar = 1e7f, kSums = 2e7f, kTiny = -3e7f;
constexpr float kNoReference = -4e7f;   // above kTiny log2 e: weight 0 for what a thread meets before its first reference
constexpr float kLeast = -1e30f;        // powers of 2 that differences count as at least

struct LogitParams {
  const void* logits;
  const int64_t* tokens;  // or NULL
  float* logprobs;
  float* entropy;         // or NULL
  int64_t* top_ids;
  float* top_logprobs;
  long long stride;
  int vocab, top;
};

// Some of a row: its largest logit, and the sums against it.
struct Part {
  float top, s, w;
};

// A whole row: what log probabilities are made of.
struct Whole {
  float top, s, w, log2_s;
};

struct Shared {
  Part of_warp[kWarps];
  unsigned warp_best[kWarps * 4];        // each warp's four largest thread maxima
  Part part;
  Whole whole;
  float bound;
  int num_batches, num_keys;
  unsigned long long best[kMostTop];     // the block's alternatives
  unsigned batches[kMostBatches];
  unsigned long long keys[kMostKeys];
};

__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// A logit in powers of 2 as a reference has it: rounded by itself, never as part of a sum (all that is taken off a reference
// has to take off the same number).
__device__ __forceinline__ float powers_of(float x) { return __fmul_rn(x, kLog2e); }

// max that keeps a NaN
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// A number that orders like the value (-0 and 0 alike).
__device__ __forceinline__ unsigned ordered(float v) {
  const unsigned b = __float_as_uint(v + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned o) {
  return __uint_as_float(o & 0x80000000u ? o & 0x7FFFFFFFu : ~o);
}
// Larger value first, then smaller index; 0: nobody.
__device__ __forceinline__ unsigned long long key_of(float v, int index) {
  return (unsigned long long)ordered(v) << 32 | (0xFFFFFFFFu - (unsigned)index);
}

// 16 bytes of logits.
template <typename T>
struct Vector;
template <>
struct Vector<__nv_bfloat16> {
  static constexpr int kSize = 8;
  using Kept = uint16_t;  // a maximum in shared memory
  static constexpr uint32_t kNothing = 0xFF80FF80u;  // -inf twice
  // The larger two of two; a NaN wins, or is passed over.
  template <bool kNaN>
  static __device__ uint32_t larger(uint32_t a, uint32_t b) {
    const __nv_bfloat162 x = *reinterpret_cast<__nv_bfloat162*>(&a), y = *reinterpret_cast<__nv_bfloat162*>(&b);
    const __nv_bfloat162 m = kNaN ? __hmax2_nan(x, y) : __hmax2(x, y);
    return *reinterpret_cast<const uint32_t*>(&m);
  }
  template <bool kNaN>
  static __device__ float largest(const uint4* q) {
    uint32_t m = 0xFF80FF80u;
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      m = larger<kNaN>(m, larger<kNaN>(larger<kNaN>(q[i].x, q[i].y), larger<kNaN>(q[i].z, q[i].w)));
    return kNaN ? max_nan(bf16_low(m), bf16_high(m)) : fmaxf(bf16_low(m), bf16_high(m));
  }
  static __device__ void floored(const uint4& q, Pair* v) {  // no smaller than kTiny; NaN stays
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    const __nv_bfloat162 tiny = __float2bfloat162_rn(kTiny);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 f = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&w[i]), tiny);
      const uint32_t u = *reinterpret_cast<const uint32_t*>(&f);
      v[i] = pair_of(bf16_low(u), bf16_high(u));
    }
  }
  static __device__ Kept kept(float m) { return (Kept)(__float_as_uint(m) >> 16); }  // (exact: it was one)
  static __device__ float value(Kept m) { return __uint_as_float((uint32_t)m << 16); }
};
template <>
struct Vector<float> {
  static constexpr int kSize = 4;
  using Kept = float;
  static constexpr uint32_t kNothing = 0xFF800000u;
  static __device__ float of(uint32_t w) { return __uint_as_float(w); }
  template <bool kNaN>
  static __device__ float larger(float a, float b) { return kNaN ? max_nan(a, b) : fmaxf(a, b); }
  template <bool kNaN>
  static __device__ float largest(const uint4* q) {
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      m = larger<kNaN>(m, larger<kNaN>(larger<kNaN>(of(q[i].x), of(q[i].y)), larger<kNaN>(of(q[i].z), of(q[i].w))));
    return m;
  }
  static __device__ void floored(const uint4& q, Pair* v) {
    v[0] = pair_of(max_nan(of(q.x), kTiny), max_nan(of(q.y), kTiny));
    v[1] = pair_of(max_nan(of(q.z), kTiny), max_nan(of(q.w), kTiny));
  }
  static __device__ Kept kept(float m) { return m; }
  static __device__ float value(Kept m) { return m; }
};

// A thread's sums, even and odd values apart.
struct Sums {
  float c = kNoReference, top = -INFINITY;
  Pair s2 = 0, w2 = 0;

  __device__ __forceinline__ float s() const { return both(s2).x + both(s2).y; }
  __device__ __forceinline__ float w() const { return both(w2).x + both(w2).y; }
  __device__ __forceinline__ void renew(float reference) {  // rare
    const float f = exp2_fast(c - reference), d = c - reference;
    const float2 s = both(s2), w = both(w2);
    w2 = f > 0.f ? pair_of(f * fmaf(d, s.x, w.x), f * fmaf(d, s.y, w.y)) : 0;
    s2 = pair_of(f * s.x, f * s.y);
    c = reference;
  }
  // In front of values up to `largest`.
  __device__ __forceinline__ void meet(float largest) {
    top = fmaxf(top, largest);
    if (powers_of(largest) > c + kSlack) renew(powers_of(largest));
  }
  // Floored values, kPairs times two.  They are added up among themselves first: a thread's sums then have so many fewer
  // roundings in a row.
  template <int kPairs>
  __device__ __forceinline__ void add(const Pair* v) {
    const Pair scale = pair_of(kLog2e, kLog2e), minus = pair_of(-c, -c);
    Pair y[kPairs], e[kPairs];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
      y[i] = fma2(v[i], scale, minus);
      const float2 q = both(y[i]);
      e[i] = pair_of(exp2_fast(q.x), exp2_fast(q.y));
    }
    Pair w = mul2(e[0], y[0]);
#pragma unroll
    for (int i = 1; i < kPairs; ++i) w = fma2(e[i], y[i], w);
    w2 = add2(w2, w);
#pragma unroll
    for (int n = kPairs / 2; n > 0; n /= 2)
#pragma unroll
      for (int i = 0; i < n; ++i) e[i] = add2(e[i], e[i + n]);
    s2 = add2(s2, e[0]);
  }
};

// A block's share of a row: vectors at 16-byte places, the first `shift` logits of which lie in front of the row.
template <typename T>
struct Share {
  static constexpr int kSize = Vector<T>::kSize;
  const T* at;  // the row
  int shift, vocab, begin, end;
  int inner, inner_end;  // vectors that lie in the row as a whole

  __device__ __forceinline__ Share(const LogitParams& p, long long r, int rank, int blocks) {
    at = static_cast<const T*>(p.logits) + r * p.stride;
    vocab = p.vocab;
    shift = (int)(reinterpret_cast<uintptr_t>(at) % 16 / sizeof(T));
    const int all = (vocab + shift + kSize - 1) / kSize, each = (all + blocks - 1) / blocks;
    begin = min(rank * each, all);
    end = min(begin + each, all);
    inner = begin == 0 && shift > 0 ? 1 : begin;
    inner_end = end == all && (vocab + shift) % kSize != 0 ? end - 1 : end;
  }
  // (an empty share has one batch, of nothing)
  __device__ __forceinline__ int batches() const { return max(1, (end - begin + kBatch * kThreads - 1) / (kBatch * kThreads)); }
  // vector i of a thread's batch
  __device__ __forceinline__ int vector(int batch, int thread, int i) const {
    return begin + (kBatch * batch + i) * kThreads + thread;
  }
  __device__ __forceinline__ int first(int v) const { return v * kSize - shift; }
  __device__ __forceinline__ bool in_row(int v, int e) const { return v < end && first(v) + e >= 0 && first(v) + e < vocab; }
  __device__ __forceinline__ float value(int v, int e) const { return in_row(v, e) ? to_float(at[first(v) + e]) : -INFINITY; }
};

// A vector: what lies outside the row is -inf, so that nothing behind has to look.
template <typename T>
__device__ __forceinline__ uint4 fetch(const Share<T>& row, int v) {
  if (v >= row.inner && v < row.inner_end) return __ldcs(reinterpret_cast<const uint4*>(row.at + row.first(v)));
  constexpr uint32_t kNothing = Vector<T>::kNothing;
  uint4 q = make_uint4(kNothing, kNothing, kNothing, kNothing);
  if (v < row.end) {  // the row begins or ends inside it
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 2)
        w[i] = pack_bf16(row.value(v, 2 * i), row.value(v, 2 * i + 1));
      else
        w[i] = __float_as_uint(row.value(v, i));
    }
    q = make_uint4(w[0], w[1], w[2], w[3]);
  }
  return q;
}

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, off));
  return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, off);
  return v;
}

// Numbers of the lanes that go up and down once (or down and up) in descending order; ascending with flip 31 (the lanes'
// numbers read backwards).  The first exchange is with the lane `from` away.
__device__ __forceinline__ void warp_merge(unsigned& v, int from, int flip) {
  const int lane = (threadIdx.x & 31) ^ flip;
#pragma unroll
  for (int j = 16; j > 0; j >>= 1) {
    if (j > from) continue;
    const unsigned other = __shfl_xor_sync(0xFFFFFFFFu, v, j);
    v = (lane & j) == 0 ? max(v, other) : min(v, other);
  }
}
__device__ __forceinline__ void warp_sort(unsigned& v, int flip) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int k = 1; k <= 16; k <<= 1)  // runs of 2 k, every other one the other way round
    warp_merge(v, k, flip ^ (k < 16 && (((lane ^ flip) & (2 * k)) != 0) ? 31 : 0));
}

__device__ __forceinline__ bool is_far(float top) { return top > -INFINITY && !(fabsf(top) < kFar); }

// A row, or a block's share, from its parts in lanes 0 .. count - 1, for all lanes of the warp.  Parts whose maximum is out of
// +-kSums have sums of 0 (or of NaN); in a far row all have been summed again against its maximum.
__device__ __forceinline__ Part join_parts(Part q, int count) {
  const int lane = threadIdx.x & 31;
  if (lane >= count) q = {-INFINITY, 0.f, 0.f};
  const float top = warp_max(q.top);
  const float d = fabsf(top) < kSums && fabsf(q.top) < kSums ? powers_of(q.top) - powers_of(top) : 0.f, f = exp2_fast(d);
  return {top, warp_sum(f * q.s), warp_sum(f > 0.f ? f * fmaf(d, q.s, q.w) : f * q.s)};
}

// (The sums' roundings leave up to 8e-8 of the wrong sign where one token has nearly all the weight: the largest term is 2 to
// the reference's own rounding, and log2 s gives that back only to a rounding.  A caller's log1p(-exp(logprob)) and sqrt(entropy)
// would be NaN, so both are held to their range.)
__device__ __forceinline__ float logprob_of(const Whole& row, float x) {
  if (row.s != row.s) return row.s;
  if (x == -INFINITY || row.top == -INFINITY) return -INFINITY;
  // in powers of 2, so that the sums' own reference cancels to the bit, but for a far row, whose sums are against the maximum
  // itself, and where the product with log2 e could leave fp32
  if (fabsf(row.top) < kFar && x > kLeast) return fminf((fmaf(x, kLog2e, -powers_of(row.top)) - row.log2_s) * kLn2, 0.f);
  return fminf(x - row.top - row.log2_s * kLn2, 0.f);
}

__device__ __forceinline__ void write_row(const LogitParams& p, long long r, const Whole& row, bool known, float given) {
  if (p.tokens) p.logprobs[r] = known ? logprob_of(row, given) : __uint_as_float(0x7FFFFFFFu);
  if (p.entropy) p.entropy[r] = row.top == -INFINITY && row.s == row.s ? 0.f : max_nan((row.log2_s - row.w / row.s) * kLn2, 0.f);
}

// The block's alternatives one after the other, where more candidates reach the bound than there is room for: many equal logits,
// or no bound, because the candidates lie in fewer than top / 4 warps (rows of 257 to 1816 logits by number of alternatives and
// type, a mask that leaves some hundred neighbours, or anything but the type's lowest value).  Through the vectors in order, the
// best so far in a warp's lanes; what only equals the least of a full list is passed over, so long runs of equal logits cost a
// look at their maxima.  64 x 1000 bf16, 20 alternatives: 94 us (with 5, by the bound, 4.6); 64 x 128000 all equal: 40.
template <typename T>
__device__ __noinline__ unsigned long long best_in_order(const Share<T> row, const typename Vector<T>::Kept* maxima, float bound,
                                                         int top) {
  const int lane = threadIdx.x & 31;
  unsigned long long mine = 0;  // lane i: the i-th best
  float least = bound;          // to be reached, and passed once the list is full (equal ones later lose)
  bool full = false;
  for (int n = 0; n < row.batches() * kBatch * kWarps; ++n) {  // 32 vectors
    const int batch = n / (kBatch * kWarps), i = n / kWarps % kBatch, thread = n % kWarps * 32;
    const float m = Vector<T>::value(maxima[batch * kThreads + thread + lane]);
    unsigned hits = __ballot_sync(0xFFFFFFFFu, m > -INFINITY && (full ? m > least : m >= least));
    while (hits) {
      const int v = row.vector(batch, thread + __ffs(hits) - 1, i);
      hits &= hits - 1;
      unsigned long long key = 0;
      if (lane < Vector<T>::kSize) {
        const float x = row.value(v, lane);
        if (x > -INFINITY) key = key_of(x, row.first(v) + lane);
      }
#pragma unroll 1
      for (int e = 0; e < Vector<T>::kSize; ++e) {
        const unsigned long long k = __shfl_sync(0xFFFFFFFFu, key, e);
        const int place = __popc(__ballot_sync(0xFFFFFFFFu, lane < top && mine > k));
        if (k == 0 || place >= top) continue;
        const unsigned long long up = __shfl_up_sync(0xFFFFFFFFu, mine, 1);
        if (lane > place) mine = up;
        if (lane == place) mine = k;
        if (lane >= top) mine = 0;
      }
      const unsigned long long last = __shfl_sync(0xFFFFFFFFu, mine, top - 1);
      if (last != 0) full = true, least = value_of((unsigned)(last >> 32));
    }
  }
  return mine;
}

// Logits of the block's share that reach sh.bound to sh.keys; false where there is no room (sh.best has them then).
template <typename T>
__device__ __forceinline__ bool gather_keys(Shared& sh, const Share<T>& row, const typename Vector<T>::Kept* maxima, int top) {
  using Kept = typename Vector<T>::Kept;
  const int tid = threadIdx.x;
  const float bound = sh.bound;  // (above -inf)
  constexpr int kAtOnce = 16 / sizeof(Kept), kSize = Vector<T>::kSize;
  for (int i0 = tid * kAtOnce; i0 < row.batches() * kThreads; i0 += kThreads * kAtOnce) {
    const uint4 q = *reinterpret_cast<const uint4*>(maxima + i0);
    const Kept* m = reinterpret_cast<const Kept*>(&q);
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const float v = Vector<T>::value(m[i]);
      if (v >= bound) {
        const int at = atomicAdd(&sh.num_batches, 1);
        if (at < kMostBatches) sh.batches[at] = i0 + i;
      }
    }
  }
  __syncthreads();
  const int batches = sh.num_batches;
  if (batches <= kMostBatches) {
    for (int n = tid; n < batches * kBatch * kSize; n += kThreads) {
      const int batch = sh.batches[n / (kBatch * kSize)], e = n % kSize;
      const int v = row.vector(batch / kThreads, batch % kThreads, n / kSize % kBatch);
      const float x = row.value(v, e);
      if (x >= bound) {
        const int at = atomicAdd(&sh.num_keys, 1);
        if (at < kMostKeys) sh.keys[at] = key_of(x, row.first(v) + e);
      }
    }
  }
  __syncthreads();
  if (batches <= kMostBatches && sh.num_keys <= kMostKeys) return true;
  if (tid < 32) {
    const unsigned long long k = best_in_order<T>(row, maxima, bound, top);
    if (tid < top) sh.best[tid] = k;
  }
  __syncthreads();
  return false;
}

template <typename T, bool kTops>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm<T>)
    toploc_token_logprobs_kernel(const __grid_constant__ LogitParams p) {
  extern __shared__ __align__(16) unsigned char raw[];
  __shared__ Shared sh;
  using V = Vector<T>;
  using Kept = typename V::Kept;
  Kept* maxima = reinterpret_cast<Kept*>(raw);
  cg::cluster_group cluster = cg::this_cluster();
  const int blocks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long r = blockIdx.x / (unsigned)blocks;
  const Share<T> row(p, r, rank, blocks);
  const bool gives = rank == 0 && tid == 0 && p.tokens;
  if (gives) asm volatile("prefetch.global.L2 [%0];" ::"l"(p.tokens + r));

  Sums sums;
  const int batches = row.batches();
  const auto take = [&](const uint4* x, int b) {
    const float m = V::template largest<true>(x);  // NaN where there is one
    if (kTops) maxima[b * kThreads + tid] = V::kept(m == m ? m : V::template largest<false>(x));
    sums.meet(m);
    // (where nothing comes near the reference, as where a mask leaves no token, the powers are below 2^-60 of the sums')
    if (powers_of(m) < sums.c - kNothing) return;
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      Pair v[V::kSize / 2];
      V::floored(x[i], v);
      sums.add<V::kSize / 2>(v);
    }
  };
  const auto take_any = [&](int b) {
    uint4 x[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) x[i] = fetch(row, row.vector(b, tid, i));
    take(x, b);
  };
  // without a look at every vector's place where the batch lies in the row as a whole
  const int inside = (row.inner_end - row.begin) / (kBatch * kThreads);  // batches up to the row's last part of a vector
  int b = 0;
  if (row.inner > row.begin) take_any(b++);  // the row begins inside a vector
  const uint4* at = reinterpret_cast<const uint4*>(row.at - row.shift) + row.vector(b, tid, 0);
#pragma unroll 1
  for (; b < inside; ++b, at += kBatch * kThreads) {
    uint4 x[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) x[i] = __ldcs(at + i * kThreads);
    take(x, b);
  }
#pragma unroll 1
  for (; b < batches; ++b) take_any(b);
  const int64_t token = gives ? p.tokens[r] : -1;
  const bool known = token >= 0 && token < p.vocab;
  const float given = known ? to_float(row.at[token]) : 0.f;

  // the warp's part
  Part part;
  part.top = warp_max(sums.top);
  if (fabsf(part.top) < kSums) {
    sums.renew(powers_of(part.top));
    part.s = warp_sum(sums.s()), part.w = warp_sum(sums.w());
  } else {  // (nothing beside a row's maximum that is not far, else summed again; a NaN stays)
    part.s = warp_sum(sums.s());
    part.s = part.w = part.s != part.s ? part.s : 0.f;
  }
  // the warp's part once more, by differences from the row's maximum: they do not overflow upwards
  const auto sum_again = [&](float top) {
    float s = 0.f, w = 0.f;
    for (int i = 0; i < kBatch * batches; ++i) {
      const int v = row.vector(i / kBatch, tid, i % kBatch);
      for (int e = 0; e < V::kSize; ++e) {
        const float y = max_nan((row.value(v, e) - top) * kLog2e, kLeast), x = exp2_fast(y);
        s += x;
        w = fmaf(x, y, w);
      }
    }
    const Part again = {top, warp_sum(s), warp_sum(w)};
    if (lane == 0) sh.of_warp[warp] = again;
    __syncthreads();
  };
  if (lane == 0) sh.of_warp[warp] = part;
  if (kTops) {
    unsigned o = sums.top > -INFINITY ? ordered(sums.top) : 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const unsigned m = __reduce_max_sync(0xFFFFFFFFu, o);
      if (lane == __ffs(__ballot_sync(0xFFFFFFFFu, o == m)) - 1) o = 0;
      if (lane == i) sh.warp_best[warp * 4 + i] = m;
    }
  }
  __syncthreads();

  if (blocks == 1) {
    float top = sh.of_warp[0].top;
#pragma unroll
    for (int i = 1; i < kWarps; ++i) top = fmaxf(top, sh.of_warp[i].top);
    if (is_far(top)) {
      __syncthreads();  // (all have read what is written again)
      sum_again(top);
    }
  }
  if (warp == 0) {
    const Part all = join_parts(sh.of_warp[lane % kWarps], kWarps);
    if (blocks == 1) {
      const Whole whole = {all.top, all.s, all.w, log2f(all.s)};
      if (lane == 0) {
        sh.whole = whole;
        write_row(p, r, whole, known, given);
      }
    } else if (lane == 0) {
      sh.part = all;
    }
  }
  if (kTops && warp == 1) {  // the bound: the top-th largest of the warps' four largest thread maxima, each of them another logit
    unsigned mine = sh.warp_best[lane];
    warp_sort(mine, 0);
    mine = __shfl_sync(0xFFFFFFFFu, mine, p.top - 1);
    if (lane == 0) {
      sh.bound = mine == 0 ? -FLT_MAX : value_of(mine);  // (every logit above -inf)
      sh.num_batches = sh.num_keys = 0;
    }
  }
  if constexpr (kTops) {
    __syncthreads();
    const bool in_keys = gather_keys<T>(sh, row, maxima, p.top);
    const int keys = in_keys ? sh.num_keys : p.top;
    const unsigned long long mine = tid < keys ? in_keys ? sh.keys[tid] : sh.best[tid] : 0;
    int place_of_mine = kMostTop;
    if (mine != 0) {  // its place: the number of larger ones
      place_of_mine = 0;
      const unsigned long long* list = in_keys ? sh.keys : sh.best;
      for (int i = 0; i < keys; ++i) place_of_mine += list[i] > mine;
    }
    if (blocks == 1) {
      const int held = __syncthreads_count(mine != 0);
      if (place_of_mine < p.top) {
        p.top_ids[r * p.top + place_of_mine] = (int64_t)(0xFFFFFFFFu - (unsigned)mine);
        p.top_logprobs[r * p.top + place_of_mine] = logprob_of(sh.whole, value_of((unsigned)(mine >> 32)));
      }
      if (tid < p.top && tid >= held) {
        p.top_ids[r * p.top + tid] = -1;
        p.top_logprobs[r * p.top + tid] = logprob_of(sh.whole, -INFINITY);
      }
    } else if (in_keys) {
      if (tid < p.top && tid >= keys) sh.best[tid] = 0;
      if (place_of_mine < p.top) sh.best[place_of_mine] = mine;
    }
  }
  if (blocks > 1) {  // the row, from the cluster's shares
    cluster.sync();
    float top = -INFINITY;
    for (int i = 0; i < blocks; ++i) top = fmaxf(top, cluster.map_shared_rank(&sh, i)->part.top);
    if (is_far(top)) {
      cluster.sync();  // (all have read what is written again)
      sum_again(top);
      if (warp == 0) {
        const Part all = join_parts(sh.of_warp[lane % kWarps], kWarps);
        if (lane == 0) sh.part = all;
      }
      cluster.sync();
    }
    unsigned long long mine = 0;
    if (rank == 0) {
      if (warp == 0) {
        const Part all = join_parts(cluster.map_shared_rank(&sh, lane % blocks)->part, blocks);
        if (lane == 0) sh.whole = {all.top, all.s, all.w, log2f(all.s)};
      }
      if (kTops && tid < blocks * p.top) mine = cluster.map_shared_rank(&sh, tid / p.top)->best[tid % p.top];
      sh.keys[tid] = mine;
    }
    const int held = __syncthreads_count(mine != 0);
    // (the other blocks may leave now: their shared memory has been read)
    auto token_of_barrier = cluster.barrier_arrive();
    if (rank == 0) {
      if (tid == 0) write_row(p, r, sh.whole, known, given);
      if constexpr (kTops) {
        if (mine != 0) {
          int above = 0;
#pragma unroll 8
          for (int i = 0; i < blocks * p.top; ++i) above += sh.keys[i] > mine;
          if (above < p.top) {
            p.top_ids[r * p.top + above] = (int64_t)(0xFFFFFFFFu - (unsigned)mine);
            p.top_logprobs[r * p.top + above] = logprob_of(sh.whole, value_of((unsigned)(mine >> 32)));
          }
        }
        if (tid < p.top && tid >= held) {
          p.top_ids[r * p.top + tid] = -1;
          p.top_logprobs[r * p.top + tid] = logprob_of(sh.whole, -INFINITY);
        }
      }
    }
    cluster.barrier_wait(std::move(token_of_barrier));
  }
}

template <typename T, bool kTops>
int launch_rows(const LogitParams& p, long long rows, int blocks, size_t bytes, cudaStream_t stream) {
  const auto kernel = toploc_token_logprobs_kernel<T, kTops>;
  static std::atomic<uint64_t> allowed{0};
  // (the most: the maxima of an eighth of the largest vocabulary)
  constexpr int kMostMaxima = (kMostVocab / Vector<T>::kSize / kMostCluster / kBatch + 2 * kThreads) *
                              (int)sizeof(typename Vector<T>::Kept);
  constexpr int kMostBytes = (kMostMaxima > kMaximaBytes ? kMostMaxima : kMaximaBytes);
  if (const int rc = allow_shared(reinterpret_cast<const void*>(kernel), kMostBytes, allowed)) return rc;
  cudaLaunchConfig_t config = {};
  config.gridDim = dim3((unsigned)(rows * blocks));
  config.blockDim = dim3(kThreads);
  config.dynamicSmemBytes = bytes;
  config.stream = stream;
  cudaLaunchAttribute cluster[1];
  cluster[0].id = cudaLaunchAttributeClusterDimension;
  cluster[0].val.clusterDim.x = (unsigned)blocks;
  cluster[0].val.clusterDim.y = cluster[0].val.clusterDim.z = 1;
  config.attrs = cluster;
  config.numAttrs = 1;
  if (cudaLaunchKernelEx(&config, kernel, p) != cudaSuccess) {
    cudaGetLastError();
    return TOPLOC_ERR_CUDA;
  }
  return launched();
}

template <typename T>
int launch(const LogitParams& p, long long rows, int sms, cudaStream_t stream) {
  constexpr int kSize = Vector<T>::kSize;
  const int vectors = (p.vocab + 2 * (kSize - 1)) / kSize;  // at most
  const auto batches = [&](int blocks) { return ((vectors + blocks - 1) / blocks + kBatch * kThreads - 1) / (kBatch * kThreads); };
  const auto bytes = [&](int blocks) { return (size_t)batches(blocks) * kThreads * sizeof(typename Vector<T>::Kept); };
  // A row's blocks: what gets through the rows soonest, as many blocks at a time as fit, where a block's time is twice its
  // batches and 7 + blocks for its beginning and end (measured with 128000 bf16, one row: 14.4, 10.7, 8.9 and 9.3 us
  // for 1, 2, 4 and 8 blocks; 64 rows: 20.8, 15.1, 12.5 and 13.8; 4097 rows: 172, 208, 297 and 510).
  int blocks = 0;
  long long least = 0;
  for (int n = 1; n <= kMostCluster; n *= 2) {
    if (p.top && n < kMostCluster && bytes(n) > kMaximaBytes) continue;
    const long long at_once = (long long)kBlocksPerSm<T> * sms, rounds = (rows * n + at_once - 1) / at_once;
    const long long cost = rounds * (2 * batches(n) + 7 + n);
    if (blocks == 0 || cost < least) blocks = n, least = cost;
  }
  if (rows * blocks > 0x7FFFFFFF) return TOPLOC_ERR_UNSUPPORTED;
  return p.top ? launch_rows<T, true>(p, rows, blocks, bytes(blocks), stream)
               : launch_rows<T, false>(p, rows, blocks, 0, stream);
}

}  // namespace

extern "C" int toploc_token_logprobs(const void* d_logits, const toploc_logprob_layout* lay, const int64_t* d_tokens_opt,
                                     float* d_logprobs_opt, float* d_entropy_opt, int64_t* d_top_ids,
                                     float* d_top_logprobs, void* cuda_stream) {
  if (!lay || lay->vocab <= 0 || lay->top < 0 || lay->rows < 0 || lay->row_stride < lay->vocab)
    return TOPLOC_ERR_INVALID_ARGUMENT;
  const int size = element_bytes(lay->dtype);
  if (size == 0 || lay->vocab > kMostVocab || lay->top > kMostTop || lay->rows > 0x7FFFFFFF) return TOPLOC_ERR_UNSUPPORTED;
  if ((d_tokens_opt == nullptr) != (d_logprobs_opt == nullptr)) return TOPLOC_ERR_INVALID_ARGUMENT;
  if (lay->rows == 0) return TOPLOC_OK;
  if (!d_logits || !aligned(d_logits, size) || !aligned(d_tokens_opt, 8) || !aligned(d_logprobs_opt, 4) ||
      !aligned(d_entropy_opt, 4))
    return TOPLOC_ERR_INVALID_ARGUMENT;
  if (lay->top > 0 && (!d_top_ids || !d_top_logprobs || !aligned(d_top_ids, 8) || !aligned(d_top_logprobs, 4)))
    return TOPLOC_ERR_INVALID_ARGUMENT;
  int sms = 0;
  if (const int rc = check_device(&sms)) return rc;
  const LogitParams p = {d_logits, d_tokens_opt, d_logprobs_opt, d_entropy_opt, d_top_ids, d_top_logprobs,
                         lay->row_stride, lay->vocab, lay->top};
  const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  return lay->dtype == TOPLOC_DTYPE_BF16 ? launch<__nv_bfloat16>(p, lay->rows, sms, stream)
                                         : launch<float>(p, lay->rows, sms, stream);
}
