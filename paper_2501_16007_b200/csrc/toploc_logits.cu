// Rows of logits: log probability of a given token, entropy, the likeliest alternatives, in one pass over them.
//
// The sums are kept in base 2 against a reference c that follows the maximum loosely: with y_j = x_j log2 e - c,
//   s = sum 2^y_j,  w = sum 2^y_j y_j;  lse = (c + log2 s) ln 2,  entropy = (log2 s - w / s) ln 2.
// c is renewed only when a value passes it by 2^8, so a few times a thread and not with every new maximum (it costs precision
// too: y_j is off by half a step, 2^-22 just below 2^3).
//
// Alternatives: while it streams, a block leaves the largest of every 8 logits in shared memory (2 bytes of 16).  The
// threads' own maxima give a bound that at least `top` logits reach; behind the pass only the groups that reach it are read
// again, a few dozen, and their logits ranked by (value, index).
#include "model_common.cuh"

#include <cooperative_groups.h>

namespace {

using namespace toploc_model;
namespace cg = cooperative_groups;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kGroup = 8;             // logits whose largest is kept
constexpr int kMostVocab = 1 << 20;
constexpr int kMostTop = TOPLOC_MAX_ALTERNATIVES;
constexpr int kMostCluster = 8;       // blocks that share a row
constexpr int kMostGroups = 512;      // groups, and logits in them, that reach the bound; more take the ordered way
constexpr int kMostKeys = 256;
static_assert(kMostKeys >= kThreads && kMostCluster * kMostTop <= kThreads, "a thread for each of a row's candidates");
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kSlack = 8.f;         // powers of 2 that a value may pass the reference by
// Beyond these a product with log2 e could leave fp32: smaller logits count as kTiny (their weight is 0 next to anything
// larger), and rows whose maximum is out of +-kFar are summed again against the maximum itself.
constexpr float kTiny = -1e30f, kFar = 1e29f;
constexpr float kNoReference = -1e30f;  // above kTiny * log2 e: weight 0 for what a thread meets before its first reference

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

// What the blocks of a row tell each other.
struct Part {
  float top, s, w;  // largest logit; sums against it (top * log2 e; kFar: top)
};

struct Shared {
  Part part;
  float warp_top[kWarps], warp_s[kWarps], warp_w[kWarps];
  unsigned warp_best[kWarps * 4];        // each warp's four largest thread maxima
  float bound;
  int num_groups, num_keys;
  unsigned long long best[kMostTop];     // the block's alternatives
  unsigned groups[kMostGroups];
  unsigned long long keys[kMostKeys];
};

__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// Two fp32 numbers in one register pair, and the instructions that take both at once.
using Pair = unsigned long long;
__device__ __forceinline__ Pair pair_of(float a, float b) {
  Pair r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 both(Pair v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ Pair add2(Pair a, Pair b) {
  Pair r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b) {
  Pair r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) {
  Pair r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
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

// Eight logits in registers.
template <typename T>
struct Eight;
template <>
struct Eight<__nv_bfloat16> {
  using Kept = __nv_bfloat16;  // a group's maximum in shared memory
  uint4 q;
  __device__ void load(const __nv_bfloat16* p) { q = __ldcs(reinterpret_cast<const uint4*>(p)); }
  __device__ float largest() const {  // passes over NaN
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&q);
    const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    return __bfloat162float(__hmax(__low2bfloat16(m), __high2bfloat16(m)));
  }
  __device__ void values(float* v) const {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = bf16_low(w[i]), v[2 * i + 1] = bf16_high(w[i]);
  }
  __device__ void floored(float* v) const {  // no smaller than kTiny; NaN stays
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&q);
    const __nv_bfloat162 tiny = __float2bfloat162_rn(kTiny);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 f = __hmax2_nan(h[i], tiny);
      const uint32_t w = *reinterpret_cast<const uint32_t*>(&f);
      v[2 * i] = bf16_low(w), v[2 * i + 1] = bf16_high(w);
    }
  }
};
template <>
struct Eight<float> {
  using Kept = float;
  float4 q[2];
  __device__ void load(const float* p) {
    q[0] = __ldcs(reinterpret_cast<const float4*>(p));
    q[1] = __ldcs(reinterpret_cast<const float4*>(p) + 1);
  }
  __device__ float largest() const {
    return fmaxf(fmaxf(fmaxf(q[0].x, q[0].y), fmaxf(q[0].z, q[0].w)), fmaxf(fmaxf(q[1].x, q[1].y), fmaxf(q[1].z, q[1].w)));
  }
  __device__ void values(float* v) const {
#pragma unroll
    for (int i = 0; i < 2; ++i) v[4 * i] = q[i].x, v[4 * i + 1] = q[i].y, v[4 * i + 2] = q[i].z, v[4 * i + 3] = q[i].w;
  }
  __device__ void floored(float* v) const {
    values(v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = max_nan(v[i], kTiny);
  }
};

__device__ __forceinline__ void keep(__nv_bfloat16* at, float v) { *at = __float2bfloat16_rn(v); }  // (exact: it was one)
__device__ __forceinline__ void keep(float* at, float v) { *at = v; }

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
  // v: floored, largest: of the eight.  The eight are added up among themselves first: a thread's sums then have an eighth of
  // the roundings in a row.
  __device__ __forceinline__ void add(const float* v, float largest) {
    top = fmaxf(top, largest);
    if (powers_of(largest) > c + kSlack) renew(powers_of(largest));
    const Pair scale = pair_of(kLog2e, kLog2e), minus = pair_of(-c, -c);
    Pair y[kGroup / 2], e[kGroup / 2];
#pragma unroll
    for (int i = 0; i < kGroup / 2; ++i) {
      y[i] = fma2(pair_of(v[2 * i], v[2 * i + 1]), scale, minus);
      const float2 q = both(y[i]);
      e[i] = pair_of(exp2_fast(q.x), exp2_fast(q.y));
    }
    s2 = add2(s2, add2(add2(e[0], e[1]), add2(e[2], e[3])));
    w2 = add2(w2, fma2(e[3], y[3], fma2(e[2], y[2], fma2(e[1], y[1], mul2(e[0], y[0])))));
  }
};

// One row, or one block's share of it.
template <typename T>
struct Row {
  const T* at;   // the row
  int shift;     // groups are laid from a 16-byte place on, `shift` logits in front of the row
  int vocab, begin, end;  // groups of this block

  __device__ int first(int g) const { return g * kGroup - shift; }
  __device__ bool whole(int g) const { return first(g) >= 0 && first(g) + kGroup <= vocab; }
  // logits of a group, -inf outside the row
  __device__ void load(int g, float* v) const {
    const int c = first(g);
#pragma unroll
    for (int e = 0; e < kGroup; ++e) v[e] = c + e >= 0 && c + e < vocab ? to_float(at[c + e]) : -INFINITY;
  }
};

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

// Sums of the block into sh.part, against the block's maximum.
__device__ void block_sums(Shared& sh, float top, float s, float w) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  s = warp_sum(s);
  w = warp_sum(w);
  if (lane == 0) sh.warp_s[warp] = s, sh.warp_w[warp] = w;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = w = 0.f;
    for (int i = 0; i < kWarps; ++i) s += sh.warp_s[i], w += sh.warp_w[i];
    sh.part = {top, s, w};
  }
}

// The block's alternatives one after the other, for rows with more candidates than fit (many equal logits, as a rule): a warp
// goes through the groups' maxima in order and keeps the best in its lanes.
template <typename T>
__device__ void best_in_order(const Row<T>& row, const typename Eight<T>::Kept* maxima, float bound, int top,
                              unsigned long long* best) {
  const int lane = threadIdx.x & 31;
  unsigned long long mine = 0;  // lane i: the i-th best
  float least = bound;          // a group has to reach it, and pass it once the list is full (equal ones later lose)
  bool full = false;
  for (int g0 = row.begin; g0 < row.end; g0 += 32) {
    const int g = g0 + lane;
    const float m = g < row.end ? to_float(maxima[g - row.begin]) : -INFINITY;
    unsigned hits = __ballot_sync(0xFFFFFFFFu, m > -INFINITY && (full ? m > least : m >= least));
    while (hits) {
      const int from = __ffs(hits) - 1;
      hits &= hits - 1;
      const int c = row.first(g0 + from) + lane;
      unsigned long long key = 0;
      if (lane < kGroup && c >= 0 && c < row.vocab) {
        const float v = to_float(row.at[c]);
        if (v > -INFINITY) key = key_of(v, c);
      }
#pragma unroll 1
      for (int e = 0; e < kGroup; ++e) {
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
  if (lane < top) best[lane] = mine;
}

// The block's `top` best into sh.best, from the groups' maxima.
template <typename T>
__device__ void block_best(Shared& sh, const Row<T>& row, const typename Eight<T>::Kept* maxima, float thread_top, int top) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // a bound: the top-th largest of the warps' four largest thread maxima, each of them another logit
  unsigned o = thread_top > -INFINITY ? ordered(thread_top) : 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned m = __reduce_max_sync(0xFFFFFFFFu, o);
    const unsigned who = __ballot_sync(0xFFFFFFFFu, o == m);
    if (lane == __ffs(who) - 1) o = 0;
    if (lane == 0) sh.warp_best[warp * 4 + i] = m;
  }
  if (tid < kMostTop) sh.best[tid] = 0;
  if (tid == 0) sh.num_groups = sh.num_keys = 0;
  __syncthreads();
  static_assert(kWarps * 4 == 32 && kMostTop == 32, "one of the warps' maxima a lane");
  if (warp == 0) {
    const unsigned mine = sh.warp_best[lane];
    int above = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const unsigned other = __shfl_sync(0xFFFFFFFFu, mine, i);
      above += other > mine || (other == mine && i < lane);
    }
    if (above == top - 1) sh.bound = mine == 0 ? -INFINITY : value_of(mine);
  }
  __syncthreads();
  const float bound = sh.bound;
  for (int g = row.begin + tid; g < row.end; g += kThreads) {
    const float m = to_float(maxima[g - row.begin]);
    if (m > -INFINITY && m >= bound) {
      const int at = atomicAdd(&sh.num_groups, 1);
      if (at < kMostGroups) sh.groups[at] = g;
    }
  }
  __syncthreads();
  const int groups = sh.num_groups;
  if (groups <= kMostGroups) {
    for (int i = tid; i < groups * kGroup; i += kThreads) {
      const int c = row.first(sh.groups[i / kGroup]) + i % kGroup;
      if (c < 0 || c >= row.vocab) continue;
      const float v = to_float(row.at[c]);
      if (v > -INFINITY && v >= bound) {
        const int at = atomicAdd(&sh.num_keys, 1);
        if (at < kMostKeys) sh.keys[at] = key_of(v, c);
      }
    }
  }
  __syncthreads();
  const int keys = sh.num_keys;
  if (groups > kMostGroups || keys > kMostKeys) {
    if (warp == 0) best_in_order<T>(row, maxima, bound, top, sh.best);
  } else if (tid < keys) {  // the place of a key is the number of larger ones
    const unsigned long long mine = sh.keys[tid];
    int place = 0;
    for (int i = 0; i < keys; ++i) place += sh.keys[i] > mine;
    if (place < top) sh.best[place] = mine;
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads, 5) toploc_token_logprobs_kernel(const __grid_constant__ LogitParams p) {
  extern __shared__ __align__(16) unsigned char raw[];
  __shared__ Shared sh;
  using Kept = typename Eight<T>::Kept;
  Kept* maxima = reinterpret_cast<Kept*>(raw);
  cg::cluster_group cluster = cg::this_cluster();
  const int blocks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const long long r = blockIdx.x / (unsigned)blocks;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

  Row<T> row;
  row.at = static_cast<const T*>(p.logits) + r * p.stride;
  row.vocab = p.vocab;
  row.shift = (int)(reinterpret_cast<uintptr_t>(row.at) % 16 / sizeof(T));
  const int all = (p.vocab + row.shift + kGroup - 1) / kGroup, share = (all + blocks - 1) / blocks;
  row.begin = min(rank * share, all);
  row.end = min(row.begin + share, all);

  float given = 0.f;
  bool known = false;
  if (rank == 0 && tid == 0 && p.tokens) {
    const int64_t t = p.tokens[r];
    known = t >= 0 && t < p.vocab;
    if (known) given = to_float(row.at[t]);
  }

  Sums sums;
  const int inner_begin = row.begin + (row.begin < row.end && !row.whole(row.begin) ? 1 : 0);
  const int inner_end = max(inner_begin, row.end - (row.begin < row.end && !row.whole(row.end - 1) ? 1 : 0));
  constexpr int kUnroll = sizeof(T) == 2 ? 4 : 2;
  for (int g0 = inner_begin + tid; g0 < inner_end; g0 += kUnroll * kThreads) {
    Eight<T> x[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (g0 + u * kThreads < inner_end) x[u].load(row.at + row.first(g0 + u * kThreads));
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int g = g0 + u * kThreads;
      if (g >= inner_end) break;
      const float m = x[u].largest();
      if (p.top) keep(maxima + (g - row.begin), m);
      float v[kGroup];
      x[u].floored(v);
      sums.add(v, m);
    }
  }
  // the first and the last group, where the row begins or ends inside them
  for (int i = 0; i < 2; ++i) {
    const int g = i == 0 ? row.begin : row.end - 1;
    const bool due = i == 0 ? inner_begin > row.begin : inner_end < row.end && row.end - 1 >= inner_begin;
    if (due && tid == i * 32) {
      float v[kGroup], m = -INFINITY;
      row.load(g, v);
#pragma unroll
      for (int e = 0; e < kGroup; ++e) m = fmaxf(m, v[e]), v[e] = max_nan(v[e], kTiny);
      if (p.top) keep(maxima + (g - row.begin), m);
      sums.add(v, m);
    }
  }

  // the block's maximum, and its sums against it
  float top = warp_max(sums.top);
  if (lane == 0) sh.warp_top[warp] = top;
  __syncthreads();
  top = sh.warp_top[0];
#pragma unroll
  for (int i = 1; i < kWarps; ++i) top = fmaxf(top, sh.warp_top[i]);
  if (fabsf(top) < kFar) sums.renew(powers_of(top));
  block_sums(sh, top, sums.s(), sums.w());
  if (p.top) block_best<T>(sh, row, maxima, sums.top, p.top);

  // the row's
  cluster.sync();
  float row_top = -INFINITY;
  for (int i = 0; i < blocks; ++i) row_top = fmaxf(row_top, cluster.map_shared_rank(&sh, i)->part.top);
  const bool far = !(fabsf(row_top) < kFar) && row_top > -INFINITY;
  if (far) {  // summed again against the maximum itself: differences from it do not overflow upwards
    cluster.sync();  // (all have read what is written again)
    float s = 0.f, w = 0.f;
    for (int g = row.begin + tid; g < row.end; g += kThreads) {
      float v[kGroup];
      row.load(g, v);
#pragma unroll
      for (int e = 0; e < kGroup; ++e) {
        const float y = max_nan((v[e] - row_top) * kLog2e, kTiny), x = exp2_fast(y);
        s += x;
        w = fmaf(x, y, w);
      }
    }
    block_sums(sh, row_top, s, w);
    cluster.sync();
  }
  if (rank == 0) {
    float s = 0.f, w = 0.f;
    for (int i = 0; i < blocks; ++i) {
      const Part q = cluster.map_shared_rank(&sh, i)->part;
      if (far) {
        s += q.s, w += q.w;
      } else {
        // (a row with nothing above -inf has sums of 0, or of NaN)
        const float d = row_top > -INFINITY ? fmaxf(powers_of(q.top), kTiny) - powers_of(row_top) : 0.f, f = exp2_fast(d);
        s += f * q.s;
        w += f > 0.f ? f * fmaf(d, q.s, q.w) : f * q.s;
      }
    }
    const float log2_s = log2f(s);
    const bool none = row_top == -INFINITY && !(s != s);
    const auto logprob = [&](float x) {
      if (none || x == -INFINITY) return s != s ? s : -INFINITY;
      return ((far ? (x - row_top) * kLog2e : fmaf(x, kLog2e, -powers_of(row_top))) - log2_s) * kLn2;
    };
    if (tid == 0) {
      if (p.tokens) p.logprobs[r] = known ? logprob(given) : __uint_as_float(0x7FFFFFFFu);
      if (p.entropy) p.entropy[r] = none ? 0.f : (log2_s - w / s) * kLn2;
    }
    if (p.top) {  // of all blocks' alternatives: the place of each is the number of larger ones
      const bool has = tid < blocks * p.top;
      const unsigned long long mine = has ? cluster.map_shared_rank(&sh, tid / p.top)->best[tid % p.top] : 0;
      sh.keys[tid] = mine;
      const int held = __syncthreads_count(mine != 0);
      if (mine != 0) {
        int place = 0;
        for (int i = 0; i < blocks; ++i) {  // (each block's are in order)
          int lo = 0, hi = p.top;
          while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (sh.keys[i * p.top + mid] > mine) lo = mid + 1; else hi = mid;
          }
          place += lo;
        }
        if (place < p.top) {
          p.top_ids[r * p.top + place] = (int64_t)(0xFFFFFFFFu - (unsigned)mine);
          p.top_logprobs[r * p.top + place] = logprob(value_of((unsigned)(mine >> 32)));
        }
      }
      if (tid < p.top && tid >= held) {
        p.top_ids[r * p.top + tid] = -1;
        p.top_logprobs[r * p.top + tid] = s != s ? s : -INFINITY;
      }
    }
  }
  cluster.sync();  // nobody leaves while its shared memory is read
}

template <typename T>
int launch(const LogitParams& p, long long rows, int sms, cudaStream_t stream) {
  using Kept = typename Eight<T>::Kept;
  const int groups = (p.vocab + 16 / (int)sizeof(T) - 1 + kGroup - 1) / kGroup;  // at most
  // A row's blocks: enough for six a processor, but none with less than two rounds of loads, and none whose maxima take more
  // than 32.5 KB (so that six fit).
  int blocks = 1;
  while (blocks < kMostCluster && ((rows * blocks < 6ll * sms && groups / (2 * blocks) >= 4 * kThreads) ||
                                   (p.top && groups / blocks * sizeof(Kept) > 32 * 1024 + 512)))
    blocks *= 2;
  if (rows * blocks > 0x7FFFFFFF) return TOPLOC_ERR_UNSUPPORTED;
  const size_t bytes = p.top ? (size_t)((groups + blocks - 1) / blocks) * sizeof(Kept) : 0;
  constexpr int kMostBytes = (kMostVocab / kGroup + 2) / kMostCluster * (int)sizeof(Kept) + 64;
  static std::atomic<uint64_t> allowed{0};
  const void* kernel = reinterpret_cast<const void*>(toploc_token_logprobs_kernel<T>);
  if (const int rc = allow_shared(kernel, kMostBytes > 65536 ? kMostBytes : 65536, allowed)) return rc;
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
  if (cudaLaunchKernelEx(&config, toploc_token_logprobs_kernel<T>, p) != cudaSuccess) {
    cudaGetLastError();
    return TOPLOC_ERR_CUDA;
  }
  return launched();
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
