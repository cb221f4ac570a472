// Queries and keys between projection and attention: the RMS norm of every head and the rotation by position in one
// pass, keys and values straight to the paged cache.
#include "model_common.cuh"

namespace {

using namespace toploc_model;

constexpr int kWarps = 4;             // of a block
constexpr int kBlocksPerSm = 7;
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
  int q_heads, kv_heads;
  int page_size;
  int lane_shift, lanes;   // a head is 2^lane_shift lanes, the first `lanes` of which have channels
  int q_steps, qk_steps, steps;  // ends of the queries' steps, the keys', of all
  int steps_per_warp;
};

// cos and sin of position * freq.  The angle is taken in turns and brought into one turn in 64 bits before it is rounded to 32
// (half a step of half a turn: 2^-26 turns).  The turns of one position, freq / (2 pi), need two numbers of 53 bits: the angle of
// position 2^31 has 2^28 whole turns, which are nothing, and with one number the rest was 2^-24 turns off.  The product with the
// position is rounded once the whole turns are off it.  What is lost is about 2^-104 of the turns: below 2^-40 turns up to
// |position * freq| = 2^64.
__device__ __forceinline__ float2 turn_of(int position, float freq) {
  constexpr double kTurns = 0.15915494309189535, kTurnsRest = -9.839338337591243e-18;  // their sum is 1 / (2 pi)
  const double p = position, f = freq, each = __dmul_rn(f, kTurns), each_rest = fma(f, kTurnsRest, fma(f, kTurns, -each));
  double t = fma(p, each_rest, fma(p, each, -rint(p * each)));
  t -= rint(t);  // (far beyond 2^53 turns the first whole ones are not all)
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
__device__ __forceinline__ void unpack(const Packed<T, kVec>& q, Pair* v) {
  const uint32_t* w = reinterpret_cast<const uint32_t*>(&q);
#pragma unroll
  for (int i = 0; i < kVec / 2; ++i) {
    if constexpr (sizeof(T) == 2)
      v[i] = pair_of(bf16_low(w[i]), bf16_high(w[i]));
    else
      v[i] = pair_of(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
  }
}

template <typename T, int kVec>
__device__ __forceinline__ Packed<T, kVec> pack(const Pair* v) {
  Packed<T, kVec> q;
  uint32_t* w = reinterpret_cast<uint32_t*>(&q);
#pragma unroll
  for (int i = 0; i < kVec / 2; ++i) {
    const float2 f = both(v[i]);
    if constexpr (sizeof(T) == 2)
      w[i] = pack_bf16(f.x, f.y);
    else
      w[2 * i] = __float_as_uint(f.x), w[2 * i + 1] = __float_as_uint(f.y);
  }
  return q;
}

__device__ __forceinline__ Pair swapped(Pair v) {
  const float2 f = both(v);
  return pair_of(f.y, f.x);
}

// Bound by memory: every head is read once and written once.  A warp takes one token and some of its heads, 32 >> lane_shift
// heads of one kind (queries, keys, values) a step.  A lane holds two vectors of a head, chosen so that turned channels meet
// in one lane: vector l and the one half the turned channels further on, or two neighbours; so the rotation needs no
// exchange, and the norm's sum a few shuffles.  The turns of a token are the same for all its heads: the warp works them out
// once (two a lane for 128 channels), and every lane keeps their products with the norm's weights in registers while the kind
// stays.  The arithmetic takes two fp32 numbers at a time.  33443 tokens of 32 + 8 + 8 heads of 128 into the cache: 136 us
// (6.0 TB/s).  Warps count for more than loads a warp: seven blocks an SM (72 registers) with two steps at a time, against 141
// with six, 143 with eight, 140 with five and four steps.
//
// A lane's places in a step's heads are 32-bit numbers, a step's heads the warp's common base.
template <typename T, int kVec, bool kNeighbours, bool kAllTurn, int kUnroll>
__global__ void __launch_bounds__(kWarps * 32, kBlocksPerSm) toploc_norm_rotary_kernel(const __grid_constant__ RotaryParams p) {
  __shared__ float2 turns[kWarps][kMostHalf];
  using Vector = Packed<T, kVec>;
  constexpr int kPairs = kVec / 2;
  const int lane = threadIdx.x & 31, warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0);
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
  const int begin = blockIdx.y * p.steps_per_warp, end = min(begin + p.steps_per_warp, p.steps);

  bool turned = false, placed = false;
  long long page = 0, at = 0;
  // (zeros stay in lanes without channels)
  Vector in_a[kUnroll] = {}, in_b[kUnroll] = {};
#pragma unroll 1
  for (int kind = 0; kind < 2; ++kind) {  // queries, keys
    const int first = kind == 0 ? 0 : p.q_steps, last = kind == 0 ? p.q_steps : p.qk_steps;
    int s = max(begin, first);
    const int stop = min(end, last);
    if (s >= stop) continue;
    const Heads& w = p.part[kind];
    // heads from the lane's on that there are (none for lanes without channels)
    int left = has ? (kind == 0 ? p.q_heads : p.kv_heads) - (s - first) * per_step - sub : 0;
    const long long head = (long long)(s - first) * per_step;
    const T* from = static_cast<const T*>(w.in) + token * w.in_token + head * w.in_head;
    const unsigned from_a = sub * (unsigned)w.in_head + a * kVec, from_b = sub * (unsigned)w.in_head + b * kVec;
    const unsigned to_a = sub * (unsigned)w.out_head + a * kVec, to_b = sub * (unsigned)w.out_head + b * kVec;
    T* to = nullptr;
    // What the norm's weight g and the turn come to together, of channels x (vector a) and y (b):
    //   halves      x <- x (g_x cos) + y (-g_y sin),  y <- y (g_y cos) + x (g_x sin)
    //   neighbours  (x0, x1) <- (x0, x1) (g0 cos, g1 cos) + (x1, x0) (-g1 sin, g0 sin), and so for y
    Pair own_x[kPairs], own_y[kPairs], other_x[kPairs], other_y[kPairs];
#pragma unroll 1
    for (; s < stop; s += kUnroll) {
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        if (s + u < stop && left > u * per_step) {
          in_a[u] = *reinterpret_cast<const Vector*>(from + from_a);
          in_b[u] = *reinterpret_cast<const Vector*>(from + from_b);
        }
        from += per_step * w.in_head;
      }
      if (!turned) {  // behind the first loads, in front of their use
        turned = true;
        const int position = p.half ? p.positions[token] : 0;
        for (int j = lane; j < p.half; j += 32) turns[warp][j] = turn_of(position, p.inv_freq[j]);
        placed = place_of(p, token, &page, &at);
        __syncwarp();
      }
      if (to == nullptr) {
        to = static_cast<T*>(w.out) + head * w.out_head +
             (kind == 0 ? token * w.out_token : page * w.out_page + at * w.out_token);
        const Pair one = pair_of(1.f, 1.f);
#pragma unroll
        for (int e = 0; e < kPairs; ++e) own_x[e] = own_y[e] = one;
        if (w.weight && has) {
          unpack<T, kVec>(__ldg(static_cast<const Vector*>(w.weight) + a), own_x);
          unpack<T, kVec>(__ldg(static_cast<const Vector*>(w.weight) + b), own_y);
        }
#pragma unroll
        for (int e = 0; e < kPairs; ++e) {
          if constexpr (kNeighbours) {
            const float2 gx = both(own_x[e]), gy = both(own_y[e]);
            const int j = l * kVec + e;
            const float2 tx = turn_a ? turns[warp][j] : make_float2(1.f, 0.f);
            const float2 ty = turn_b ? turns[warp][j + kPairs] : make_float2(1.f, 0.f);
            own_x[e] = mul2(own_x[e], pair_of(tx.x, tx.x)), own_y[e] = mul2(own_y[e], pair_of(ty.x, ty.x));
            other_x[e] = pair_of(-gx.y * tx.y, gx.x * tx.y), other_y[e] = pair_of(-gy.y * ty.y, gy.x * ty.y);
          } else {
            const int j = l * kVec + 2 * e;
            const float2 t0 = turn_a ? turns[warp][j] : make_float2(1.f, 0.f);
            const float2 t1 = turn_a ? turns[warp][j + 1] : make_float2(1.f, 0.f);
            const Pair cs = pair_of(t0.x, t1.x);
            other_x[e] = mul2(own_y[e], pair_of(-t0.y, -t1.y)), other_y[e] = mul2(own_x[e], pair_of(t0.y, t1.y));
            own_x[e] = mul2(own_x[e], cs), own_y[e] = mul2(own_y[e], cs);
          }
        }
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        if (s + u >= stop) break;
        Pair x[kPairs], y[kPairs];
        unpack<T, kVec>(in_a[u], x);
        unpack<T, kVec>(in_b[u], y);
        float r = 1.f;
        if (w.weight) {
          Pair sum = mul2(x[0], x[0]);
#pragma unroll
          for (int e = 1; e < kPairs; ++e) sum = fma2(x[e], x[e], sum);
#pragma unroll
          for (int e = 0; e < kPairs; ++e) sum = fma2(y[e], y[e], sum);
          float ss = both(sum).x + both(sum).y;
#pragma unroll
          for (int off = 16; off > 0; off >>= 1)
            if (off < width) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, off);
          r = rsqrtf(fmaf(ss, p.per_channel, p.eps));
        }
        const Pair rr = pair_of(r, r);
#pragma unroll
        for (int e = 0; e < kPairs; ++e) x[e] = mul2(x[e], rr), y[e] = mul2(y[e], rr);
        Pair xx[kPairs], yy[kPairs];
#pragma unroll
        for (int e = 0; e < kPairs; ++e) xx[e] = mul2(x[e], own_x[e]), yy[e] = mul2(y[e], own_y[e]);
        // (channels that do not turn must not meet others: 0 times infinity)
        if (kAllTurn || turn_a) {
#pragma unroll
          for (int e = 0; e < kPairs; ++e) xx[e] = fma2(kNeighbours ? swapped(x[e]) : y[e], other_x[e], xx[e]);
        }
        if (kAllTurn || turn_b) {
#pragma unroll
          for (int e = 0; e < kPairs; ++e) yy[e] = fma2(kNeighbours ? swapped(y[e]) : x[e], other_y[e], yy[e]);
        }
        const Vector out_a = pack<T, kVec>(xx), out_b = pack<T, kVec>(yy);
        if (left > u * per_step && (kind == 0 || placed)) {
          *reinterpret_cast<Vector*>(to + to_a) = out_a;
          *reinterpret_cast<Vector*>(to + to_b) = out_b;
        }
        to += per_step * w.out_head;
      }
      left -= kUnroll * per_step;
    }
  }

  // values, as they are
  const int s = max(begin, p.qk_steps);
  if (s >= end) return;
  if (!turned) placed = place_of(p, token, &page, &at);
  if (!placed) return;
  const Heads& w = p.part[2];
  const T* from = static_cast<const T*>(w.in) + token * w.in_token + (s - p.qk_steps) * per_step * w.in_head;
  T* to = static_cast<T*>(w.out) + page * w.out_page + at * w.out_token + (s - p.qk_steps) * per_step * w.out_head;
  const unsigned from_lane = sub * (unsigned)w.in_head + l * kVec, to_lane = sub * (unsigned)w.out_head + l * kVec;
  int left = has ? p.kv_heads - (s - p.qk_steps) * per_step - sub : 0;
#pragma unroll 4
  for (int i = s; i < end; ++i) {
    if (left > 0) {
      const Vector x = *reinterpret_cast<const Vector*>(from + from_lane);
      const Vector y = *reinterpret_cast<const Vector*>(from + from_lane + p.lanes * kVec);
      *reinterpret_cast<Vector*>(to + to_lane) = x;
      *reinterpret_cast<Vector*>(to + to_lane + p.lanes * kVec) = y;
    }
    left -= per_step;
    from += per_step * w.in_head;
    to += per_step * w.out_head;
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
  const int which = h < p.q_heads ? 0 : h < p.q_heads + p.kv_heads ? 1 : 2;
  const int first = which == 0 ? 0 : which == 1 ? p.q_heads : p.q_heads + p.kv_heads;
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
  for (int j = lane; j < p.half; j += 32) {  // (a pair's turn once: it takes longer than the rest of its channels)
    float& a = head[warp][neighbours ? 2 * j : j];
    float& b = head[warp][neighbours ? 2 * j + 1 : j + p.half];
    const float x = a, y = b;
    const float2 t = turn_of(position, p.inv_freq[j]);
    a = x * t.x - y * t.y;
    b = x * t.y + y * t.x;
  }
  __syncwarp();
  for (int c = lane; c < p.head_dim; c += 32) store_as(out + c, head[warp][c]);
}

template <typename T, int kVec>
void launch_vectors(const RotaryParams& p, bool neighbours, bool all_turn, dim3 grid, cudaStream_t stream) {
  constexpr int kUnroll = 2, kBlock = kWarps * 32;
  if (neighbours && all_turn)
    toploc_norm_rotary_kernel<T, kVec, true, true, kUnroll><<<grid, kBlock, 0, stream>>>(p);
  else if (neighbours)
    toploc_norm_rotary_kernel<T, kVec, true, false, kUnroll><<<grid, kBlock, 0, stream>>>(p);
  else if (all_turn)
    toploc_norm_rotary_kernel<T, kVec, false, true, kUnroll><<<grid, kBlock, 0, stream>>>(p);
  else
    toploc_norm_rotary_kernel<T, kVec, false, false, kUnroll><<<grid, kBlock, 0, stream>>>(p);
}

// Memory of an argument: runs of `bytes`, `count` of them `step` bytes apart in two directions (heads, tokens).
struct Area {
  uintptr_t at;
  long long bytes, count[2], step[2];
  __int128 extent;

  Area(const void* p, long long bytes) : Area(p, bytes, 1, 0, 1, 0) {}
  Area(const void* p, long long run, long long heads, long long head_step, long long tokens, long long token_step)
      : at(reinterpret_cast<uintptr_t>(p)), bytes(p ? run : 0), count{heads, tokens}, step{head_step, token_step} {
    for (int n = 0; n < 2; ++n)
      for (int d = 0; d < 2; ++d)  // runs side by side are one
        if (count[d] == 1 || step[d] <= bytes) bytes += (count[d] - 1) * step[d], count[d] = 1, step[d] = 0;
    extent = bytes;
    for (int d = 0; d < 2; ++d) extent += (__int128)(count[d] - 1) * step[d];
  }
};

// Whether two areas share memory.  Known where their steps are the same, or one has none, in either direction; others count as
// apart.
bool meet(const Area& a, const Area& b) {
  if (a.bytes <= 0 || b.bytes <= 0 || a.extent > 1ll << 60 || b.extent > 1ll << 60) return false;
  const long long away = (long long)(a.at - b.at);
  if (away >= (long long)b.extent || away <= -(long long)a.extent) return false;
  long long step[2], low[2], high[2];  // of the places of a run of a, less those of one of b
  for (int d = 0; d < 2; ++d) {
    if (a.count[d] > 1 && b.count[d] > 1 && a.step[d] != b.step[d]) return false;
    step[d] = max(a.step[d], b.step[d]), low[d] = 1 - b.count[d], high[d] = a.count[d] - 1;
  }
  const int outer = high[0] - low[0] <= high[1] - low[1] ? 0 : 1, inner = 1 - outer;
  for (long long e = low[outer]; e <= high[outer]; ++e) {
    // the first place in the other direction that is not in front of b's run
    const long long from = away + e * step[outer], least = -a.bytes - from;
    long long i = low[inner];
    if (step[inner] > 0)
      i = max(i, least >= 0 ? least / step[inner] + 1 : -((-least - 1) / step[inner]));
    const long long gap = from + i * step[inner];
    if (i <= high[inner] && gap > -a.bytes && gap < b.bytes) return true;
  }
  return false;
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
    // in place, but not each head at its own place
    const int heads = i == 0 ? lay->q_heads : lay->kv_heads;
    if (w.in == w.out && (i == 0 || parts == 2) &&
        ((lay->num_tokens > 1 && w.in_token != w.out_token) || (heads > 1 && w.in_head != w.out_head)))
      return TOPLOC_ERR_INVALID_ARGUMENT;
  }
  const long long head = (long long)lay->head_dim * size;
  // outputs (not the caches) apart from inputs and each other: other warps read and write them
  const auto area = [&](int i, bool out) {
    const Heads& w = p.part[i];
    const auto bytes = [&](long long step) { return min(step, 1ll << 57) * size; };
    return Area(out ? w.out : w.in, head, i == 0 ? lay->q_heads : lay->kv_heads,
                bytes(out ? w.out_head : w.in_head), lay->num_tokens, bytes(out ? w.out_token : w.in_token));
  };
  const Area vectors[] = {{lay->rotary_dim > 0 ? positions : nullptr, lay->num_tokens * 4}, {inv_freq, lay->rotary_dim * 2ll},
                          {p.part[0].weight, head}, {p.part[1].weight, head}, {p.slots, lay->num_tokens * 8}};
  for (int o = 0; o < (parts == 2 ? 2 : 1); ++o) {
    const Area out = area(o, true);
    for (int i = 0; i < parts; ++i)
      if ((i != o || p.part[i].in != p.part[o].out) && meet(out, area(i, false))) return TOPLOC_ERR_INVALID_ARGUMENT;
    for (const Area& v : vectors)
      if (meet(out, v)) return TOPLOC_ERR_INVALID_ARGUMENT;
    if (o == 1 && meet(out, area(0, true))) return TOPLOC_ERR_INVALID_ARGUMENT;
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
  p.kv_heads = lay->kv_heads;
  const int heads = p.q_heads + (parts - 1) * p.kv_heads;
  const bool neighbours = lay->pairing == TOPLOC_ROTARY_NEIGHBOURS;

  // Whole vectors of `vec` elements everywhere: two a lane, turned channels in whole vectors.  16 bytes where they fit (34
  // thousand tokens of heads of 128: 136 us, with 8 bytes 172, element by element 609), else 8 (heads of 80 of which 40 turn:
  // 164 us, element by element 567).
  const auto fits = [&](int vec) {
    const uintptr_t bytes = vec * size;
    long long off = 0;  // bits of places and steps that a vector's must not have
    uintptr_t away = 0;
    for (int i = 0; i < parts; ++i) {
      const Heads& w = p.part[i];
      away |= reinterpret_cast<uintptr_t>(w.in) | reinterpret_cast<uintptr_t>(w.out) | reinterpret_cast<uintptr_t>(w.weight);
      off |= w.in_token | w.in_head | w.out_page | w.out_token | w.out_head;
      if (w.in_head >= 1ll << 26 || w.out_head >= 1ll << 26) return false;  // (places in a step's 32 heads at most: 32 bits)
    }
    return p.head_dim % (2 * vec) == 0 && (neighbours ? lay->rotary_dim : p.half) % vec == 0 &&
           p.head_dim / (2 * vec) <= 32 && (away & (bytes - 1)) == 0 && (off & (vec - 1)) == 0;
  };
  const int wide = 16 / size, vec = fits(wide) ? wide : size == 2 && fits(4) ? 4 : 0;
  const unsigned blocks = (unsigned)((p.num_tokens + kWarps - 1) / kWarps);
  if (vec == 0) {
    const dim3 grid(blocks, (unsigned)heads);
    if (size == 2)
      toploc_norm_rotary_any_kernel<__nv_bfloat16><<<grid, kWarps * 32, 0, stream>>>(p, neighbours);
    else
      toploc_norm_rotary_any_kernel<float><<<grid, kWarps * 32, 0, stream>>>(p, neighbours);
    return launched();
  }
  const bool all_turn = lay->rotary_dim == p.head_dim;
  p.lanes = p.head_dim / (2 * vec);
  while (1 << p.lane_shift < p.lanes) ++p.lane_shift;
  const int per_step = 32 >> p.lane_shift;
  p.q_steps = (p.q_heads + per_step - 1) / per_step;
  p.qk_steps = p.q_steps + (p.kv_heads + per_step - 1) / per_step;
  p.steps = p.q_steps + (parts - 1) * (p.qk_steps - p.q_steps);
  // As many heads a warp as leave the SMs enough warps (32 each), so that few of them work the same turns out again (2000
  // tokens of 48 heads of 128: 15.1, 12.8 and 20.8 us with 8, 32 and 200).
  const long long split = min((long long)p.steps, max(1ll, 32ll * sms / p.num_tokens));
  p.steps_per_warp = (int)((p.steps + split - 1) / split);
  const dim3 grid(blocks, (unsigned)((p.steps + p.steps_per_warp - 1) / p.steps_per_warp));
  if (size == 4)
    launch_vectors<float, 4>(p, neighbours, all_turn, grid, stream);
  else if (vec == 8)
    launch_vectors<__nv_bfloat16, 8>(p, neighbours, all_turn, grid, stream);
  else
    launch_vectors<__nv_bfloat16, 4>(p, neighbours, all_turn, grid, stream);
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
