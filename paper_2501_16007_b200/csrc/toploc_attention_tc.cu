// Attention on the tensor cores (bf16, head_dim 64 or 128).
//
//   S = Q K^T (128 rows x 128 keys, fp32 in tensor memory),  P = 2^(scale S - m),  O += P V
//
// The rows of a tile are (token, head of the group) pairs of one key head, so a tile of keys is read once
// for all of them, a chunk of 32 tokens with four heads a group fills a tile, and a single token still
// has its heads side by side.
//
// A block has two groups of four warps that do the softmax, a thread per row (no exchange between threads: the
// running maximum and sum of a row live in one), a warp that finds the work and copies queries and keys into a ring of
// tiles, one that copies values, and one that issues the products.  While one group works on its scores the tensor cores
// run the other group's products.  The groups hold, item by item,
//   two row tiles against the same keys      (more than 128 rows), or
//   one row tile against every other key tile (fewer rows: bound by reading the keys, so both groups serve the stream and
//                                              join at the end).
//
// The work is cut evenly, not by items: the keys that all row tiles see, one after the other, are one long line, and
// each of the persistent blocks (one an SM) takes an equal stretch of it.  A tile whose keys lie in several stretches
// leaves partial results (normalised outputs and lse) that a second kernel joins, always in the same order.  So a
// single long sequence and a batch of ragged ones both keep every SM busy to the end, whatever the lengths on the
// device are; there is no bound on them to tune by.  The feeding warps run ahead into the next item while the last one
// is finished.
//
// What bounds it.  A pair of row tiles against a tile of keys (head_dim 128) needs 2048 clocks of the tensor cores and as
// many of the special-function units (256 * 128 exponentials, 16 a clock); it takes about 3300.  A group's softmax and
// then its two products are one chain (2400 and 1700 clocks in a trace of an earlier, slower version), two groups in turn
// hide half of it, and tensor memory (2 * 128 columns of scores, 2 * 128 of outputs) has no room for scores ahead.
// Packed prompts of 16383 rows: 754 us over 30 passes one behind the other (1.14 PFLOP/s, 0.70 of the measured bf16 rate),
// 830 over 200 (the power cap), 880 to 890 on inputs that change from pass to pass (0.60); one sequence of 131000 keys and
// 17 tokens: 136 to 141, and 163 us.  Instruction fetch is the other bound: eleven warps run seven different pieces of code,
// and the kernel gained more from small code (loops that are not unrolled, one code for both feeding warps, rare branches
// out of line: 76 to 57 KB, 146 to 136 us, prompts 840 to 770, all one behind the other) than from fewer instructions.  Tried and not kept: two threads a row with
// 16 softmax warps (the same time, short prompts 52 against 46 us: the maxima have to be exchanged), a share of the
// exponentials as a polynomial on the fp32 units (2 to 10 % slower), the row's scores kept in registers between maximum
// and weights (the same where tiles are many, 10 % slower on short prompts: its code is unrolled).
//
// The output is not rescaled whenever the maximum grows but only where it grew by more than kLazyLog2.
#include "attention_tc.cuh"

#include <type_traits>

namespace {

constexpr int kTcThreads = 384;  // two groups of softmax, and one whose first three warps feed and issue
// Registers move from the third group of warps to the softmax.  The block is launched with 168 a thread (65536 / 384, in
// steps of 8); 2 * 216 + 72 = 3 * 168.
constexpr int kSoftmaxRegisters = 216, kOtherRegisters = 72;

template <int D>
struct Shared {
  static constexpr int kHalves = D / 64;
  static constexpr int kTileBytes = kHalves * kBlockBytes;
  static constexpr int kStages = D == 128 ? 5 : 10;
  struct Head {
    uint64_t full[kStages], empty[kStages];
    uint64_t s_full[2], p_most[2], p_full[2], o_full[2];
    uint64_t q_full, q_empty, drain;
    uint64_t join;  // both groups (one row tile): their sums are exchanged, their outputs read
    uint64_t item_full[kItems], item_empty[kItems];
    Item items[kItems];
    uint32_t tmem;
    alignas(8) int gave_up[2];  // a wait ran out; the limit of a wait
    uint32_t fed[kStages];      // by stage: place of the last copy there + 1
    uint32_t queries_fed;       // copies of queries
    Stretch stretch;            // of the block's work
    uint64_t cleaned[kStages];  // the stage's value tile, one with hidden keys, may be used
    int bad_values[8];  // number of the item (of 8) in whose hidden keys' tiles a value was not finite
  };
  static constexpr int kHeadBytes = 1024, kExchangeBytes = 2 * 128 * 8;
  static_assert(sizeof(Head) <= kHeadBytes, "head");
  static constexpr int kBytes = kHeadBytes + kExchangeBytes + (2 + kStages) * kTileBytes;
  static_assert(kBytes <= 232448, "shared memory of a block");
};

__device__ __forceinline__ void store_32_bytes(void* at, const uint32_t* v) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]),
               "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}

// The largest of three, NaN where one is.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// Scores beyond column `last` become minus infinity, whatever was there.
__device__ __forceinline__ void hide(uint32_t (&x)[32], int last) {
#pragma unroll
  for (int e = 0; e < 32; ++e)
    if (e > last) x[e] = 0xFF800000u;
}

// Two fp32 products and sums in one instruction.
__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpair(uint64_t p, float& a, float& b) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p));
}
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add_pair(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

template <int D>
__global__ void __launch_bounds__(kTcThreads, 1)
toploc_attention_tc_kernel(const __grid_constant__ TcParams tp, const __grid_constant__ CUtensorMap map_q,
                           const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  using S = Shared<D>;
  constexpr int kStages = S::kStages, kHalves = S::kHalves;
  extern __shared__ __align__(1024) unsigned char base[];
  const AttentionParams& p = tp.p;
  typename S::Head& sh = *reinterpret_cast<typename S::Head*>(base);
  float2* exchange = reinterpret_cast<float2*>(base + S::kHeadBytes);  // (maximum, sum) of [group][row]
  unsigned char* q_tiles = base + S::kHeadBytes + S::kExchangeBytes;
  unsigned char* ring = q_tiles + 2 * S::kTileBytes;
  const int warp = __shfl_sync(0xFFFFFFFFu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  volatile int* gave_up = sh.gave_up;

  // tell the join kernel that it may be scheduled (it waits for this grid to end)
  asm volatile("griddepcontrol.launch_dependents;");
  if (threadIdx.x == 0) {
#pragma unroll 1
    for (int i = 0; i < kStages; ++i) {
      barrier_init(shared_address(&sh.full[i]), 1);
      barrier_init(shared_address(&sh.empty[i]), 1);
      barrier_init(shared_address(&sh.cleaned[i]), 1);
      sh.fed[i] = 0;
    }
    for (int w = 0; w < 2; ++w) {
      barrier_init(shared_address(&sh.s_full[w]), 1);
      barrier_init(shared_address(&sh.p_most[w]), 4);
      barrier_init(shared_address(&sh.p_full[w]), 4);
      barrier_init(shared_address(&sh.o_full[w]), 1);
    }
    barrier_init(shared_address(&sh.q_full), 1);
    barrier_init(shared_address(&sh.q_empty), 1);
    barrier_init(shared_address(&sh.drain), 1);
    barrier_init(shared_address(&sh.join), 8);
#pragma unroll 1
    for (int i = 0; i < kItems; ++i) {
      barrier_init(shared_address(&sh.item_full[i]), 1);
      barrier_init(shared_address(&sh.item_empty[i]), 10);
    }
#pragma unroll 1
    for (int i = 0; i < 8; ++i) sh.bad_values[i] = -1;
    sh.gave_up[0] = 0;
    sh.gave_up[1] = tp.wait_tries;
    barrier_init_fence();
  }
  if (warp == 9) tmem_alloc(shared_address(&sh.tmem), 512);
  float* run_cost = reinterpret_cast<float*>(ring);  // where the ring's first tile comes later
  lay_line<kTcThreads>(tp, run_cost);
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, sh.tmem, 0);
  constexpr uint32_t kOut = 256;  // scores of group w at 128 w, outputs at 256 + D w

  if (warp < 8) {  // (first: behind the other roles it made the prompts 1.5 % slower)
    raise_registers<kSoftmaxRegisters>();
    // ---- softmax: a thread per row ----
    const int w = warp >> 2, r = threadIdx.x & 127;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // the warp's 32 rows of tensor memory
    const uint32_t s_at = tmem + lanes + 128 * w;
    uint32_t s_uses = 0, pv[2] = {0, 0};
    const float scale = p.scale_log2;
    uint32_t joins = 0;
    const auto join = [&] {  // both groups are here
      __syncwarp();
      if (lane == 0) barrier_arrive(shared_address(&sh.join));
      return warp_wait(sh.join, joins++ & 1, gave_up);
    };
#pragma unroll 1
    for (uint32_t number = 0;; ++number) {
      const uint32_t slot = number % kItems;
      if (!warp_wait(sh.item_full[slot], (number / kItems) & 1, gave_up)) break;
      const Item im = sh.items[slot];
      __syncwarp();
      if (lane == 0) barrier_arrive(shared_address(&sh.item_empty[slot]));
      if (im.seq < 0) break;
      const int n = item_tiles(im);
      const bool two = im.two;
      const int row = im.row0 + (two ? w * tp.tile_rows : 0) + r;            // packed row
      const bool valid = r < tp.tile_rows && row < im.rows;
      const int token = row / p.group;
      const int newest = valid ? im.behind + token : -1;                     // the newest key the row sees
      // keys up to `common` are seen by every row of the group's tile
      const int common = im.behind + (im.row0 + (two ? w * tp.tile_rows : 0)) / p.group;
      const int hidden_from = max(im.behind + im.row0 / p.group + 1, 0);     // first key hidden from a row of the item
      const bool live = __any_sync(0xFFFFFFFFu, valid);                      // else nobody reads the warp's rows
      const int tiles = two ? (w ? im.n1 : im.n0) : (n + 1 - w) / 2;
      float m = -INFINITY, l = 0.f;
      bool ok = true;
#pragma unroll 1
      for (int i = 0; i < tiles; ++i) {
        const int j = two ? i : 2 * i + w;
        const int key0 = im.kbegin + j * kKeyTile;
        const bool masked = key0 + kKeyTile - 1 > common;
        ok = warp_wait(sh.s_full[w], s_uses++ & 1, gave_up);
        if (!ok) break;
        if (live) {
          // columns up to `seen` are seen by every row of the warp (that counts), none from `upto` on by any
          const int last = newest - key0;
          int seen = kKeyTile, upto = kKeyTile;
          if (masked) {
            seen = __reduce_min_sync(0xFFFFFFFFu, valid ? last : kKeyTile);
            upto = min(__reduce_max_sync(0xFFFFFFFFu, valid ? last : -1) + 1, kKeyTile);
          }
          // loops over quarters of the row, not unrolled, the scores read twice (see above)
          tmem_fence_after();
          float peak = -INFINITY;
          // (tiles with hidden keys have loops of their own: branches in the ordinary ones cost 6 % of the kernel)
          const auto highest = [&](int c, auto hiding) {
            uint32_t x[32];
            tmem_load(x, s_at + 32 * c);
            tmem_wait_load();
            tmem_ready(x);
            if (decltype(hiding)::value && 32 * c + 31 > seen) hide(x, last - 32 * c);
            float top[4] = {peak, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int e = 0; e < 32; e += 2)
              top[e / 2 % 4] = max3(top[e / 2 % 4], __uint_as_float(x[e]), __uint_as_float(x[e + 1]));
            peak = max3(max3(top[0], top[1], top[2]), top[3], -INFINITY);
          };
          if (!masked) {
#pragma unroll 1
            for (int c = 0; c < 4; ++c) highest(c, std::false_type());
          } else {
#pragma unroll 1
            for (int c = 0; 32 * c < upto; ++c) highest(c, std::true_type());
          }
          // (peak - m) * scale > the limit, also where m is -inf; not where both are
          const bool grow = valid && peak > m && !((peak - m) * scale <= kLazyLog2);
          if (__any_sync(0xFFFFFFFFu, grow)) {
            const float shrink = grow ? exp2_approx((m - peak) * scale) : 1.f;
            if (grow) m = peak;
            l *= shrink;
            if (i > 0) {  // what the group has summed so far, once its last product is done
              ok = warp_wait(sh.o_full[w], (pv[w] - 1) & 1, gave_up);
              if (!ok) break;
              tmem_fence_after();
              const uint64_t both = pair(shrink, shrink);
#pragma unroll 1
              for (int c = 0; c < D / 32; ++c) {
                uint32_t o[32];
                tmem_load(o, tmem + lanes + kOut + D * w + 32 * c);
                tmem_wait_load();
                tmem_ready(o);
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                  float a, b;
                  unpair(fma_pair(pair(__uint_as_float(o[e]), __uint_as_float(o[e + 1])), both, 0ull), a, b);
                  o[e] = __float_as_uint(a);
                  o[e + 1] = __float_as_uint(b);
                }
                tmem_store(tmem + lanes + kOut + D * w + 32 * c, o);
              }
            }
          }
          const float ref = m == -INFINITY ? 0.f : m * scale;
          const uint64_t scales = pair(scale, scale), refs = pair(-ref, -ref);
          uint64_t sum[2] = {0ull, 0ull};
          const auto weigh = [&](int c, auto hiding) {
            uint32_t x[32], packed[16];
            tmem_load(x, s_at + 32 * c);  // (weights go where scores have been read: 16 columns of every 32)
            tmem_wait_load();
            tmem_ready(x);
            if (decltype(hiding)::value && 32 * c + 31 > seen) hide(x, last - 32 * c);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const uint64_t t =
                  fma_pair(pair(__uint_as_float(x[2 * e]), __uint_as_float(x[2 * e + 1])), scales, refs);
              float a, b;
              unpair(t, a, b);
              a = exp2_approx(a);
              b = exp2_approx(b);
              sum[e & 1] = add_pair(sum[e & 1], pair(a, b));
              packed[e] = pack_bf16(a, b);
            }
            tmem_store(s_at + 16 * c, packed);
          };
          const auto hand_over = [&](uint64_t& bar) {
            tmem_wait_store();
            tmem_fence_before();
            __syncwarp();
            if (lane == 0) barrier_arrive(shared_address(&bar));
          };
          // three quarters of the weights go ahead: their product runs during the last one
          if (!masked) {
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
              weigh(c, std::false_type());
              if (c == 2) hand_over(sh.p_most[w]);
            }
          } else {
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
              if (32 * c < upto) {
                weigh(c, std::true_type());
              } else {
                uint32_t none[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) none[e] = 0u;
                tmem_store(s_at + 16 * c, none);
              }
              if (c == 2) hand_over(sh.p_most[w]);
            }
          }
          float a, b;
          unpair(add_pair(sum[0], sum[1]), a, b);
          l += a + b;
          if (!(peak < INFINITY)) l = NAN;  // a NaN or infinity among the scores: the softmax of the row is NaN
          hand_over(sh.p_full[w]);
        } else if (lane == 0) {
          barrier_arrive(shared_address(&sh.p_most[w]));
          barrier_arrive(shared_address(&sh.p_full[w]));
        }
        ++pv[w];
      }
      if (!ok) break;

      // ---- the rows' results ----
      pv[w ^ 1] += two ? (w ? im.n0 : im.n1) : (n + 1 - (w ^ 1)) / 2;  // the other group's products
      float weight[2] = {1.f, 0.f}, total = l, top = m;  // one row tile: of the groups' outputs
      if (!two) {
        exchange[w * 128 + r] = make_float2(m, l);
        ok = join();
        if (!ok) break;
        const float2 a = exchange[r], b = exchange[128 + r];
        top = fmaxf(a.x, b.x);
        const float ref = top == -INFINITY ? 0.f : top;
        weight[0] = a.x == -INFINITY ? 0.f : exp2_approx((a.x - ref) * scale);
        weight[1] = b.x == -INFINITY ? 0.f : exp2_approx((b.x - ref) * scale);
        if (top == INFINITY) weight[0] = weight[1] = NAN;
        total = a.y * weight[0] + b.y * weight[1];
        if (a.y != a.y || b.y != b.y) total = NAN;  // a NaN score leaves no trace in a maximum
      }
      const bool any_keys = total != 0.f;
      // 1 / sum, with the groups' weights; 0 where their outputs do not count (and may be anything)
      const float inv = any_keys ? reciprocal(total) : 0.f;
      const float factor[2] = {weight[0] * inv, weight[1] * inv};
      const int head = im.head * p.group + row - token * p.group;
      const long long at = (long long)(im.first + token) * p.q_heads + head;
      // where the row's part of a split tile goes
      const long long part = ((long long)blockIdx.x * 2 + im.slot) * tp.item_rows + (row - im.row0);
      // two row tiles: a group writes its rows; one: each group writes half of the channels
      const int width = two ? D : D / 2, c0 = two ? 0 : w * width;
      const bool mine = (two ? tiles : n) > 0, others = !two && n > 1;
      const uint32_t o_at = tmem + lanes + kOut + (two ? D * w : 0);
      if (two ? mine && w == 0 : mine) ok = warp_wait(sh.o_full[0], (pv[0] - 1) & 1, gave_up);
      if (two ? mine && w == 1 : others) ok = ok && warp_wait(sh.o_full[1], (pv[1] - 1) & 1, gave_up);
      if (!ok) break;
      tmem_fence_after();
      const bool repair = *(volatile int*)&sh.bad_values[number & 7] == (int)number;
#pragma unroll 1
      for (int c = c0; c < c0 + width; c += 32) {
        float o[32];
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] = 0.f;
        if (live && mine) {
          uint32_t x[32];
          tmem_load(x, o_at + c);
          tmem_wait_load();
          tmem_ready(x);
          if (factor[0] != 0.f) {
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = __uint_as_float(x[e]) * factor[0];
          }
          if (others) {
            tmem_load(x, o_at + D + c);
            tmem_wait_load();
            tmem_ready(x);
            if (factor[1] != 0.f) {
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] = fmaf(__uint_as_float(x[e]), factor[1], o[e]);
            }
          }
        }
        if (!valid) continue;
        if (repair) {  // values that were taken out of tiles with hidden keys: back to the rows that see them
          float copy[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) copy[e] = o[e];
          give_back(p, im.seq, im.head, im.first, max(im.kbegin, hidden_from), min(newest + 1, im.kend), c, 32, copy);
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = copy[e];
        }
        if (im.slot < 0) {
          uint32_t packed[16];
#pragma unroll
          for (int e = 0; e < 32; e += 2) packed[e / 2] = pack_bf16(o[e], o[e + 1]);
          __nv_bfloat16* out =
              static_cast<__nv_bfloat16*>(p.out) + (im.first + token) * p.out_token + head * p.out_head + c;
          if (tp.wide_out) {
            store_32_bytes(out, packed);
            store_32_bytes(out + 16, packed + 8);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              reinterpret_cast<uint4*>(out)[e] =
                  make_uint4(packed[4 * e], packed[4 * e + 1], packed[4 * e + 2], packed[4 * e + 3]);
          }
        } else {
          uint32_t words[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) words[e] = __float_as_uint(o[e]);
#pragma unroll
          for (int e = 0; e < 32; e += 8) store_32_bytes(p.part_out + part * D + c + e, words + e);
        }
      }
      if (valid && (two || w == 0)) {
        const float lse2 = any_keys ? (top == -INFINITY ? 0.f : top) * scale + log2_approx(total) : -INFINITY;
        if (im.slot >= 0)
          p.part_lse[part] = lse2;
        else if (p.lse)
          p.lse[at] = lse2 * kLn2;
      }
      if (!two) {  // both have read: the next item may overwrite
        tmem_fence_before();
        if (!join()) break;
      }
    }
  } else {  // the third group of warps: all four hand in their registers together (the last has no other part)
    lower_registers<kOtherRegisters>();
    if (warp == 8 || warp == 10) {
      // ---- feeding: warp 8 finds the items, copies queries and keys, warp 10 values (one code for both: less to fetch) ----
      const bool keys = warp == 8;
      Walk walk(tp);
      if (keys) {
        if (lane == 0) {
          prefetch_map(&map_q);
          prefetch_map(&map_k);
          prefetch_map(&map_v);
        }
        walk.begin<kTcThreads>(run_cost);
        if (lane == 0) sh.stretch = Stretch{walk.at, walk.end};
      }
      uint32_t q_uses = 0;
      Feeder<S> feeder(tp, keys ? &map_k : &map_v, sh, ring, gave_up);
  #pragma unroll 1
      for (uint32_t number = 0;; ++number) {
        const uint32_t slot = number % kItems, parity = (number / kItems) & 1;
        if (!warp_wait(keys ? sh.item_empty[slot] : sh.item_full[slot], keys ? parity ^ 1 : parity, gave_up)) break;
        Item im;
        if (keys)
          walk.next(im);
        else
          im = sh.items[slot];
        im = uniform(im);
        if (keys && lane == 0) sh.items[slot] = im;
        __syncwarp();
        if (lane == 0) barrier_arrive(shared_address(keys ? &sh.item_full[slot] : &sh.item_empty[slot]));
        if (im.seq < 0) break;
        const int n = item_tiles(im), hidden_from = max(im.behind + im.row0 / p.group + 1, 0);
        if (keys && n > 0) {  // queries: each tile in blocks of 64 channels
          if (!warp_wait(sh.q_empty, (q_uses & 1) ^ 1, gave_up)) break;
          ++q_uses;
          const uint32_t q_bar = shared_address(&sh.q_full);
          if (elect_one()) {
            const int tiles = im.two ? 2 : 1;
            barrier_arrive_expect(q_bar, tiles * tp.q_bytes);
  #pragma unroll 1
            for (int w = 0; w < tiles; ++w)
  #pragma unroll
              for (int h = 0; h < kHalves; ++h)
                copy_3d(shared_address(q_tiles + w * S::kTileBytes + h * kBlockBytes), &map_q, q_bar, h * 64,
                        im.head * p.group, im.first + im.row0 / tp.item_rows * tp.item_tokens + w * tp.tile_tokens);
          }
          __syncwarp();
        }
        feeder.item(im, n);
        // Value tiles with hidden keys are cleaned one behind the copies: at once when a tile has landed would hold up the
        // copies, later would hold up the ring.
  #pragma unroll 1
        for (int j = 0; j <= n && feeder.fine; ++j) {
          if (j < n) feeder.feed(j, keys ? key_place(im.two, j) : value_place(im.two, j, n));
          const int landed = j - 1;
          if (keys || !feeder.fine || landed < im.clean || landed < 0) continue;
          const uint32_t place = feeder.base + value_place(im.two, landed, n), stage = ring_stage(place, kStages);
          feeder.fine = warp_wait(sh.full[stage], ring_parity(place, kStages), gave_up);
          if (!feeder.fine) break;
          const int key0 = im.kbegin + landed * kKeyTile;
          clean_values<kHalves, 32>(ring + stage * S::kTileBytes, max(hidden_from - key0, 0), im.kend - key0, lane,
                                    &sh.bad_values[number & 7], (int)number);
          __syncwarp();
          if (lane == 0) barrier_arrive(shared_address(&sh.cleaned[stage]));
        }
        if (!feeder.fine) break;
      }
      if (keys && lane == 0) sh.queries_fed = q_uses;
    } else if (warp == 9) {
      // ---- products: the whole warp follows, one lane issues ----
      constexpr uint32_t kScores = bf16_product(128, false, false), kValues = bf16_product(D, false, true);
      const uint32_t q_low = operand_low(shared_address(q_tiles), 16);
      const uint32_t k_low = operand_low(shared_address(ring), 16), v_low = operand_low(shared_address(ring), kBlockBytes);
      uint32_t used = 0, q_uses = 0, p_parity = 0, cleans = 0;  // cleans: by stage, the parity of its next cleaning
      const auto full = [&](uint32_t n) {
        const bool ok = warp_wait(sh.full[ring_stage(n, kStages)], ring_parity(n, kStages), gave_up);
        tmem_fence_after();
        return ok;
      };
      const auto release = [&](uint32_t n) {
        if (elect_one()) mma_commit(shared_address(&sh.empty[ring_stage(n, kStages)]));
      };
      const auto scores = [&](int w, uint32_t n, bool two) {  // scores of group w against the key tile at place n
        const uint32_t a = q_low + (two ? w : 0) * (S::kTileBytes / 16);
        const uint32_t b = k_low + ring_stage(n, kStages) * (S::kTileBytes / 16);
        if (elect_one()) {
  #pragma unroll
          for (int k = 0; k < D / 16; ++k) {
            const uint32_t at = ((k / 4) * kBlockBytes + (k % 4) * 32) / 16;
            mma_shared(tmem + 128 * w, a + at, b + at, kScores, k > 0);
          }
          mma_commit(shared_address(&sh.s_full[w]));
        }
      };
      const auto values = [&](int w, uint32_t n, bool add) {  // as the group's weights come into tensor memory
        const uint32_t b = v_low + ring_stage(n, kStages) * (S::kTileBytes / 16), parity = p_parity >> w & 1;
        p_parity ^= 1u << w;
        if (!warp_wait(sh.p_most[w], parity, gave_up)) return false;
        tmem_fence_after();
        if (elect_one()) {
  #pragma unroll
          for (int k = 0; k < 6; ++k)
            mma_tmem(tmem + kOut + D * w, tmem + 128 * w + 8 * k, b + k * (2048 / 16), kValues, add || k > 0);
        }
        if (!warp_wait(sh.p_full[w], parity, gave_up)) return false;
        tmem_fence_after();
        if (elect_one()) {
  #pragma unroll
          for (int k = 6; k < 8; ++k)
            mma_tmem(tmem + kOut + D * w, tmem + 128 * w + 8 * k, b + k * (2048 / 16), kValues, true);
          mma_commit(shared_address(&sh.o_full[w]));
        }
        return true;
      };
      const auto queries_used = [&] {
        if (elect_one()) mma_commit(shared_address(&sh.q_empty));
      };
  #pragma unroll 1
      for (uint32_t number = 0;; ++number) {
        const uint32_t slot = number % kItems;
        if (!warp_wait(sh.item_full[slot], (number / kItems) & 1, gave_up)) break;
        // (through a shuffle: the same for every lane, and known to be)
        const int seq = __shfl_sync(0xFFFFFFFFu, sh.items[slot].seq, 0);
        const int n0 = __shfl_sync(0xFFFFFFFFu, sh.items[slot].n0, 0), n1 = __shfl_sync(0xFFFFFFFFu, sh.items[slot].n1, 0);
        const int clean = __shfl_sync(0xFFFFFFFFu, sh.items[slot].clean, 0);
        const bool two = __shfl_sync(0xFFFFFFFFu, sh.items[slot].two, 0);
        __syncwarp();
        if (lane == 0) barrier_arrive(shared_address(&sh.item_empty[slot]));
        if (seq < 0) break;
        const int n = two ? max(n0, n1) : n0;
        if (n == 0) continue;
        bool ok = warp_wait(sh.q_full, q_uses++ & 1, gave_up);
        // Round by round, group by group: the group's weights of a tile times the values, then its scores of the tile it
        // takes next (two row tiles: both groups take every tile, group 1 after group 0; one: tiles in turn).  The first
        // round has only scores.
        const int rounds = two ? n : (n + 1) / 2;
        int cleaned_to = clean;
  #pragma unroll 1
        for (int round = -1; ok && round < rounds; ++round) {
  #pragma unroll 1
          for (int w = 0; w < 2; ++w) {
            const int tiles = two ? (w ? n1 : n0) : n;
            const int j = two ? round : 2 * round + w, next = j + (two ? 1 : 2);
            const bool weigh = round >= 0 && j < tiles, score = next < tiles;
            const uint32_t v_at = used + value_place(two, j, n), k_at = used + key_place(two, next);
            // (group 1 of two row tiles meets what group 0 has waited for, unless group 0 has no such tile)
            if (weigh && (w == 0 || !two || j >= n0)) ok = ok && full(v_at);
            if (score && (w == 0 || !two || next >= n0)) ok = ok && full(k_at);
            if (weigh && j >= cleaned_to) {
              const uint32_t stage = ring_stage(v_at, kStages);
              ok = ok && warp_wait(sh.cleaned[stage], cleans >> stage & 1, gave_up);
              cleans ^= 1u << stage;
              cleaned_to = j + 1;
            }
            if (weigh) {
              ok = ok && values(w, v_at, j >= (two ? 1 : 2));
              if (ok && (w == 1 || !two)) release(v_at);
            }
            if (score && ok) {
              scores(w, k_at, two);
              if (w == 1 || !two) {
                release(k_at);
                if (next == n - 1) queries_used();
              }
            }
          }
        }
        if (!ok) break;
        used += 2 * n;
      }
    }
  }
  __syncthreads();
  if (sh.gave_up[0]) {  // the same for all threads
    if (warp == 9) drain_block<S>(sh);
    if (warp == 0) abandon(tp, sh.stretch);
    __syncthreads();
  }
  if (warp == 9) tmem_free(tmem, 512);
}

// ---- joining the parts ---------------------------------------------------------------------------
//
// Block (b, y) looks after the row tile that block b of the first kernel began and did not finish: its parts are that
// block's slot 1 and slot 0 of the next ones up to the one that finished it.  Part i has out_i = sum p v / sum p and
// lse_i over its keys; the whole is sum_i w_i out_i / sum_i w_i, w_i = 2^(lse_i - max).  A warp per row, parts in order.
constexpr int kJoinRows = 8, kJoinThreads = 256;  // rows of a block: one a warp

template <int D>
__global__ void __launch_bounds__(kJoinThreads) toploc_attention_tc_join_kernel(const __grid_constant__ TcParams tp) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const AttentionParams& p = tp.p;
  const int b = blockIdx.x, lane = threadIdx.x & 31, rows_item = tp.item_rows;
  const Part part = tp.parts[2 * b + 1];
  if (part.seq < 0) return;
  // the block with the last part, 32 at a time (blocks between may have had nothing to do)
  int end = b;
  for (bool more = true; more;) {
    const int i = end + 1 + lane;
    const bool stop = i >= (int)gridDim.x || (tp.parts[2 * i].seq >= 0 && tp.parts[2 * i].last);
    const unsigned stops = __ballot_sync(0xFFFFFFFFu, stop);
    more = stops == 0;
    end += more ? 32 : __ffs(stops);
  }
  end = min(end, (int)gridDim.x - 1);
  const int r = blockIdx.y * kJoinRows + (threadIdx.x >> 5), row = part.row0 + r;
  if (r >= rows_item || row >= part.rows) return;
  // 16 bytes a lane: D / 4 lanes cover a row, so a warp takes 128 / D parts at once, and eight of those in flight (nothing
  // is loaded that waits for another load: the maximum runs along)
  constexpr int kLanes = D / 4, kAtOnce = 32 / kLanes;
  const auto place = [&](int i) { return (long long)(i == b ? 2 * b + 1 : 2 * i) * rows_item + r; };
  float top = -INFINITY, sum = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  const auto add = [&](float lse, float4 from) {
    const float now = fmaxf(top, lse), ref = now == -INFINITY ? 0.f : now;
    const float shrink = exp2f(top - ref), w = exp2f(lse - ref);
    top = now;
    sum = fmaf(sum, shrink, w);
    o.x = fmaf(o.x, shrink, w * from.x);
    o.y = fmaf(o.y, shrink, w * from.y);
    o.z = fmaf(o.z, shrink, w * from.z);
    o.w = fmaf(o.w, shrink, w * from.w);
  };
#pragma unroll 8
  for (int i = b + lane / kLanes; i <= end; i += kAtOnce) {
    const bool there = i == b || tp.parts[2 * i].seq >= 0;
    const float lse = p.part_lse[place(i)];
    const float4 from = *reinterpret_cast<const float4*>(p.part_out + place(i) * D + lane % kLanes * 4);
    if (there) add(lse, from);
  }
  if (kAtOnce == 2) {  // the other half's parts, in the same order for both
    const float other_top = __shfl_xor_sync(0xFFFFFFFFu, top, 16), other_sum = __shfl_xor_sync(0xFFFFFFFFu, sum, 16);
    const float4 other = make_float4(__shfl_xor_sync(0xFFFFFFFFu, o.x, 16), __shfl_xor_sync(0xFFFFFFFFu, o.y, 16),
                                     __shfl_xor_sync(0xFFFFFFFFu, o.z, 16), __shfl_xor_sync(0xFFFFFFFFu, o.w, 16));
    const float now = fmaxf(top, other_top), ref = now == -INFINITY ? 0.f : now;
    const float mine = exp2f(top - ref), theirs = exp2f(other_top - ref);
    top = now;
    sum = sum * mine + other_sum * theirs;
    o = make_float4(o.x * mine + other.x * theirs, o.y * mine + other.y * theirs, o.z * mine + other.z * theirs,
                    o.w * mine + other.w * theirs);
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  const int token = row / p.group, head = part.head * p.group + row - token * p.group;
  if (lane < kLanes) {
    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.out) + (part.first + token) * p.out_token + head * p.out_head;
    reinterpret_cast<uint2*>(out)[lane] = make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
  }
  if (p.lse && lane == 0)
    p.lse[(long long)(part.first + token) * p.q_heads + head] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

// ---- host ------------------------------------------------------------------------------------------

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                 const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                 CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
  static const EncodeTiled fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeTiled>(p);
  }();
  return fn;
}

// A bf16 tensor [.., extent[1], extent[0]] copied in boxes of 64 contiguous elements with the 128-byte swizzle.
// strides: elements, of dimensions 1 and up (of no meaning where the extent is 1).
bool make_map(CUtensorMap* map, const void* at, int rank, const int64_t* extent, const int64_t* stride, const int* box) {
  cuuint64_t sizes[4], steps[3];
  cuuint32_t boxes[4], ones[4] = {1, 1, 1, 1};
  for (int i = 0; i < rank; ++i) {
    sizes[i] = (cuuint64_t)extent[i];
    boxes[i] = (cuuint32_t)box[i];
    if (i > 0) steps[i - 1] = extent[i] == 1 ? 16 : (cuuint64_t)stride[i - 1] * 2;
  }
  return encode_tiled()(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)rank, const_cast<void*>(at), sizes, steps, boxes,
                        ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D>
int launch_join(const TcParams& tp, int blocks, cudaStream_t stream) {
  if (blocks == 1) return TOPLOC_OK;
  cudaLaunchConfig_t config = {};
  config.gridDim = dim3((unsigned)blocks, (unsigned)((tp.item_rows + kJoinRows - 1) / kJoinRows));
  config.blockDim = dim3(kJoinThreads);
  config.stream = stream;
  cudaLaunchAttribute early;
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  config.attrs = &early;
  config.numAttrs = 1;
  return cudaLaunchKernelEx(&config, toploc_attention_tc_join_kernel<D>, tp) == cudaSuccess ? TOPLOC_OK : TOPLOC_ERR_CUDA;
}

template <int D>
int launch(const TcParams& tp, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, int blocks,
           cudaStream_t stream) {
  constexpr int kBytes = Shared<D>::kBytes;
  static std::atomic<uint64_t> allowed{0};
  if (const int rc = allow_shared(reinterpret_cast<const void*>(toploc_attention_tc_kernel<D>), kBytes, allowed)) return rc;
  toploc_attention_tc_kernel<D><<<blocks, kTcThreads, kBytes, stream>>>(tp, q, k, v);
  return launched();
}

}  // namespace

namespace toploc_model {

bool tensor_cores_take(const toploc_attention_layout* lay, const toploc_kv_layout* kv, const void* q, const void* k,
                       const void* v, const void* out) {
  if (lay->dtype != TOPLOC_DTYPE_BF16 || (lay->head_dim != 64 && lay->head_dim != 128)) return false;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16)) return false;
  const int page = kv->page_size;
  if (page > 0 && (page % 8 != 0 || (kKeyTile % page != 0 && page % kKeyTile != 0) || kv->num_pages == 0)) return false;
  // steps of a tensor copy are positive multiples of 16 bytes below 2^40
  const auto step = [](int64_t stride, int64_t extent) {
    return extent <= 1 || (stride > 0 && stride % 8 == 0 && stride < ((int64_t)1 << 39));
  };
  return step(lay->q_token_stride, lay->total_tokens) && step(lay->q_head_stride, lay->q_heads) &&
         step(lay->out_token_stride, lay->total_tokens) && step(lay->out_head_stride, lay->q_heads) &&
         step(kv->k_token_stride, page > 0 ? page : lay->total_tokens) && step(kv->k_head_stride, lay->kv_heads) &&
         step(kv->v_token_stride, page > 0 ? page : lay->total_tokens) && step(kv->v_head_stride, lay->kv_heads) &&
         (page == 0 || (step(kv->k_page_stride, kv->num_pages) && step(kv->v_page_stride, kv->num_pages)));
}

// Whether a row tile's keys can lie in two blocks' stretches: three tiles of keys are never cut (find_stretch).
static bool can_be_cut(const toploc_attention_layout* lay, const toploc_kv_layout* kv) {
  const long long most_keys = kv->page_size > 0 ? (long long)kv->max_pages * kv->page_size : lay->max_new_tokens;
  return most_keys > 3 * kKeyTile;
}

// Parts (outputs, lse, who they belong to) of two row tiles a block; the kernel for few rows has twice the blocks and at
// most kFewRows rows of an item.  Where nothing can be cut, the records alone.
size_t tensor_core_workspace_bytes(const toploc_attention_layout* lay, const toploc_kv_layout* kv) {
  const int group = lay->q_heads / lay->kv_heads;
  const size_t rows = can_be_cut(lay, kv) ? 2 * (128 / group * group) : 0;
  return (size_t)2 * kSms * (rows * (size_t)(lay->head_dim + 1) * 4 + 2 * sizeof(Part));
}

int launch_tensor_cores(AttentionParams& p, const toploc_attention_layout* lay, const toploc_kv_layout* kv, void* workspace,
                        cudaStream_t stream) {
  if (encode_tiled() == nullptr) return TOPLOC_ERR_CUDA;
  const int page = kv->page_size;
  int sms = 0;
  if (const int rc = check_device(&sms)) return rc;
  sms = min(sms, kSms);
  const bool few = (long long)p.max_new * p.group <= kFewRows;
  const int blocks = few ? 2 * sms : sms, tokens = min(128 / p.group, p.max_new);  // tokens of a query copy
  TcParams tp;
  tp.tile_rows = few ? p.max_new * p.group : 128 / p.group * p.group;
  tp.item_rows = few ? tp.tile_rows : 2 * tp.tile_rows;
  tp.tile_tokens = tp.tile_rows / p.group;
  tp.item_tokens = tp.item_rows / p.group;
  tp.piece = few ? 2 : 4;
  tp.share_scale = 1.f / (float)blocks;
  tp.wait_tries = lay->wait_tries > 0 ? lay->wait_tries : kWaitTries;
  tp.page_shift = 0;
  while (page >> (tp.page_shift + 1) > 0) ++tp.page_shift;
  tp.page_tiles = page > kKeyTile ? page / kKeyTile : 1;
  tp.box_rows = page > 0 ? min(page, kKeyTile) : kKeyTile;
  tp.q_bytes = p.head_dim * 2 * p.group * tokens;
  tp.wide_out = aligned(p.out, 32) && p.out_token % 16 == 0 && p.out_head % 16 == 0;
  const bool cut = can_be_cut(lay, kv);
  const long long part_rows = cut ? (long long)2 * blocks * tp.item_rows : 0;
  p.part_out = static_cast<float*>(workspace);
  p.part_lse = p.part_out + part_rows * p.head_dim;
  tp.parts = reinterpret_cast<Part*>(p.part_lse + part_rows);
  tp.p = p;
  CUtensorMap q, k, v;
  const int64_t q_extent[3] = {p.head_dim, p.q_heads, p.total_tokens}, q_stride[2] = {p.q_head, p.q_token};
  const int q_box[3] = {64, p.group, tokens};
  const int64_t kv_extent[4] = {p.head_dim, page > 0 ? page : p.total_tokens, p.kv_heads, page > 0 ? p.num_pages : 1};
  const int64_t k_stride[3] = {p.k_token, p.k_head, p.k_page}, v_stride[3] = {p.v_token, p.v_head, p.v_page};
  const int kv_box[4] = {64, tp.box_rows, 1, 1};
  if (!make_map(&q, p.q, 3, q_extent, q_stride, q_box) || !make_map(&k, p.k, 4, kv_extent, k_stride, kv_box) ||
      !make_map(&v, p.v, 4, kv_extent, v_stride, kv_box))
    return TOPLOC_ERR_CUDA;
  const int rc = few ? launch_few_rows(&tp, &q, &k, &v, blocks, stream)
                 : p.head_dim == 128 ? launch<128>(tp, q, k, v, blocks, stream) : launch<64>(tp, q, k, v, blocks, stream);
  if (rc != TOPLOC_OK) return rc;
  if (!cut) return TOPLOC_OK;  // nothing to join
  return p.head_dim == 128 ? launch_join<128>(tp, blocks, stream) : launch_join<64>(tp, blocks, stream);
}

}  // namespace toploc_model
