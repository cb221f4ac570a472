// Attention on the tensor cores where a sequence brings few rows (up to 8 packed ones: a token, perhaps two, all heads of a
// key head), bf16, head_dim 64 or 128.  Bound by reading the keys and values.
//
//   S^T = K Q^T (128 keys x 16 rows),  P^T = 2^(scale S^T - m),  O^T += V^T P^T (head_dim x 16)
//
// With so few rows the other order (rows along a product's 128) would leave most of the products and of the softmax
// threads empty.  Here a thread has a key and weighs it for all R rows (R exponentials, not 128), and the products are 16
// wide, the least there is.  R is 4 or 8: loops over rows are unrolled, and code for rows that are not there would only
// crowd the instruction caches (with that and other code made small at once, 98 to 59 us at four rows).  A row's
// maximum and sum run over threads, but seldom: the maximum of the first tile stays the reference for the whole item
// unless a score exceeds it by more than the limit that the kernel for many rows has too, so a tile needs
// one vote, and the threads' own sums are added up once at the end.
//
// Two blocks share an SM, three tiles of 32 KB in flight each (head_dim 128).  A block: four warps of softmax, a warp that
// finds the items and copies queries and keys, one that copies values, one that issues the products; the scores of the
// next tile are computed while the weights of this one are.  The work is cut as in the kernel for many rows.
//
// 64 sequences of up to 2048 keys (286 MB), 4 rows: 59 us, 4.9 TB/s, 0.74 of the measured copy (the kernel for many rows:
// 69); 8 rows: 62 (70); 16 rows 85 (72), 32 rows 156 (74), so the other kernel takes those.  Four times the keys: 183 us,
// 6.2 TB/s: what is missing at the smaller size is the start and end of the kernel, and the join.
#include "attention_tc.cuh"

namespace {

constexpr int kFewThreads = 224;
constexpr float kFewLimit = kLazyLog2;
// The reference of a row that has met no score but minus infinity: any other score exceeds it by more than the limit, and
// the weights of minus infinities against it are 0.
constexpr float kNoScore = -3e38f;

template <int D>
struct FewShared {
  static constexpr int N = 16;  // rows of the products
  static constexpr int kHalves = D / 64;
  static constexpr int kTileBytes = kHalves * kBlockBytes;
  static constexpr int kStages = D == 128 ? 3 : 6;
  static constexpr int kQueryBytes = N * 128 * kHalves, kWeightBytes = kKeyTile * N * 2;
  struct Head {
    uint64_t full[kStages], empty[kStages];
    uint64_t s_full[2], p_full, o_full;
    uint64_t q_full, q_empty, drain;
    uint64_t group;  // the four warps of the softmax
    uint64_t item_full[kItems], item_empty[kItems];
    Item items[kItems];
    uint32_t tmem;
    alignas(8) int gave_up[2];  // a wait ran out; the limit of a wait
    uint32_t fed[kStages];      // by stage: place of the last copy there + 1
    uint32_t queries_fed;       // copies of queries
    Stretch stretch;            // of the block's work
    int bad_values[2];    // number of the item (by parity) in whose hidden keys' tiles a value was not finite
    uint32_t exceeds[2];  // number of the tile (by parity) with a score over the limit
    float rows[4][N];     // by warp: maxima, or sums
  };
  static constexpr int kHeadBytes = 1024;
  static_assert(sizeof(Head) <= kHeadBytes, "head");
  static constexpr int kBytes = kHeadBytes + kStages * kTileBytes + kQueryBytes + kWeightBytes;
  static_assert(kBytes <= 115712, "shared memory of half an SM");
};

template <int D, int R>
__global__ void __launch_bounds__(kFewThreads, 2)
toploc_attention_few_kernel(const __grid_constant__ TcParams tp, const __grid_constant__ CUtensorMap map_q,
                            const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v) {
  using S = FewShared<D>;
  constexpr int N = S::N;
  constexpr int kStages = S::kStages, kHalves = S::kHalves;
  extern __shared__ __align__(1024) unsigned char base[];
  const AttentionParams& p = tp.p;
  typename S::Head& sh = *reinterpret_cast<typename S::Head*>(base);
  unsigned char* ring = base + S::kHeadBytes;
  unsigned char* queries = ring + kStages * S::kTileBytes;
  unsigned char* weights = queries + S::kQueryBytes;
  const int warp = __shfl_sync(0xFFFFFFFFu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  volatile int* gave_up = sh.gave_up;

  asm volatile("griddepcontrol.launch_dependents;");  // the join waits for this grid to end
  if (threadIdx.x == 0) {
#pragma unroll 1
    for (int i = 0; i < kStages; ++i) {
      barrier_init(shared_address(&sh.full[i]), 1);
      barrier_init(shared_address(&sh.empty[i]), 1);
      sh.fed[i] = 0;
    }
    for (int i = 0; i < 2; ++i) {
      barrier_init(shared_address(&sh.s_full[i]), 1);
      sh.bad_values[i] = -1;
      sh.exceeds[i] = 0;
    }
    barrier_init(shared_address(&sh.p_full), 4);
    barrier_init(shared_address(&sh.o_full), 1);
    barrier_init(shared_address(&sh.q_full), 1);
    barrier_init(shared_address(&sh.q_empty), 1);
    barrier_init(shared_address(&sh.drain), 1);
    barrier_init(shared_address(&sh.group), 4);
#pragma unroll 1
    for (int i = 0; i < kItems; ++i) {
      barrier_init(shared_address(&sh.item_full[i]), 1);
      barrier_init(shared_address(&sh.item_empty[i]), 6);
    }
    sh.gave_up[0] = 0;
    sh.gave_up[1] = tp.wait_tries;
    barrier_init_fence();
  }
  constexpr uint32_t kColumns = 4 * N;  // tensor memory: two tiles of scores, the outputs (a power of two at least 32)
  if (warp == 5) tmem_alloc(shared_address(&sh.tmem), kColumns);
  float* run_cost = reinterpret_cast<float*>(ring);  // where the ring's first tile comes later
  lay_line<kFewThreads>(tp, run_cost);
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  const uint32_t tmem = __shfl_sync(0xFFFFFFFFu, sh.tmem, 0);
  constexpr uint32_t kOut = 2 * N;  // scores of tile j at N (j % 2), outputs at 2 N

  if (warp == 4 || warp == 6) {
    // ---- feeding: warp 4 finds the items, copies queries and keys, warp 6 values (one code for both: less to fetch) ----
    const bool keys = warp == 4;
    Walk walk(tp);
    if (keys) {
      if (lane == 0) {
        prefetch_map(&map_q);
        prefetch_map(&map_k);
        prefetch_map(&map_v);
      }
      walk.begin<kFewThreads>(run_cost);
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
      if (keys && im.n0 > 0) {
        if (!warp_wait(sh.q_empty, (q_uses & 1) ^ 1, gave_up)) break;
        ++q_uses;
        if (elect_one()) {
          const uint32_t bar = shared_address(&sh.q_full);
          barrier_arrive_expect(bar, tp.q_bytes);
#pragma unroll
          for (int h = 0; h < kHalves; ++h)
            copy_3d(shared_address(queries + h * N * 128), &map_q, bar, h * 64, im.head * p.group, im.first);
        }
        __syncwarp();
      }
      feeder.item(im, im.n0);
#pragma unroll 1
      for (int j = 0; j < im.n0 && feeder.fine; ++j)
        feeder.feed(j, keys ? key_place(false, j) : value_place(false, j, im.n0));
      if (!feeder.fine) break;
    }
    if (keys && lane == 0) sh.queries_fed = q_uses;
  } else if (warp == 5) {
    // ---- products: the whole warp follows, one lane issues ----
    constexpr uint32_t kScores = bf16_product(N, false, false), kValues = bf16_product(N, true, true);
    // (head_dim 64: the upper 64 rows of the second product repeat the lower ones and are not read)
    const uint32_t k_low = operand_low(shared_address(ring), 16);
    const uint32_t v_low = operand_low(shared_address(ring), D == 128 ? kBlockBytes : 0);
    const uint32_t q_low = operand_low(shared_address(queries), 16), w_low = operand_low(shared_address(weights), 128);
    uint32_t used = 0, q_uses = 0, p_uses = 0;
    const auto full = [&](uint32_t n) {
      const bool ok = warp_wait(sh.full[ring_stage(n, kStages)], ring_parity(n, kStages), gave_up);
      tmem_fence_after();
      return ok;
    };
    const auto release = [&](uint32_t n) {
      if (elect_one()) mma_commit(shared_address(&sh.empty[ring_stage(n, kStages)]));
    };
    const auto scores = [&](int j, uint32_t n) {
      const uint32_t a = k_low + ring_stage(n, kStages) * (S::kTileBytes / 16);
      if (elect_one()) {
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
          mma_shared(tmem + N * (j & 1), a + ((k / 4) * kBlockBytes + (k % 4) * 32) / 16,
                     q_low + ((k / 4) * N * 128 + (k % 4) * 32) / 16, kScores, k > 0);
        mma_commit(shared_address(&sh.s_full[j & 1]));
      }
    };
    const auto values = [&](uint32_t n, bool add) {
      const uint32_t a = v_low + ring_stage(n, kStages) * (S::kTileBytes / 16);
      if (elect_one()) {
#pragma unroll
        for (int k = 0; k < kKeyTile / 16; ++k)
          mma_shared<kSwizzledHigh, plain_high(2048)>(tmem + kOut, a + k * (2048 / 16), w_low + k * (256 / 16), kValues,
                                                      add || k > 0);
        mma_commit(shared_address(&sh.o_full));
      }
    };
#pragma unroll 1
    for (uint32_t number = 0;; ++number) {
      const uint32_t slot = number % kItems;
      if (!warp_wait(sh.item_full[slot], (number / kItems) & 1, gave_up)) break;
      const int seq = __shfl_sync(0xFFFFFFFFu, sh.items[slot].seq, 0), n = __shfl_sync(0xFFFFFFFFu, sh.items[slot].n0, 0);
      __syncwarp();
      if (lane == 0) barrier_arrive(shared_address(&sh.item_empty[slot]));
      if (seq < 0) break;
      if (n == 0) continue;
      bool ok = warp_wait(sh.q_full, q_uses++ & 1, gave_up);
      ok = ok && full(used);
      if (!ok) break;
      scores(0, used);
      release(used);
#pragma unroll 1
      for (int j = 0; ok && j < n; ++j) {
        if (j + 1 < n) {
          const uint32_t at = used + key_place(false, j + 1);
          ok = full(at);
          if (!ok) break;
          scores(j + 1, at);
          release(at);
        } else if (elect_one()) {
          mma_commit(shared_address(&sh.q_empty));
        }
        const uint32_t at = used + value_place(false, j, n);
        ok = full(at) && warp_wait(sh.p_full, p_uses++ & 1, gave_up);
        if (!ok) break;
        tmem_fence_after();
        values(at, j > 0);
        release(at);
      }
      if (!ok) break;
      used += 2 * n;
    }
  } else {
    // ---- softmax: a thread per key; at the end a thread per channel ----
    const int me = threadIdx.x;  // 0 .. 127
    const uint32_t lanes = (uint32_t)warp << 21;
    const float scale = p.scale_log2;
    uint32_t used = 0, s_uses[2] = {0, 0}, pv = 0, syncs = 0, tiles_done = 0;
    const auto sync = [&] {  // the four warps
      __syncwarp();
      if (lane == 0) barrier_arrive(shared_address(&sh.group));
      return warp_wait(sh.group, syncs++ & 1, gave_up);
    };
#pragma unroll 1
    for (uint32_t number = 0;; ++number) {
      const uint32_t slot = number % kItems;
      if (!warp_wait(sh.item_full[slot], (number / kItems) & 1, gave_up)) break;
      const Item im = uniform(sh.items[slot]);
      __syncwarp();
      if (lane == 0) barrier_arrive(shared_address(&sh.item_empty[slot]));
      if (im.seq < 0) break;
      const int n = im.n0, rows = im.rows;
      const int hidden_from = max(im.behind + 1, 0);  // first key hidden from a row of the item
      float ref[R], l[R];
#pragma unroll
      for (int r = 0; r < R; ++r) ref[r] = kNoScore, l[r] = 0.f;
      bool ok = true;
#pragma unroll 1
      for (int j = 0; j < n; ++j) {
        const int key0 = im.kbegin + j * kKeyTile, key = key0 + me, buffer = j & 1;
        const bool masked = key0 + kKeyTile - 1 > im.behind;
        ok = warp_wait(sh.s_full[buffer], s_uses[buffer]++ & 1, gave_up);
        if (!ok) break;
        tmem_fence_after();
        uint32_t x[R];
        tmem_load(x, tmem + lanes + N * buffer);
        tmem_wait_load();
        tmem_ready(x);
        float s[R];
#pragma unroll
        for (int r = 0; r < R; ++r) s[r] = __uint_as_float(x[r]) * scale;
        if (masked) {
          int newest = im.behind, head = 0;  // of row r's token
#pragma unroll
          for (int r = 0; r < R; ++r) {
            if (key > newest) s[r] = -INFINITY;  // whatever was there
            if (++head == p.group) head = 0, ++newest;
          }
        }
        // does a score exceed its reference by too much? (tile 0: there is none yet)
        bool renew = j == 0;
        ++tiles_done;
        if (j > 0) {
          bool over = false;
#pragma unroll
          for (int r = 0; r < R; ++r)
            if (r < rows) over = over || s[r] - ref[r] > kFewLimit;
          if (__any_sync(0xFFFFFFFFu, over) && lane == 0) *(volatile uint32_t*)&sh.exceeds[tiles_done & 1] = tiles_done;
          ok = sync();
          if (!ok) break;
          renew = *(volatile uint32_t*)&sh.exceeds[tiles_done & 1] == tiles_done;
        }
        if (renew) {
#pragma unroll
          for (int r = 0; r < R; ++r) {
            if (r < rows) {
              float top = s[r];
#pragma unroll
              for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, off));
              if (lane == 0) sh.rows[warp][r] = top;
            }
          }
          ok = sync();
          if (!ok) break;
          float shrink[R];
#pragma unroll
          for (int r = 0; r < R; ++r) {
            shrink[r] = 0.f;
            if (r < rows) {
              const float top = fmaxf(fmaxf(sh.rows[0][r], sh.rows[1][r]), fmaxf(sh.rows[2][r], sh.rows[3][r]));
              const float now = fmaxf(ref[r], top);
              shrink[r] = exp2_approx(ref[r] - now);
              ref[r] = now;
              l[r] *= shrink[r];
            }
          }
          ok = sync();  // the maxima have been read
          if (!ok) break;
          if (j > 0) {
            ok = warp_wait(sh.o_full, (pv - 1) & 1, gave_up);
            if (!ok) break;
            tmem_fence_after();
            tmem_load(x, tmem + lanes + kOut);
            tmem_wait_load();
            tmem_ready(x);
#pragma unroll
            for (int r = 0; r < R; ++r) x[r] = __float_as_uint(__uint_as_float(x[r]) * shrink[r]);
            tmem_store(tmem + lanes + kOut, x);
            tmem_wait_store();
          }
        }
        uint32_t packed[4];  // of 8 rows
#pragma unroll
        for (int r = 0; r < 4; ++r) packed[r] = 0u;
#pragma unroll
        for (int r = 0; r < R; r += 2) {
          float a = 0.f, b = 0.f;
          if (r < rows) a = exp2_approx(s[r] - ref[r]);
          if (r + 1 < rows) b = exp2_approx(s[r + 1] - ref[r + 1]);
          l[r] += a;
          l[r + 1] += b;
          packed[r / 2] = pack_bf16(a, b);
        }
        if (j > 0) {  // the weights of the tile before have been used
          ok = warp_wait(sh.o_full, (pv - 1) & 1, gave_up);
          if (!ok) break;
        }
        // 8 rows of a key are 16 bytes, keys side by side (the other 8 rows of the product come out as anything)
        *reinterpret_cast<uint4*>(weights + me * 16) = make_uint4(packed[0], packed[1], packed[2], packed[3]);
        if (masked) {
          const uint32_t place = used + value_place(false, j, n), stage = ring_stage(place, kStages);
          ok = warp_wait(sh.full[stage], ring_parity(place, kStages), gave_up);
          if (!ok) break;
          clean_values<kHalves, 128>(ring + stage * S::kTileBytes, max(hidden_from - key0, 0), im.kend - key0, me,
                                     &sh.bad_values[number & 1], (int)number);
        }
        fence_async_shared();
        tmem_fence_before();
        __syncwarp();
        if (lane == 0) barrier_arrive(shared_address(&sh.p_full));
        ++pv;
      }
      if (!ok) break;
      used += 2 * n;

      // ---- the rows' results ----
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (r < rows) {
#pragma unroll
          for (int off = 16; off > 0; off >>= 1) l[r] += __shfl_xor_sync(0xFFFFFFFFu, l[r], off);
          if (lane == 0) sh.rows[warp][r] = l[r];
        }
      }
      ok = sync();
      if (ok && n > 0) ok = warp_wait(sh.o_full, (pv - 1) & 1, gave_up);
      if (!ok) break;
      tmem_fence_after();
      uint32_t x[R];
      if (n > 0) {
        tmem_load(x, tmem + lanes + kOut);
        tmem_wait_load();
        tmem_ready(x);
      }
      const bool repair = *(volatile int*)&sh.bad_values[number & 1] == (int)number;
      float o[R];
#pragma unroll
      for (int r = 0; r < R; ++r) o[r] = n > 0 ? __uint_as_float(x[r]) : 0.f;
      if (repair && me < D) {  // values that were taken out of tiles with hidden keys: back to the rows that see them
        float copy[R];
#pragma unroll
        for (int r = 0; r < R; ++r) copy[r] = o[r];
#pragma unroll 1
        for (int r = 0; r < rows; ++r)
          give_back(p, im.seq, im.head, im.first, max(im.kbegin, hidden_from), min(im.behind + r / p.group + 1, im.kend),
                    me, 1, copy + r);
#pragma unroll
        for (int r = 0; r < R; ++r) o[r] = copy[r];
      }
      // row r's place: of the output, or of the block's part
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.out) + im.first * p.out_token + im.head * p.group * p.out_head + me;
      float* lse = p.lse + (long long)im.first * p.q_heads + im.head * p.group;
      const long long part = ((long long)blockIdx.x * 2 + im.slot) * tp.item_rows;
      int head = 0;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (r < rows) {
          const float total = sh.rows[0][r] + sh.rows[1][r] + sh.rows[2][r] + sh.rows[3][r];
          const bool any_keys = total != 0.f;
          const float value = any_keys ? o[r] * reciprocal(total) : 0.f;
          const float lse2 = any_keys ? ref[r] + log2_approx(total) : -INFINITY;
          if (im.slot >= 0) {
            if (me < D) p.part_out[(part + r) * D + me] = value;
            if (me == r) p.part_lse[part + r] = lse2;
          } else {
            if (me < D) *out = __float2bfloat16_rn(value);
            if (me == r && p.lse) *lse = lse2 * kLn2;
          }
        }
        out += p.out_head;
        ++lse;
        if (++head == p.group) {  // the next token
          head = 0;
          out += p.out_token - p.group * p.out_head;
          lse += p.q_heads - p.group;
        }
      }
      tmem_fence_before();
      if (!sync()) break;  // all have read: the next item may overwrite
    }
  }
  __syncthreads();
  if (sh.gave_up[0]) {  // the same for all threads
    if (warp == 5) drain_block<S>(sh);
    if (warp == 0) abandon(tp, sh.stretch);
    __syncthreads();
  }
  if (warp == 5) tmem_free(tmem, kColumns);
}

template <int D, int R>
int launch(const TcParams& tp, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, int blocks,
           cudaStream_t stream) {
  constexpr int kBytes = FewShared<D>::kBytes;
  static std::atomic<uint64_t> allowed{0};
  if (const int rc = allow_shared(reinterpret_cast<const void*>(toploc_attention_few_kernel<D, R>), kBytes, allowed)) return rc;
  toploc_attention_few_kernel<D, R><<<blocks, kFewThreads, kBytes, stream>>>(tp, q, k, v);
  return launched();
}

template <int D>
int launch_rows(const TcParams& tp, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, int blocks,
                cudaStream_t stream) {
  return tp.item_rows <= 4 ? launch<D, 4>(tp, q, k, v, blocks, stream) : launch<D, 8>(tp, q, k, v, blocks, stream);
}

}  // namespace

namespace toploc_model {

int launch_few_rows(const void* params, const void* map_q, const void* map_k, const void* map_v, int blocks,
                    cudaStream_t stream) {
  const TcParams& tp = *static_cast<const TcParams*>(params);
  const CUtensorMap& q = *static_cast<const CUtensorMap*>(map_q);
  const CUtensorMap& k = *static_cast<const CUtensorMap*>(map_k);
  const CUtensorMap& v = *static_cast<const CUtensorMap*>(map_v);
  return tp.p.head_dim == 128 ? launch_rows<128>(tp, q, k, v, blocks, stream)
                              : launch_rows<64>(tp, q, k, v, blocks, stream);
}

}  // namespace toploc_model
