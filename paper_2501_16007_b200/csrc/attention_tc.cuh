// What the tensor-core kernels of attention share: how the work is cut over the blocks, the feeding of keys and values
// by tensor copies, and the join of partial results.
#pragma once

#include "attention_common.cuh"
#include "sm100.cuh"

namespace {

using namespace toploc_model;
using namespace sm100;

constexpr int kItems = 4;                  // items announced ahead
// A row's reference is renewed where a score exceeds it by more than this factor of 2^8: weights stay below 2^8, and the
// output, the sum and the weights share the reference, so the quotient is the same.  (Sums of weighted values are fp32: up
// to 2^8 times the keys times the values has to fit it.)
constexpr float kLazyLog2 = 8.0f;
constexpr int kBlockBytes = 128 * 128;     // 128 rows of 64 elements

// One piece of work: two tiles of rows (or the one that is left) of a sequence and key head against a range of keys.
struct Item {
  int seq;     // -1: no more work
  int head;    // key head
  int slot;    // where the result goes: -1 the output, 0 a part whose row tile began in an earlier block, 1 in this one
  int first;   // row of the packed tensors its sequence starts at
  int behind;  // keys in front of the sequence's first new token (may be negative)
  int row0;    // first packed row (token * group + head in group)
  int rows;    // packed rows of the sequence
  int kbegin;  // keys kbegin .. kend - 1, kbegin a multiple of the tile
  int kend;
  int two;     // two row tiles
  int n0, n1;  // key tiles of the two groups, or n0 in all
  int clean;   // tiles from here on hold keys that are hidden from a row (or none at all at their end)
};

// The parts a block leaves, for the join.
struct Part {
  int seq, head, row0, first, rows;  // seq -1: none
  int last;                          // slot 0: the row tile's keys end here
};

struct TcParams {
  AttentionParams p;
  int tile_rows;  // packed rows of a row tile: 128 rounded down to whole tokens
  int tile_tokens, item_tokens;  // tokens of a row tile, of an item
  int item_rows;  // packed rows of an item: two tiles (a few rows: all that a sequence can bring)
  int piece;      // tiles (a power of two): where a block's share is short, row tiles are cut at multiples only
  int box_rows;   // rows of a key copy
  int page_shift, page_tiles;  // pages below a tile: log2 of their size; others: tiles a page
  float share_scale;  // 1 / blocks
  int q_bytes;    // bytes of a query tile's copy
  int wait_tries; // limit of a wait
  bool wide_out;  // rows of the output at multiples of 32 bytes
  Part* parts;    // [blocks][2]
};

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ float reciprocal(float x) {  // within an ulp
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float log2_approx(float x) {  // within 2^-22
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ uint32_t ring_stage(uint32_t n, int stages) { return n % (uint32_t)stages; }
__device__ __forceinline__ uint32_t ring_parity(uint32_t n, int stages) { return (n / (uint32_t)stages) & 1u; }

// A wait of a whole warp: all lanes or none go on.
__device__ __forceinline__ bool warp_wait(const uint64_t& bar, uint32_t parity, volatile int* gave_up) {
  return __all_sync(0xFFFFFFFFu, barrier_wait(shared_address(&bar), parity, gave_up));
}

// Tiles of the ring an item takes, and the places of key and value tile j among them.
__device__ __forceinline__ int item_tiles(const Item& im) { return im.two ? max(im.n0, im.n1) : im.n0; }
__device__ __forceinline__ int key_place(bool two, int j) { return two ? 2 * j : max(2 * j - 1, 0); }
__device__ __forceinline__ int value_place(bool two, int j, int n) {
  return two ? 2 * j + 1 : min(n, j + 2) + j;  // K0 V0 K1 V1 .. or K0 K1 V0 K2 V1 ..
}

// ---- the line of work ----------------------------------------------------------------------------
//
// A sequence of T rows and c keys in front of them has L levels of rows_item rows per key head; a level stands for
// kLevelCost (what an item costs beside its keys, in keys) + c + the tokens up to its end.  Sequences follow one
// another, in them key heads, in them levels.

//
// In fp32: the line decides only where it is cut, every block computes the same numbers, and code is what the start of
// these kernels waits for (instruction caches that are empty at a launch; 64-bit arithmetic and divisions were most of it).

constexpr float kLevelCost = 192.f;

struct Line {
  float front;  // kLevelCost + keys in front
  float tokens_item, cut;  // cut: tokens that the last level lacks
  int levels;
  __device__ Line(const TcParams& tp, const SeqRange& s)
      : front(kLevelCost + (float)max(s.keys - s.rows, 0)), tokens_item((float)tp.item_tokens),
        levels((s.rows + tp.item_tokens - 1) / tp.item_tokens) {
    cut = (float)levels * tokens_item - (float)s.rows;
  }
  __device__ float upto(int level) const {  // of levels 0 .. level - 1
    const float n = (float)level;
    return n * (front + 0.5f * tokens_item * (n + 1.f)) - (level < levels ? 0.f : cut);
  }
};

// A place on the line: a key tile of a level.
struct Place {
  int seq, head, level, tile;
};

__device__ __forceinline__ bool before(const Place& a, const Place& b) {
  const int d = a.seq != b.seq ? a.seq - b.seq : a.head != b.head ? a.head - b.head
                : a.level != b.level ? a.level - b.level : a.tile - b.tile;
  return d < 0;
}

// Key tiles that a level's rows see in all.
__device__ __forceinline__ int tiles_seen(const SeqRange& s, int tokens_upto) {
  const int seen = min(s.keys, s.keys - s.rows + tokens_upto);
  return seen > 0 ? (seen + kKeyTile - 1) / kKeyTile : 0;
}

// The line's beginning: a run of sequences per thread (kRuns threads), the work in front of every run in run_cost and the
// whole in run_cost[kRuns] (kRuns + 1 + kRuns / 32 entries in shared memory).  A __syncthreads has to follow.
template <int kRuns>
__device__ __forceinline__ void lay_line(const TcParams& tp, float* run_cost) {
  const AttentionParams& p = tp.p;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, per = (p.num_seqs + kRuns - 1) / kRuns;
  float* warp_cost = run_cost + kRuns + 1;
  float cost = 0.f;
#pragma unroll 1
  for (int i = threadIdx.x * per; i < min(((int)threadIdx.x + 1) * per, p.num_seqs); ++i) {
    const SeqRange s = sequence(p, i);
    if (s.bad && p.status && blockIdx.x == 0) p.status[i] = TOPLOC_SEQ_BAD_LENGTH;
    const Line line(tp, s);
    cost += line.upto(line.levels) * (float)p.kv_heads;
  }
  float incl = cost;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const float up = __shfl_up_sync(0xFFFFFFFFu, incl, off);
    if (lane >= off) incl += up;
  }
  const float before_lane = __shfl_up_sync(0xFFFFFFFFu, incl, 1);
  if (lane == 31) warp_cost[warp] = incl;
  __syncthreads();
  float in_front = 0.f;
#pragma unroll 1
  for (int w = 0; w < warp; ++w) in_front += warp_cost[w];
  run_cost[threadIdx.x] = in_front + (lane > 0 ? before_lane : 0.f);
  if (threadIdx.x == kRuns - 1) run_cost[kRuns] = in_front + incl;
  fence_async_shared();  // tensor copies write there next
}

// Where the stretches of this block and of the next one begin (lane 0 and 1 of a warp look for one each; all get both).
// A cut in front of a level's second tile or behind its last but one moves to the level's ends (so a level of three tiles
// is never cut).
struct Stretch {
  Place begin, end;
};

template <int kRuns>
__device__ __forceinline__ Stretch find_stretch(const TcParams& tp, const float* run_cost) {
  const AttentionParams& p = tp.p;
  const int per = (p.num_seqs + kRuns - 1) / kRuns, lane = threadIdx.x & 31;
  const int block = blockIdx.x + min(lane, 1);
  const float all_work = run_cost[kRuns];
  const float share = all_work * tp.share_scale;
  const int piece = share >= (float)(4 * kKeyTile * tp.piece) ? 1 : tp.piece;
  float at = share * (float)block;
  Place place = {p.num_seqs, 0, 0, 0};
  if (at < all_work && block < gridDim.x) {  // (the last block's stretch ends with the line, whatever the rounding)
    int lo = 0, hi = kRuns;                  // run_cost[lo] <= at < run_cost[hi]
#pragma unroll 1
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (run_cost[mid] <= at) lo = mid; else hi = mid;
    }
    at -= run_cost[lo];
#pragma unroll 1
    for (int i = lo * per; i < p.num_seqs; ++i) {
      const SeqRange s = sequence(p, i);
      const Line line(tp, s);
      const float one = line.upto(line.levels), all = one * (float)p.kv_heads;
      if (at >= all) {
        at -= all;
        continue;
      }
      const int head = min((int)__fdividef(at, one), p.kv_heads - 1);
      at = max(at - (float)head * one, 0.f);
      int a = 0, b = line.levels;  // upto(a) <= at < upto(b)
#pragma unroll 1
      while (b - a > 1) {
        const int mid = (a + b) >> 1;
        if (line.upto(mid) <= at) a = mid; else b = mid;
      }
      at -= line.upto(a);
      const int n = tiles_seen(s, min((a + 1) * tp.item_tokens, s.rows));
      const int near = (int)max((at - kLevelCost) * (1.f / kKeyTile) + 0.5f, 0.f), tile = (near + piece / 2) & -piece;
      place = Place{i, head, a, tile <= 1 ? 0 : tile};
      if (tile > 1 && tile >= n - 1) {
        place.tile = 0;
        if (++place.level == line.levels) {
          place.level = 0;
          if (++place.head == p.kv_heads) place = Place{i + 1, 0, 0, 0};
        }
      }
      break;
    }
  }
  __syncwarp();
  const auto of = [&](int l) {
    return Place{__shfl_sync(0xFFFFFFFFu, place.seq, l), __shfl_sync(0xFFFFFFFFu, place.head, l),
                 __shfl_sync(0xFFFFFFFFu, place.level, l), __shfl_sync(0xFFFFFFFFu, place.tile, l)};
  };
  return Stretch{of(0), of(1)};
}

// A warp's walk over its block's stretch: the items one after the other.
struct Walk {
  const TcParams& tp;
  Place at, end;
  SeqRange s = {0, 0, 0, false};
  int s_of = -1;

  __device__ Walk(const TcParams& tp) : tp(tp), at{0, 0, 0, 0}, end{0, 0, 0, 0} {}

  template <int kRuns>
  __device__ void begin(const float* run_cost) {
    const Stretch stretch = find_stretch<kRuns>(tp, run_cost);
    at = stretch.begin;
    end = stretch.end;
    if ((threadIdx.x & 31) < 2) tp.parts[2 * blockIdx.x + (threadIdx.x & 31)].seq = -1;
    __syncwarp();  // (run_cost has been read: the ring's place is free)
  }

  // The next item (seq -1 and false: there is none), the same in every lane; notes the part that it leaves.
  __device__ bool next(Item& im) {
    const AttentionParams& p = tp.p;
    im = Item{};
    im.seq = -1;
#pragma unroll 1
    for (;; at = Place{at.seq + 1, 0, 0, 0}) {  // past the sequences without rows
      if (!before(at, end)) return false;
      if (s_of != at.seq) {
        s = sequence(p, at.seq);
        s_of = at.seq;
      }
      if (s.rows > 0) break;
    }
    const int tokens = min((at.level + 1) * tp.item_tokens, s.rows);
    im.seq = at.seq;
    im.head = at.head;
    im.first = s.first;
    im.behind = s.keys - s.rows;
    im.row0 = at.level * tp.item_rows;
    im.rows = s.rows * p.group;
    const bool ends_here = end.seq == at.seq && end.head == at.head && end.level == at.level;
    const int tile_end = ends_here ? end.tile : tiles_seen(s, tokens);
    im.kbegin = at.tile * kKeyTile;
    im.kend = min(min(s.keys, im.behind + tokens), tile_end * kKeyTile);
    im.two = im.row0 + tp.tile_rows < im.rows;
    if (im.two) {
      const int first = tiles_seen(s, at.level * tp.item_tokens + tp.tile_tokens);
      im.n0 = max(min(first, tile_end) - at.tile, 0);
      im.n1 = max(tile_end - at.tile, 0);
    } else {
      im.n0 = max(tile_end - at.tile, 0);
    }
    im.clean = max(im.behind + at.level * tp.item_tokens + 1 - im.kbegin, 0) / kKeyTile;
    im.slot = at.tile > 0 ? 0 : ends_here ? 1 : -1;
    if (im.slot >= 0 && (threadIdx.x & 31) == 0)
      tp.parts[2 * blockIdx.x + im.slot] = Part{im.seq, im.head, im.row0, im.first, im.rows, ends_here ? 0 : 1};
    at.tile = 0;
    if (ends_here) {
      at = end;
    } else if (tp.item_rows * (++at.level) >= im.rows) {
      at.level = 0;
      if (++at.head == p.kv_heads) at = Place{at.seq + 1, 0, 0, 0};
    }
    return true;
  }
};

// The block ends early: nothing in its stretch counts.  The sequences of the stretch are flagged and their rows there become
// NaN, so that the failure shows without a status too; of a row tile that other blocks share in, the part's lse does, which
// makes the joined rows NaN whatever an earlier call has left in the workspace (the records of the parts are written again:
// the block may have given up in front of them).  By a whole warp, all roles having left their loops.
__device__ __noinline__ void abandon(const TcParams& tp, const Stretch& stretch) {
  const AttentionParams& p = tp.p;
  const int lane = threadIdx.x & 31;
  Walk walk(tp);
  walk.at = stretch.begin;
  walk.end = stretch.end;
  Item im;
#pragma unroll 1
  while (walk.next(im)) {
    if (p.status && lane == 0) p.status[im.seq] = TOPLOC_SEQ_WAIT_EXPIRED;
#pragma unroll 1
    for (int r = lane; r < min(tp.item_rows, im.rows - im.row0); r += 32) {
      if (im.slot >= 0) {
        p.part_lse[((long long)blockIdx.x * 2 + im.slot) * tp.item_rows + r] = NAN;
        continue;
      }
      const int token = (im.row0 + r) / p.group, head = im.head * p.group + im.row0 + r - token * p.group;
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.out) + (im.first + token) * p.out_token + head * p.out_head;
#pragma unroll 1
      for (int c = 0; c < p.head_dim; ++c) out[c] = __float2bfloat16_rn(NAN);
      if (p.lse) p.lse[(long long)(im.first + token) * p.q_heads + head] = NAN;
    }
  }
}

// One warp's copies into the ring: the keys, or the values, of item after item.
template <typename S>
struct Feeder {
  static constexpr int kStages = S::kStages;
  const TcParams& tp;
  const CUtensorMap* map;
  typename S::Head& sh;
  uint32_t ring, base = 0;             // places in front of the item
  volatile int* gave_up;
  Item im;
  int tiles = 0, page = 0, next = 0, lane = threadIdx.x & 31;
  bool fine = true;

  __device__ Feeder(const TcParams& tp, const CUtensorMap* map, typename S::Head& sh, void* ring, volatile int* gave_up)
      : tp(tp), map(map), sh(sh), ring(shared_address(ring)), gave_up(gave_up) {}

  // The page of this lane's copy of tile j, as the table has it (looked up ahead of its use).
  __device__ int page_of(int j) const {
    const int key = im.kbegin + j * kKeyTile + lane * tp.box_rows;
    const bool copied = tp.p.kv_lens && j < tiles && lane * tp.box_rows < kKeyTile && key < im.kend;
    const int col = tp.box_rows < kKeyTile ? key >> tp.page_shift : (unsigned)(key / kKeyTile) / (unsigned)tp.page_tiles;
    return copied ? tp.p.table[im.seq * tp.p.table_stride + col] : 0;
  }

  __device__ void item(const Item& next_item, int n) {
    base += 2 * tiles;
    im = next_item;
    tiles = n;
#pragma unroll 1
    for (int j = 0; j < 2; ++j) {
      page = next;
      next = page_of(j);
    }
  }

  __device__ void feed(int j, int at) {
    const uint32_t place = base + at, stage = ring_stage(place, kStages);
    const uint32_t bar = shared_address(&sh.full[stage]), dst = ring + stage * S::kTileBytes;
    const int after = page_of(j + 2);
    fine = warp_wait(sh.empty[stage], ring_parity(place, kStages) ^ 1, gave_up);
    if (!fine) return;
    if (lane == 0) sh.fed[stage] = place + 1;  // (the other feeding warp's word too: a stage's copies follow one another)
    const int key0 = im.kbegin + j * kKeyTile;
    if (tp.p.kv_lens) {
      if (page < 0 || page >= tp.p.num_pages) {
        if (tp.p.status) tp.p.status[im.seq] = TOPLOC_SEQ_BAD_PAGE;
        page = tp.p.num_pages;  // past the end: the copy fills zeros
      }
      const int copies = (min(kKeyTile, im.kend - key0) + tp.box_rows - 1) / tp.box_rows;
      const int in_page = tp.page_tiles > 1 ? (unsigned)(key0 / kKeyTile) % (unsigned)tp.page_tiles * kKeyTile : 0;
      if (elect_one()) barrier_arrive_expect(bar, copies * S::kHalves * tp.box_rows * 128);
      __syncwarp();
#pragma unroll 1
      for (int c = 0; c < copies; ++c) {
        const int which = __shfl_sync(0xFFFFFFFFu, page, c);
        if (elect_one()) {
#pragma unroll
          for (int h = 0; h < S::kHalves; ++h)
            copy_4d(dst + h * kBlockBytes + c * tp.box_rows * 128, map, bar, h * 64, in_page, im.head, which);
        }
      }
    } else if (elect_one()) {
      barrier_arrive_expect(bar, S::kTileBytes);
#pragma unroll
      for (int h = 0; h < S::kHalves; ++h)
        copy_4d(dst + h * kBlockBytes, map, bar, h * 64, im.first + key0, im.head, 0);
    }
    __syncwarp();
    page = next;
    next = after;
  }
};

// The block ends early: a wait gave up, in whatever role, and all roles have left their loops (the threads are
// synchronised in front of this and behind it).  Copies have to land before the block ends, products to end before tensor
// memory is freed.  By a whole warp, the one that issued the products.
template <typename S>
__device__ __noinline__ void drain_block(typename S::Head& sh) {
  if (sh.queries_fed > 0) barrier_drain(shared_address(&sh.q_full), (sh.queries_fed - 1) & 1);
#pragma unroll 1
  for (int i = 0; i < S::kStages; ++i)  // (a stage's last copy: what the other feeding warp had there before has been used)
    if (sh.fed[i] > 0) barrier_drain(shared_address(&sh.full[i]), ring_parity(sh.fed[i] - 1, S::kStages));
  if (elect_one()) mma_commit(shared_address(&sh.drain));
  barrier_drain(shared_address(&sh.drain), 0);
}

__device__ __forceinline__ Item uniform(const Item& im) {  // the same for every lane, and known to be
  Item r;
  r.seq = __shfl_sync(0xFFFFFFFFu, im.seq, 0);
  r.head = __shfl_sync(0xFFFFFFFFu, im.head, 0);
  r.slot = __shfl_sync(0xFFFFFFFFu, im.slot, 0);
  r.first = __shfl_sync(0xFFFFFFFFu, im.first, 0);
  r.behind = __shfl_sync(0xFFFFFFFFu, im.behind, 0);
  r.row0 = __shfl_sync(0xFFFFFFFFu, im.row0, 0);
  r.rows = __shfl_sync(0xFFFFFFFFu, im.rows, 0);
  r.kbegin = __shfl_sync(0xFFFFFFFFu, im.kbegin, 0);
  r.kend = __shfl_sync(0xFFFFFFFFu, im.kend, 0);
  r.two = __shfl_sync(0xFFFFFFFFu, im.two, 0);
  r.n0 = __shfl_sync(0xFFFFFFFFu, im.n0, 0);
  r.n1 = __shfl_sync(0xFFFFFFFFu, im.n1, 0);
  r.clean = __shfl_sync(0xFFFFFFFFu, im.clean, 0);
  return r;
}

// Values of hidden keys meet weights of zero, and 0 * NaN is NaN.  Rows of a value tile past the item's keys (never
// loaded, or another sequence's: rows `keys` and on) become zero.  So does, in rows from `from` on, a value that is not
// finite; *bad gets the item's number then, and the rows that do see the key get the value back at the end.  By kThreads
// threads, number `me` of them this one; what follows has to wait for them all.
template <int kHalves, int kThreads>
__device__ __forceinline__ void clean_values(unsigned char* tile, int from, int keys, int me, int* bad, int number) {
#pragma unroll 1
  for (int e = me; e < (kKeyTile - from) * 8; e += kThreads) {
    const int row = from + (e >> 3);
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      uint4* at = reinterpret_cast<uint4*>(tile + h * kBlockBytes + row * 128 + (e & 7) * 16);
      if (row >= keys) {
        *at = make_uint4(0, 0, 0, 0);
      } else {
        const uint4 v = *at;
        // an exponent of all ones carries into the sign's place
        const uint32_t ones = ((v.x & 0x7F807F80u) + 0x00800080u) | ((v.y & 0x7F807F80u) + 0x00800080u) |
                              ((v.z & 0x7F807F80u) + 0x00800080u) | ((v.w & 0x7F807F80u) + 0x00800080u);
        if (ones & 0x80008000u) {
          *(volatile int*)bad = number;
          __threadfence_block();
          uint16_t* x = reinterpret_cast<uint16_t*>(at);
#pragma unroll 1
          for (int i = 0; i < 8; ++i)
            if ((x[i] & 0x7F80u) == 0x7F80u) x[i] = 0;
        }
      }
    }
  }
  fence_async_shared();
}

// Adds what clean_values took out of the values of keys begin .. end - 1 (NaN and infinities, as a rule nothing) to the
// channels c .. c + count - 1 of a row that sees these keys.  Not inlined: as good as never called.
__device__ __noinline__ void give_back(const AttentionParams& p, int seq, int key_head, int first, int begin, int end,
                                       int c, int count, float* out) {
#pragma unroll 1
  for (int key = begin; key < end; ++key) {
    const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(p.v) + (long long)key_head * p.v_head + c;
    if (p.kv_lens == nullptr) {
      v += (long long)(first + key) * p.v_token;
    } else {
      const int col = key / p.page_size, page = p.table[seq * p.table_stride + col];
      if (page < 0 || page >= p.num_pages) continue;
      v += page * p.v_page + (long long)(key - col * p.page_size) * p.v_token;
    }
#pragma unroll 1
    for (int e = 0; e < count; ++e) {
      const float f = __bfloat162float(v[e]);
      if (!(fabsf(f) < INFINITY)) out[e] += f;
    }
  }
}

}  // namespace

namespace toploc_model {

constexpr int kFewRows = 8;  // packed rows of a sequence that the kernel for few rows takes (figures: there)
// (tp: a TcParams, maps: CUtensorMap)
int launch_few_rows(const void* tp, const void* map_q, const void* map_k, const void* map_v, int blocks,
                    cudaStream_t stream);

}  // namespace toploc_model
