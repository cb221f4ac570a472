// What the tensor-core kernels of attention share: how the work is cut over the blocks, the feeding of keys and values
// by tensor copies, and the join of partial results.
#pragma once

#include "attention_common.cuh"
#include "sm100.cuh"

namespace {

using namespace toploc_model;
using namespace sm100;

constexpr int kItems = 4;                  // items announced ahead
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
};

// The parts a block leaves, for the join.
struct Part {
  int seq, head, row0, first, rows;  // seq -1: none
  int last;                          // slot 0: the row tile's keys end here
};

struct TcParams {
  AttentionParams p;
  int tile_rows;  // packed rows of a row tile: 128 rounded down to whole tokens
  int item_rows;  // packed rows of an item: two tiles (a few rows: all that a sequence can bring)
  int least_share;  // keys that are worth a block
  int box_rows;   // rows of a key copy
  int q_bytes;    // bytes of a query tile's copy
  bool wide_out;  // rows of the output at multiples of 32 bytes
  Part* parts;    // [blocks][2]
};

__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
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

constexpr long long kLevelCost = 192;

struct Line {
  long long front;  // kLevelCost + keys in front
  int rows_item, tokens_item, tokens, levels;
  __device__ Line(const TcParams& tp, const SeqRange& s)
      : front(kLevelCost + max(s.keys - s.rows, 0)), rows_item(tp.item_rows), tokens_item(rows_item / tp.p.group),
        tokens(s.rows), levels((s.rows + tokens_item - 1) / tokens_item) {}
  __device__ long long upto(int level) const {  // of levels 0 .. level - 1
    const long long whole = level * front + (long long)tokens_item * level * (level + 1) / 2;
    return level < levels ? whole : whole - ((long long)levels * tokens_item - tokens);
  }
};

// A place on the line: a key tile of a level.
struct Place {
  int seq, head, level, tile;
};

__device__ __forceinline__ bool before(const Place& a, const Place& b) {
  if (a.seq != b.seq) return a.seq < b.seq;
  if (a.head != b.head) return a.head < b.head;
  if (a.level != b.level) return a.level < b.level;
  return a.tile < b.tile;
}

// Key tiles that a level's rows see in all.
__device__ __forceinline__ int tiles_seen(const SeqRange& s, int tokens_upto) {
  const int seen = min(s.keys, s.keys - s.rows + tokens_upto);
  return seen > 0 ? (seen + kKeyTile - 1) / kKeyTile : 0;
}

// The line's beginning: a run of sequences per thread (kRuns threads), the work in front of every run in run_cost and the
// whole in run_cost[kRuns] (kRuns + 1 + kRuns / 32 entries in shared memory).  Ends with the writes on their way; a
// __syncthreads has to follow.
template <int kRuns>
__device__ __forceinline__ void lay_line(const TcParams& tp, long long* run_cost) {
  const AttentionParams& p = tp.p;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, per = (p.num_seqs + kRuns - 1) / kRuns;
  long long* warp_cost = run_cost + kRuns + 1;
  long long cost = 0;
  for (int i = threadIdx.x * per; i < min(((int)threadIdx.x + 1) * per, p.num_seqs); ++i) {
    const SeqRange s = sequence(p, i);
    if (s.bad && p.status && blockIdx.x == 0) p.status[i] = TOPLOC_SEQ_BAD_LENGTH;
    const Line line(tp, s);
    cost += line.upto(line.levels) * p.kv_heads;
  }
  long long incl = cost;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const long long up = __shfl_up_sync(0xFFFFFFFFu, incl, off);
    if (lane >= off) incl += up;
  }
  if (lane == 31) warp_cost[warp] = incl;
  __syncthreads();
  long long in_front = incl - cost;
  for (int w = 0; w < warp; ++w) in_front += warp_cost[w];
  run_cost[threadIdx.x] = in_front;
  if (threadIdx.x == kRuns - 1) run_cost[kRuns] = in_front + cost;
  fence_async_shared();  // tensor copies write there next
}

// Where the stretch of a block begins; a cut in front of a level's second tile or behind its last but one moves to the
// level's ends.
template <int kRuns>
__device__ __forceinline__ Place find_place(const TcParams& tp, const long long* run_cost, int block) {
  const AttentionParams& p = tp.p;
  const int per = (p.num_seqs + kRuns - 1) / kRuns;
  long long at = max((run_cost[kRuns] + gridDim.x - 1) / gridDim.x, (long long)tp.least_share) * block;
  if (at >= run_cost[kRuns]) return Place{p.num_seqs, 0, 0, 0};
  int lo = 0, hi = kRuns;  // run_cost[lo] <= at < run_cost[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (run_cost[mid] <= at) lo = mid; else hi = mid;
  }
  at -= run_cost[lo];
  for (int i = lo * per; i < p.num_seqs; ++i) {
    const SeqRange s = sequence(p, i);
    const Line line(tp, s);
    const long long one = line.upto(line.levels), all = one * p.kv_heads;
    if (at >= all) {
      at -= all;
      continue;
    }
    Place place = {i, (int)(at / one), 0, 0};
    at -= place.head * one;
    int a = 0, b = line.levels;  // upto(a) <= at < upto(b)
    while (b - a > 1) {
      const int mid = (a + b) >> 1;
      if (line.upto(mid) <= at) a = mid; else b = mid;
    }
    place.level = a;
    at -= line.upto(a);
    const int n = tiles_seen(s, min((a + 1) * line.tokens_item, line.tokens));
    const long long tile = (at - kLevelCost + kKeyTile / 2) / kKeyTile;
    if (at <= kLevelCost || tile <= 1) return place;
    if (tile >= n - 1) {
      if (++place.level == line.levels) {
        place.level = 0;
        if (++place.head == p.kv_heads) return Place{i + 1, 0, 0, 0};
      }
      return place;
    }
    place.tile = (int)tile;
    return place;
  }
  return Place{p.num_seqs, 0, 0, 0};
}

// A warp's walk over its block's stretch: the items one after the other.
struct Walk {
  const TcParams& tp;
  Place at, end;
  SeqRange s = {0, 0, 0, false};
  int s_of = -1;

  __device__ Walk(const TcParams& tp, const Place& begin, const Place& end) : tp(tp), at(begin), end(end) {
    if ((threadIdx.x & 31) < 2) tp.parts[2 * blockIdx.x + (threadIdx.x & 31)].seq = -1;
    __syncwarp();
  }

  // The next item (seq -1 and false: there is none), the same in every lane; notes the part that it leaves.
  __device__ bool next(Item& im) {
    const AttentionParams& p = tp.p;
    im = Item{};
    im.seq = -1;
    while (before(at, end)) {  // past the sequences without rows
      if (s_of != at.seq) {
        s = sequence(p, at.seq);
        s_of = at.seq;
      }
      if (s.rows > 0) break;
      at = Place{at.seq + 1, 0, 0, 0};
    }
    if (!before(at, end)) return false;
    const int tokens_item = tp.item_rows / p.group, tokens = min((at.level + 1) * tokens_item, s.rows);
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
      const int first = tiles_seen(s, at.level * tokens_item + tp.tile_rows / p.group);
      im.n0 = max(min(first, tile_end) - at.tile, 0);
      im.n1 = max(tile_end - at.tile, 0);
    } else {
      im.n0 = max(tile_end - at.tile, 0);
    }
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

// One warp's copies into the ring: the keys, or the values, of item after item.
template <typename S>
struct Feeder {
  static constexpr int kStages = S::kStages;
  const TcParams& tp;
  const CUtensorMap* map;
  typename S::Head& sh;
  uint32_t ring, base = 0;             // places in front of the item
  uint32_t fed = 0, fed_parity = 0;    // by stage: this warp's last copy there
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
    return copied ? tp.p.table[im.seq * tp.p.table_stride + key / tp.p.page_size] : 0;
  }

  __device__ void item(const Item& next_item, int n) {
    base += 2 * tiles;
    im = next_item;
    tiles = n;
    page = page_of(0);
    next = page_of(1);
  }

  __device__ void feed(int j, int at) {
    const uint32_t place = base + at, stage = ring_stage(place, kStages);
    const uint32_t bar = shared_address(&sh.full[stage]), dst = ring + stage * S::kTileBytes;
    const int after = page_of(j + 2);
    fine = warp_wait(sh.empty[stage], ring_parity(place, kStages) ^ 1, gave_up);
    if (!fine) return;
    fed |= 1u << stage;
    fed_parity = (fed_parity & ~(1u << stage)) | ring_parity(place, kStages) << stage;
    const int key0 = im.kbegin + j * kKeyTile;
    if (tp.p.kv_lens) {
      if (page < 0 || page >= tp.p.num_pages) {
        if (tp.p.status) tp.p.status[im.seq] = TOPLOC_SEQ_BAD_PAGE;
        page = tp.p.num_pages;  // past the end: the copy fills zeros
      }
      const int copies = (min(kKeyTile, im.kend - key0) + tp.box_rows - 1) / tp.box_rows;
      const int in_page = tp.box_rows < kKeyTile ? 0 : key0 % tp.p.page_size;
      if (elect_one()) barrier_arrive_expect(bar, copies * S::kHalves * tp.box_rows * 128);
      __syncwarp();
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

  // After a wait gave up: no copy of this warp is in flight when it returns.
  __device__ void drain() const {
    for (int i = 0; i < kStages; ++i)
      if (fed >> i & 1) barrier_drain(shared_address(&sh.full[i]), fed_parity >> i & 1);
  }
};

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
  return r;
}

// Values of hidden keys meet weights of zero, and 0 * NaN is NaN.  Rows of a value tile past the item's keys (never
// loaded, or another sequence's: rows `keys` and on) become zero.  So does, in rows from `from` on, a value that is not
// finite; *bad gets the item's number then, and the rows that do see the key get the value back at the end.  Called by
// 128 threads, each for its share; what follows has to wait for them all.
template <int kHalves>
__device__ __forceinline__ void clean_values(unsigned char* tile, int from, int keys, int* bad, int number) {
  for (int e = threadIdx.x & 127; e < (kKeyTile - from) * 8; e += 128) {
    const int row = from + (e >> 3);
    const bool past = row >= keys;
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      uint4* at = reinterpret_cast<uint4*>(tile + h * kBlockBytes + row * 128 + (e & 7) * 16);
      uint4 v = make_uint4(0, 0, 0, 0);
      bool write = past;
      if (!past) {
        v = *at;
        uint32_t* x = &v.x;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if ((x[q] & 0x7F80u) == 0x7F80u) x[q] &= 0xFFFF0000u, write = true;
          if ((x[q] & 0x7F800000u) == 0x7F800000u) x[q] &= 0xFFFFu, write = true;
        }
        if (write) {
          *(volatile int*)bad = number;
          __threadfence_block();
        }
      }
      if (write) *at = v;
    }
  }
  fence_async_shared();
}

// Value [key] of a sequence and key head (first channel), NULL where its page lies outside the cache.
__device__ __forceinline__ const __nv_bfloat16* value_of(const AttentionParams& p, const Item& im, int key) {
  const __nv_bfloat16* v = static_cast<const __nv_bfloat16*>(p.v) + (long long)im.head * p.v_head;
  if (p.kv_lens == nullptr) return v + (long long)(im.first + key) * p.v_token;
  const int col = key / p.page_size, page = p.table[im.seq * p.table_stride + col];
  if (page < 0 || page >= p.num_pages) return nullptr;
  return v + page * p.v_page + (long long)(key - col * p.page_size) * p.v_token;
}

}  // namespace

namespace toploc_model {

constexpr int kFewRows = 32;  // packed rows of a sequence that the kernel for few rows takes
// (tp: a TcParams, maps: CUtensorMap)
int launch_few_rows(const void* tp, const void* map_q, const void* map_k, const void* map_v, int blocks,
                    cudaStream_t stream);

}  // namespace toploc_model
