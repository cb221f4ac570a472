// Pages that sequences share, give back or move: forks, releases, the compaction of a pool, and the copies of pages that
// follow from them.
//
// The planners move little (a table's entries and an integer or two a page) and have to agree on counts between their steps.
// Each is one launch of one block, or of one cluster of eight where there is more to do: the barriers are the hardware's, so no
// block spins on another, and a step's counts go through the blocks' shared memory.  A row of the table belongs to the same
// warp of all blocks, its columns to the blocks in turn; a page belongs to one warp, in ascending order, so that what is
// numbered comes out in order whatever the atomics' order was.
//
// Small plans are bound by latency: steps of dependent loads from L2, and code that is fetched for the first time (so little is
// unrolled).  One block's barriers take a tenth of a cluster's (1000 to 3000 clocks each).
#include "model_common.cuh"

#include <cooperative_groups.h>

namespace {

using namespace toploc_model;
namespace cg = cooperative_groups;

constexpr int kMostBlocks = 8;                 // of a planner's cluster
constexpr int kThreads = 1024;
constexpr int kWarps = kThreads / 32;          // of a block
// Entries of the table (at most: its width is known on the host, what is held is not) and pages that one block plans for; in
// tables little wider than their longest sequence a cluster of eight is faster from there on (releases of
// 4, 8, 15 and 57 thousand: 5.0, 5.6, 7.7 and 15.5 us against 6.3, 6.3, 6.6 and 8.0; forks of 1, 5 and 18: 7.5, 9.9 and 17.8
// against 8.7, 9.7 and 10.0; compactions of 1, 6 and 12: 9.0, 12.0 and 16.2 against 11.4, 13.1 and 14.3).
constexpr long long kOneBlock = 8192;
// And of a release that one cluster does.  Three launches over all SMs are faster on the GPU from 50 thousand on (57, 112 and
// 412 thousand: 7.5, 8.4 and 11.9 us against 8.0, 10.7 and 22.2), but take 4 us more of the calling thread.
constexpr long long kOneCluster = 131072;
constexpr int kAtOnce = 4;                     // loads of a thread on their way at once

struct PoolParams {
  const int32_t* parents;    // fork
  const uint8_t* release;    // release
  const int32_t* kv_lens;
  const int32_t* shares;
  const int32_t* free_in;    // fork
  const int32_t* first_free; // fork, release
  const int32_t* table_in;   // compact
  int32_t* table;            // fork: in and out; release: in; compact: out
  int32_t* kv_lens_out;
  int32_t* shares_out;
  int32_t* free_out;         // release, compact
  int32_t* copy_from;
  int32_t* copy_to;
  int32_t* num_copies;
  int32_t* next_free;
  uint8_t* status;
  long long table_stride, table_in_stride;
  int num_seqs, num_pages, num_free, page_size, max_pages;
};

__device__ __forceinline__ int pages_for(int tokens, int page_size) {
  return (int)(((unsigned)tokens + (unsigned)page_size - 1u) / (unsigned)page_size);
}

// What another block of the cluster may have written since: from L2.
__device__ __forceinline__ int32_t fresh(const int32_t* p) { return __ldcg(p); }

__device__ __forceinline__ int warp_total(int v) { return __reduce_add_sync(0xFFFFFFFFu, v); }

// Pages of a sequence that a release or a compaction goes by, and what is wrong with its length.
__device__ __forceinline__ int held_pages(const PoolParams& p, int len, int* status) {
  *status = TOPLOC_SEQ_OK;
  if (len < 0) {
    *status = TOPLOC_SEQ_BAD_LENGTH;
    return 0;
  }
  const int pages = pages_for(len, p.page_size);
  if (pages > p.max_pages) *status = TOPLOC_SEQ_BAD_LENGTH;
  return min(pages, p.max_pages);
}

// The planner's threads: one block, or the blocks of one cluster.
struct Team {
  int blocks, block, all_warps, all_threads, warp_of_all, all_tid;

  __device__ __forceinline__ Team() {
    const cg::cluster_group cluster = cg::this_cluster();
    blocks = (int)cluster.num_blocks();
    block = (int)cluster.block_rank();
    all_warps = blocks * kWarps;
    all_threads = blocks * kThreads;
    all_tid = block * kThreads + (int)threadIdx.x;
    warp_of_all = all_tid >> 5;
  }
  __device__ __forceinline__ void sync() const {
    if (blocks == 1)
      __syncthreads();
    else
      cg::this_cluster().sync();
  }
};

// Entries of the rows' held pages, kAtOnce rows of a warp together: visit(rows, column, pages, valid), arrays of kAtOnce; all
// lanes of a warp together.  held(row): pages of a row (its length is read by one lane a row).
template <typename Held, typename Visit>
__device__ __forceinline__ void for_entries(const PoolParams& p, const Team& team, const int32_t* table, long long stride,
                                            Held held, Visit visit) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll 1
  for (int base = warp; base < p.num_seqs; base += kWarps * 32) {
    const int row = base + lane * kWarps;
    const int mine = row < p.num_seqs ? held(row) : 0;
    const int count = min(32, (p.num_seqs - base + kWarps - 1) / kWarps);
#pragma unroll 1
    for (int first = 0; first < count; first += kAtOnce) {
      int rows[kAtOnce], held_of[kAtOnce], most = 0;
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        rows[i] = base + (first + i) * kWarps;
        held_of[i] = __shfl_sync(0xFFFFFFFFu, mine, (first + i) & 31);
        if (first + i >= count) held_of[i] = 0;
        most = max(most, held_of[i]);
      }
#pragma unroll 1
      for (unsigned c0 = team.block * 32; c0 < (unsigned)most; c0 += team.blocks * 32) {  // (rows of up to 2^31 - 1)
        int32_t page[kAtOnce];
        bool valid[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          valid[i] = c0 + lane < (unsigned)held_of[i];
          page[i] = valid[i] ? table[rows[i] * stride + c0 + lane] : 0;
        }
        visit(rows, c0 + lane, page, valid);
      }
    }
  }
}

// The range of pages of one warp of the team, whole groups of 32.
__device__ __forceinline__ int groups_each(const PoolParams& p, const Team& team) {
  return ((p.num_pages + 31) / 32 + team.all_warps - 1) / team.all_warps;
}
__device__ __forceinline__ void pages_of_warp(const PoolParams& p, int each, int warp_of_all, int* begin, int* end) {
  *begin = (int)min((long long)warp_of_all * each * 32, (long long)p.num_pages);
  *end = (int)min((long long)*begin + each * 32, (long long)p.num_pages);
}

// Calls visit(page, value) for the pages of a warp's range in groups of 32, in order, all lanes together (value 0 past the
// end).
template <typename Visit>
__device__ __forceinline__ void for_pages(const int32_t* values, int begin, int end, Visit visit) {
  const int lane = threadIdx.x & 31;
#pragma unroll 1
  for (int base = begin; base < end; base += 32 * kAtOnce) {
    int32_t v[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const int i = base + k * 32 + lane;
      v[k] = i < end ? fresh(values + i) : 0;
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k)
      if (base + k * 32 < end) visit(base + k * 32 + lane, v[k]);
  }
}

// Copies a vector, the team's threads side by side.
__device__ __forceinline__ void copy_vector(int32_t* to, const int32_t* from, int count, const Team& team) {
#pragma unroll 1
  for (long long i = team.all_tid; i < count; i += (long long)team.all_threads * kAtOnce) {
    int32_t v[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k)
      if (i + k * team.all_threads < count) v[k] = from[i + k * team.all_threads];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k)
      if (i + k * team.all_threads < count) to[i + k * team.all_threads] = v[k];
  }
}

// Every warp's count to all blocks: counts[w] of every warp of the team in shared memory, behind a barrier of the team.
__device__ __forceinline__ void tell_count(const Team& team, int* counts, int count) {
  const int lane = threadIdx.x & 31;
  if (lane < team.blocks) cg::this_cluster().map_shared_rank(counts, lane)[team.warp_of_all] = count;
}

// Sum of the counts in front of a warp and of all, for all lanes.
__device__ __forceinline__ int counted_before(const Team& team, const int* counts, int warp_of_all, int* all) {
  const int lane = threadIdx.x & 31;
  int before = 0, total = 0;
  for (int i = lane; i < team.all_warps; i += 32) {
    const int c = counts[i];
    total += c;
    if (i < warp_of_all) before += c;
  }
  *all = warp_total(total);
  return warp_total(before);
}

// Exclusive prefix sum over the block's threads; *total gets the sum.
__device__ __forceinline__ int block_scan(int v, int* warp_sums, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int incl = v;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int up = __shfl_up_sync(0xFFFFFFFFu, incl, off);
    if (lane >= off) incl += up;
  }
  if (lane == 31) warp_sums[warp] = incl;
  __syncthreads();
  int before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const int s = warp_sums[w];
    if (w < warp) before += s;
    sum += s;
  }
  __syncthreads();
  *total = sum;
  return before + incl - v;
}

// ---- forks ---------------------------------------------------------------------------------------

constexpr int kNeedsPage = 0x80;  // of a status byte until the end: the child asks for a page

__device__ __forceinline__ int status_of(const PoolParams& p, int i) { return __ldcg(p.status + i); }

// Pages that the children in front of i ask for; all lanes of a warp together.
__device__ __forceinline__ int asked_before(const PoolParams& p, const int* run_before, int per, int i) {
  int more = 0;
  for (int j = i / per * per + (threadIdx.x & 31); j < i; j += 32) more += status_of(p, j) >> 7;
  return run_before[i / per] + warp_total(more);
}

__global__ void __launch_bounds__(kThreads, 1) toploc_fork_pages_kernel(const __grid_constant__ PoolParams p) {
  __shared__ int warp_sums[kWarps], run_before[kThreads];
  const Team team;
  const int tid = threadIdx.x, lane = tid & 31, all_tid = team.all_tid;

  asm volatile("griddepcontrol.launch_dependents;");  // the copies may get ready

  // who can be forked: a lane a sequence, then the warp a parent's row
  copy_vector(p.shares_out, p.shares, p.num_pages, team);
#pragma unroll 1
  for (int base = team.warp_of_all; base < p.num_seqs; base += team.all_warps * 32) {
    const int i = base + lane * team.all_warps;
    int parent = -1, status = TOPLOC_SEQ_OK, own = 0, len = 0, pages = 0;
    if (i < p.num_seqs) {
      parent = p.parents[i];
      own = len = p.kv_lens[i];
    }
    if (parent >= 0) {
      const bool there = parent < p.num_seqs;
      const int theirs = there ? p.kv_lens[parent] : 0;
      if (!there || p.parents[parent] >= 0) {
        status = TOPLOC_SEQ_BAD_PARENT;
      } else if (own != 0) {
        status = TOPLOC_SEQ_IN_USE;
      } else {
        pages = held_pages(p, theirs, &status);
        len = theirs;
        if (status == TOPLOC_SEQ_OK && len % p.page_size > 0) status = kNeedsPage;
      }
    }
    if ((status & ~kNeedsPage) != TOPLOC_SEQ_OK) len = own, pages = 0;
    const int most = __reduce_max_sync(0xFFFFFFFFu, pages);
    if (most > 0) {  // entries outside the pool, of all the lanes' parents
      const int count = min(32, (p.num_seqs - base + team.all_warps - 1) / team.all_warps);
#pragma unroll 1
      for (int first = 0; first < count; first += kAtOnce) {
        bool bad[kAtOnce] = {};
        int from[kAtOnce];
        unsigned held[kAtOnce], longest = 0;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
          held[k] = first + k < 32 ? __shfl_sync(0xFFFFFFFFu, pages, (first + k) & 31) : 0;
          from[k] = __shfl_sync(0xFFFFFFFFu, parent, (first + k) & 31);
          longest = max(longest, held[k]);
        }
#pragma unroll 1
        for (unsigned j = lane; j < longest; j += 32) {
          int32_t page[kAtOnce];
#pragma unroll
          for (int k = 0; k < kAtOnce; ++k) page[k] = j < held[k] ? p.table[from[k] * p.table_stride + j] : 0;
#pragma unroll
          for (int k = 0; k < kAtOnce; ++k) bad[k] = bad[k] || (j < held[k] && (unsigned)page[k] >= (unsigned)p.num_pages);
        }
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k)
          if (__any_sync(0xFFFFFFFFu, bad[k]) && lane == first + k) status = TOPLOC_SEQ_BAD_PAGE, len = own;
      }
    }
    if (i < p.num_seqs) {
      p.kv_lens_out[i] = len;
      p.status[i] = (uint8_t)status;
    }
  }
  team.sync();

  // pages asked for in front of every thread's run of sequences (every block for itself)
  const int per = max(1, (p.num_seqs + kThreads - 1) / kThreads);
  const int begin = min(tid * per, p.num_seqs), end = min(begin + per, p.num_seqs);
  int asked = 0, total;
  for (int i = begin; i < end; ++i) asked += status_of(p, i) >> 7;
  run_before[tid] = block_scan(asked, warp_sums, &total);
  __syncthreads();
  const int head = p.first_free[0];
  const int room = head < 0 ? 0 : max(0, p.num_free - head), taken = min(total, room);
  if (all_tid == 0) {
    p.num_copies[0] = taken;
    p.next_free[0] = head + taken;
  }
  for (int i = taken + all_tid; i < p.num_seqs; i += team.all_threads) p.copy_from[i] = p.copy_to[i] = -1;

  // the children's rows (a status keeps its mark for those that still count)
  for (int i = team.warp_of_all; i < p.num_seqs; i += team.all_warps) {
    const int parent = p.parents[i], was = status_of(p, i);
    if (parent < 0 || (was & ~kNeedsPage) != TOPLOC_SEQ_OK) continue;
    const unsigned whole = (unsigned)fresh(p.kv_lens_out + i) / (unsigned)p.page_size;
    const int32_t* theirs = p.table + parent * p.table_stride;
    int32_t* row = p.table + i * p.table_stride;
    int status = TOPLOC_SEQ_OK;
    if (was == kNeedsPage) {
      const int place = asked_before(p, run_before, per, i);
      if (place >= room) {
        status = TOPLOC_SEQ_NO_PAGES;
      } else {
        const int32_t page = p.free_in[head + place];
        if ((unsigned)page >= (unsigned)p.num_pages) status = TOPLOC_SEQ_BAD_PAGE;
        if (lane == 0) {
          if (status == TOPLOC_SEQ_OK) row[whole] = page;
          p.copy_from[place] = status == TOPLOC_SEQ_OK ? theirs[whole] : -1;
          p.copy_to[place] = status == TOPLOC_SEQ_OK ? page : -1;
        }
      }
      if (status != TOPLOC_SEQ_OK && lane == 0) p.status[i] = (uint8_t)(status | kNeedsPage);
    }
    if (status != TOPLOC_SEQ_OK) continue;
    for (unsigned j0 = lane; j0 < whole; j0 += 32 * kAtOnce) {
      int32_t page[kAtOnce];
#pragma unroll
      for (int e = 0; e < kAtOnce; ++e) page[e] = j0 + e * 32 < whole ? theirs[j0 + e * 32] : 0;
#pragma unroll
      for (int e = 0; e < kAtOnce; ++e) {
        if (j0 + e * 32 >= whole) break;
        row[j0 + e * 32] = page[e];
        atomicAdd(p.shares_out + page[e], 1);
      }
    }
  }
  team.sync();
  for (int i = all_tid; i < p.num_seqs; i += team.all_threads) {
    const int was = status_of(p, i);
    if (was & kNeedsPage) {
      p.status[i] = (uint8_t)(was & ~kNeedsPage);
      if (was != kNeedsPage) p.kv_lens_out[i] = p.kv_lens[i];
    }
  }
}

// ---- releases ------------------------------------------------------------------------------------

// What a sequence's length and status become; pages of those that are released.
__device__ __forceinline__ void release_sequence(const PoolParams& p, int i) {
  const int len = p.kv_lens[i];
  int status = TOPLOC_SEQ_OK;
  const bool gone = p.release[i] != 0;
  if (gone) held_pages(p, len, &status);
  p.kv_lens_out[i] = gone ? 0 : len;
  p.status[i] = (uint8_t)status;
}
__device__ __forceinline__ int released_pages(const PoolParams& p, int i) {
  int status;
  return p.release[i] != 0 ? held_pages(p, p.kv_lens[i], &status) : 0;
}
// A holder less; below zero: nobody is left.
__device__ __forceinline__ void release_entry(const PoolParams& p, int seq, int32_t page) {
  if ((unsigned)page < (unsigned)p.num_pages)
    atomicSub(p.shares_out + page, 1);
  else
    p.status[seq] = TOPLOC_SEQ_BAD_PAGE;
}

// Large releases take three launches: an SM sends an atomic every other clock, so the sequences' pages (65 thousand take eight
// SMs 10 us) are spread over all SMs, and so is the copy of the shares; the numbering behind them stays with the cluster.
constexpr int kWideThreads = 256;
constexpr int kEntriesAtOnce = 32 * kAtOnce;  // of a row, a warp's

__global__ void __launch_bounds__(kWideThreads) toploc_release_begin_kernel(const __grid_constant__ PoolParams p) {
  asm volatile("griddepcontrol.launch_dependents;");
  const int all = gridDim.x * kWideThreads, tid = blockIdx.x * kWideThreads + threadIdx.x;
  for (long long i = tid; i < p.num_pages; i += all) p.shares_out[i] = p.shares[i];
  for (int i = tid; i < p.num_seqs; i += all) release_sequence(p, i);
}

__global__ void __launch_bounds__(kWideThreads) toploc_release_entries_kernel(const __grid_constant__ PoolParams p) {
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31, parts = ((unsigned)p.max_pages + kEntriesAtOnce - 1) / kEntriesAtOnce;
  const long long warps = gridDim.x * (kWideThreads / 32), items = (long long)p.num_seqs * parts;
  for (long long item = blockIdx.x * (kWideThreads / 32) + threadIdx.x / 32; item < items; item += warps) {
    const int seq = (int)(item / parts);
    const unsigned first = (unsigned)(item - (long long)seq * parts) * kEntriesAtOnce + lane;
    const unsigned pages = released_pages(p, seq);
    int32_t page[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k)
      if (first + k * 32 < pages) page[k] = p.table[seq * p.table_stride + first + k * 32];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k)
      if (first + k * 32 < pages) release_entry(p, seq, page[k]);
  }
}

// kAll: the whole release, else what is left to do behind the two kernels above.
template <bool kAll>
__global__ void __launch_bounds__(kThreads, 1) toploc_release_pages_kernel(const __grid_constant__ PoolParams p) {
  __shared__ int counts[kMostBlocks * kWarps];
  const Team team;
  const int lane = threadIdx.x & 31, all_tid = team.all_tid;

  if constexpr (kAll) {
    copy_vector(p.shares_out, p.shares, p.num_pages, team);
    for (int i = all_tid; i < p.num_seqs; i += team.all_threads) release_sequence(p, i);
    team.sync();
    for_entries(
        p, team, p.table, p.table_stride, [&](int row) { return released_pages(p, row); },
        [&](const int* rows, unsigned, const int32_t* page, const bool* valid) {
#pragma unroll
          for (int i = 0; i < kAtOnce; ++i)
            if (valid[i]) release_entry(p, rows[i], page[i]);
        });
  } else {
    asm volatile("griddepcontrol.wait;" ::: "memory");
  }
  team.sync();

  // the pages that came back: counted, then numbered in order
  int begin, end, count = 0, total;
  const int each = groups_each(p, team);
  pages_of_warp(p, each, team.warp_of_all, &begin, &end);
  unsigned mine = 0;  // lane k: those of the range's k-th group of 32
  int group = 0;
  for_pages(p.shares_out, begin, end, [&](int, int left) {
    const unsigned freed = __ballot_sync(0xFFFFFFFFu, left < 0);
    if (lane == group) mine = freed;
    count += __popc(freed);
    ++group;
  });
  tell_count(team, counts, count);
  team.sync();

  int place = counted_before(team, counts, team.warp_of_all, &total);
  const int room = min(max(p.first_free[0], 0), p.num_free), fit = min(total, room);
  const auto give_back = [&](int i, unsigned freed) {
    if (freed >> lane & 1) {
      const int at = place + __popc(freed & ((1u << lane) - 1));
      if (at < fit) p.free_out[room - fit + at] = i;
      p.shares_out[i] = 0;
    }
    place += __popc(freed);
  };
  if (each <= 32) {
    for (int k = 0; k < group; ++k) give_back(begin + k * 32 + lane, __shfl_sync(0xFFFFFFFFu, mine, k));
  } else {
    for_pages(p.shares_out, begin, end, [&](int i, int left) { give_back(i, __ballot_sync(0xFFFFFFFFu, left < 0)); });
  }
  if (all_tid == 0) p.next_free[0] = room - fit;
  if (total > room) {
    for (int i = all_tid; i < p.num_seqs; i += team.all_threads)
      if (released_pages(p, i) > 0 && status_of(p, i) == TOPLOC_SEQ_OK) p.status[i] = TOPLOC_SEQ_NO_ROOM;
  }
}

// ---- compaction ----------------------------------------------------------------------------------

// While it runs, shares_out holds marks: 0 for unused pages, 1 for used ones, 1 + number of the copy for those that move.
__global__ void __launch_bounds__(kThreads, 1) toploc_compact_pages_kernel(const __grid_constant__ PoolParams p) {
  __shared__ int counts[kMostBlocks * kWarps];
  const Team team;
  const int lane = threadIdx.x & 31, all_tid = team.all_tid;
  int32_t* marks = p.shares_out;
  asm volatile("griddepcontrol.launch_dependents;");  // the copies may get ready

  for (int i = all_tid; i < p.num_pages; i += team.all_threads) {
    marks[i] = 0;
    p.copy_from[i] = p.copy_to[i] = -1;
  }
  for (int i = all_tid; i < p.num_seqs; i += team.all_threads) {
    int status;
    held_pages(p, p.kv_lens[i], &status);
    p.status[i] = (uint8_t)status;
  }
  team.sync();

  const auto held = [&](int row) {
    int status;
    return held_pages(p, p.kv_lens[row], &status);
  };
  for_entries(p, team, p.table_in, p.table_in_stride, held,
              [&](const int* rows, unsigned, const int32_t* page, const bool* valid) {
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) {
                  if (!valid[i]) continue;
                  if ((unsigned)page[i] < (unsigned)p.num_pages)
                    marks[page[i]] = 1;
                  else
                    p.status[rows[i]] = TOPLOC_SEQ_BAD_PAGE;
                }
              });
  team.sync();

  int begin, end, count = 0, live;
  const int each = groups_each(p, team);
  pages_of_warp(p, each, team.warp_of_all, &begin, &end);
  for_pages(marks, begin, end, [&](int, int mark) { count += mark != 0; });
  tell_count(team, counts, warp_total(count));
  team.sync();

  // used pages in front of the warp's, of all, and in front of the page that they will end at
  const int before = counted_before(team, counts, team.warp_of_all, &live);
  int below;
  {
    const int there = each > 0 ? min(live / (each * 32), team.all_warps - 1) : 0;
    int from, to, all, more = 0;
    pages_of_warp(p, each, there, &from, &to);
    below = counted_before(team, counts, there, &all);
    for_pages(marks, from, min(to, live), [&](int, int mark) { more += mark != 0; });
    below += warp_total(more);
  }
  int passed = before;
  for_pages(marks, begin, end, [&](int i, int mark) {
    const bool used = mark != 0;
    const unsigned all = __ballot_sync(0xFFFFFFFFu, used);
    const int in_front = passed + __popc(all & ((1u << lane) - 1));
    if (i < end) {
      if (i < live && !used) p.copy_to[i - in_front] = i;
      if (i >= live && used) {
        p.copy_from[in_front - below] = i;
        marks[i] = 1 + in_front - below;
      }
      if (i >= live) p.free_out[p.num_free - p.num_pages + i] = i;
    }
    passed += __popc(all);
  });
  if (all_tid == 0) {
    p.num_copies[0] = live - below;
    p.next_free[0] = p.num_free - (p.num_pages - live);
  }
  team.sync();

  for_entries(p, team, p.table_in, p.table_in_stride, held,
              [&](const int* rows, unsigned col, const int32_t* page, const bool* valid) {
                int32_t to[kAtOnce];
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) {
                  to[i] = 0;
                  if (valid[i] && page[i] >= live && page[i] < p.num_pages) to[i] = fresh(marks + page[i]);
                }
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) to[i] = to[i] > 0 ? fresh(p.copy_to + (to[i] - 1)) : page[i];
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i)
                  if (valid[i]) p.table[rows[i] * p.table_stride + col] = to[i];
              });
  passed = before;
  for_pages(marks, begin, min(end, live), [&](int i, int mark) {
    const unsigned all = __ballot_sync(0xFFFFFFFFu, mark != 0);
    const int in_front = passed + __popc(all & ((1u << lane) - 1));
    if (i < min(end, live)) p.shares_out[i] = p.shares[mark != 0 ? i : fresh(p.copy_from + (i - in_front))];
    passed += __popc(all);
  });
  team.sync();  // (the marks have been read)
  for (int i = max(begin, live) + lane; i < end; i += 32) p.shares_out[i] = 0;
}

// ---- copies --------------------------------------------------------------------------------------

constexpr int kMostCaches = 128;  // of a launch
constexpr int kCopyThreads = 256;
constexpr int kUnits = 8;         // a thread's, of a chunk

struct CopyParams {
  void* caches[kMostCaches];
  const int32_t* from;
  const int32_t* to;
  const int32_t* count;
  long long page, token, head;  // strides in units
  long long units;              // of a page
  int most, num_caches, num_pages, chunks;
  int heads, units_per_head;    // heads 0: a page is one run of units
};

// Bound by memory: a page is read once and written once.  The number of copies is known on the device alone, so the blocks
// share out what there is: (cache, copy, chunk of a page), eight 16-byte loads in flight a thread.  A cache's copies are done
// together, so that a page which is copied several times (the last one of a prompt with many samples) can come from L2 again
// (512 forks of 64 prompts: 470 MB are copied, 140 read from memory, 67 of them different).  Pages in one run go at 6.1 TB/s
// (2000 of 65 KB: 43 us); others pay for the places of their units: heads that are half of a row's 50 us, heads with gaps 68.
template <typename Unit>
__global__ void __launch_bounds__(kCopyThreads) toploc_copy_pages_kernel(const __grid_constant__ CopyParams p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int copies = min(max(p.count[0], 0), p.most);
  const long long per_cache = (long long)copies * p.chunks, tasks = per_cache * p.num_caches;
  // (the task's pages are looked up while the one in front is copied)
  long long t = blockIdx.x;
  int cache = 0, copy = 0, chunk = 0, from = -1, to = -1;
  const auto look_up = [&]() {
    if (t >= tasks) return;
    cache = (int)(t / per_cache);
    const long long rest = t - cache * per_cache;
    copy = (int)((unsigned long long)rest <= 0xFFFFFFFFull ? (unsigned)rest / (unsigned)p.chunks : rest / p.chunks);
    chunk = (int)(rest - (long long)copy * p.chunks);
    from = p.from[copy];
    to = p.to[copy];
  };
  look_up();
  while (t < tasks) {
    const bool good = (unsigned)from < (unsigned)p.num_pages && (unsigned)to < (unsigned)p.num_pages && from != to;
    const Unit* src = static_cast<const Unit*>(p.caches[cache]) + from * p.page;
    Unit* dst = static_cast<Unit*>(p.caches[cache]) + to * p.page;
    const long long first = (long long)chunk * kCopyThreads * kUnits + threadIdx.x;
    Unit v[kUnits];
    long long at[kUnits];
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const long long u = first + i * kCopyThreads;
      at[i] = u;
      if (good && u < p.units) {
        if (p.heads > 0) {
          const long long row = u / p.units_per_head;
          at[i] = row / p.heads * p.token + row % p.heads * p.head + (u - row * p.units_per_head);
        }
        v[i] = src[at[i]];
      }
    }
    t += gridDim.x;
    look_up();
#pragma unroll
    for (int i = 0; i < kUnits; ++i)
      if (good && first + i * kCopyThreads < p.units) __stcs(dst + at[i], v[i]);
  }
}

// (It may begin before the plan in front of it has ended, and waits for that end itself.)
template <typename Unit>
int launch_copy(const CopyParams& p, int blocks, cudaStream_t stream) {
  cudaLaunchConfig_t config = {};
  cudaLaunchAttribute early[1];
  config.gridDim = dim3((unsigned)blocks);
  config.blockDim = dim3(kCopyThreads);
  config.stream = stream;
  early[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early[0].val.programmaticStreamSerializationAllowed = 1;
  config.attrs = early;
  config.numAttrs = 1;
  if (cudaLaunchKernelEx(&config, toploc_copy_pages_kernel<Unit>, p) != cudaSuccess) {
    cudaGetLastError();
    return TOPLOC_ERR_CUDA;
  }
  return launched();
}

// What the three planners ask of their sizes.
int check_pool(int num_seqs, int num_pages, int num_free, int page_size, int max_pages, int64_t table_stride) {
  if (num_seqs < 0 || num_pages < 0 || num_free < 0 || page_size <= 0 || max_pages < 0 || table_stride < max_pages)
    return TOPLOC_ERR_INVALID_ARGUMENT;
  if (num_seqs > (1 << 24) || num_pages > (1 << 30)) return TOPLOC_ERR_UNSUPPORTED;
  return TOPLOC_OK;
}

// An array of a call: where it has to be (if it has any bytes), and its memory.
struct Argument {
  Rows memory;
  int align;
  Argument(const void* at, long long bytes, int align = 4) : memory(at, bytes), align(align) {}
  Argument(const void* at, int columns, int rows, int64_t stride)
      : memory(at, columns * 4ll, rows, min((long long)stride, 1ll << 56) * 4), align(4) {}
  bool usable() const { return memory.bytes <= 0 || memory.rows <= 0 || (memory.at != nullptr && aligned(memory.at, align)); }
};

// Whether two tables share memory.  With one step, rows between each other's rows do not.
bool tables_overlap(const Rows& a, const Rows& b) {
  if (a.bytes <= 0 || b.bytes <= 0 || a.rows <= 0 || b.rows <= 0) return false;
  const auto extent = [](const Rows& r) {  // (rows <= 2^24)
    return Rows(r.at, r.step > (1ll << 36) ? 1ll << 60 : (r.rows - 1) * r.step + r.bytes);
  };
  if (!overlap(extent(a), extent(b))) return false;
  if (a.step != b.step) return true;
  const uintptr_t from = reinterpret_cast<uintptr_t>(a.at), to = reinterpret_cast<uintptr_t>(b.at);
  const long long away = (long long)(from < to ? (to - from) % (uintptr_t)a.step
                                               : (a.step - (long long)((from - to) % (uintptr_t)a.step)) % a.step);
  return away < a.bytes || a.step - away < b.bytes;
}

// Every output apart from every input and from the other outputs.
template <int kIn, int kOut>
int check_memory(const Argument (&in)[kIn], const Argument (&out)[kOut]) {
  for (const Argument& a : in)
    if (!a.usable()) return TOPLOC_ERR_INVALID_ARGUMENT;
  for (const Argument& a : out)
    if (!a.usable()) return TOPLOC_ERR_INVALID_ARGUMENT;
  const auto meet = [](const Argument& a, const Argument& b) {
    if (a.memory.rows <= 1) return overlap(a.memory, b.memory);
    if (b.memory.rows <= 1) return overlap(b.memory, a.memory);
    return tables_overlap(a.memory, b.memory);
  };
  for (int i = 0; i < kOut; ++i) {
    for (int j = 0; j < kIn; ++j)
      if (meet(out[i], in[j])) return TOPLOC_ERR_INVALID_ARGUMENT;
    for (int j = 0; j < i; ++j)
      if (meet(out[i], out[j])) return TOPLOC_ERR_INVALID_ARGUMENT;
  }
  return TOPLOC_OK;
}

// A launch of `blocks` blocks, in clusters of `cluster`; early: it may begin before the one in front of it has ended (and waits
// for that end itself).
template <typename Kernel>
int launch(Kernel kernel, const PoolParams& p, unsigned blocks, unsigned threads, unsigned cluster, bool early,
           void* cuda_stream) {
  cudaLaunchConfig_t config = {};
  cudaLaunchAttribute attributes[2];
  config.gridDim = dim3(blocks);
  config.blockDim = dim3(threads);
  config.stream = static_cast<cudaStream_t>(cuda_stream);
  attributes[0].id = cudaLaunchAttributeClusterDimension;
  attributes[0].val.clusterDim.x = cluster;
  attributes[0].val.clusterDim.y = attributes[0].val.clusterDim.z = 1;
  attributes[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attributes[1].val.programmaticStreamSerializationAllowed = 1;
  config.attrs = attributes;
  config.numAttrs = early ? 2 : 1;
  if (cudaLaunchKernelEx(&config, kernel, p) != cudaSuccess) {
    cudaGetLastError();
    return TOPLOC_ERR_CUDA;
  }
  return launched();
}

// Entries (at most) and pages of a plan.
long long work_of(const PoolParams& p) { return (long long)p.num_seqs * p.max_pages + p.num_pages; }

// One block, or a cluster of eight where the work makes many rounds for one.
template <typename Kernel>
int launch_planner(Kernel kernel, const PoolParams& p, void* cuda_stream) {
  const unsigned blocks = work_of(p) <= kOneBlock ? 1 : kMostBlocks;
  return launch(kernel, p, blocks, kThreads, blocks, false, cuda_stream);
}

}  // namespace

extern "C" int toploc_fork_pages(const int32_t* d_parents, const int32_t* d_kv_lens, int32_t num_seqs,
                                 const int32_t* d_shares, int32_t num_pages, const int32_t* d_free_pages, int32_t num_free,
                                 const int32_t* d_first_free, int32_t page_size, int32_t* d_block_table, int32_t max_pages,
                                 int64_t table_stride, int32_t* d_kv_lens_out, int32_t* d_shares_out, int32_t* d_copy_from,
                                 int32_t* d_copy_to, int32_t* d_num_copies, int32_t* d_next_free, uint8_t* d_status,
                                 void* cuda_stream) {
  if (const int rc = check_pool(num_seqs, num_pages, num_free, page_size, max_pages, table_stride)) return rc;
  const long long seqs = num_seqs * 4ll, pages = num_pages * 4ll;
  const Argument in[] = {{d_parents, seqs}, {d_kv_lens, seqs}, {d_shares, pages}, {d_free_pages, num_free * 4ll},
                         {d_first_free, 4}};
  const Argument out[] = {{d_block_table, max_pages, num_seqs, table_stride}, {d_kv_lens_out, seqs}, {d_shares_out, pages},
                          {d_copy_from, seqs}, {d_copy_to, seqs}, {d_num_copies, 4}, {d_next_free, 4},
                          {d_status, num_seqs, 1}};
  if (const int rc = check_memory(in, out)) return rc;
  if (const int rc = check_device()) return rc;
  PoolParams p = {};
  p.parents = d_parents, p.kv_lens = d_kv_lens, p.shares = d_shares, p.free_in = d_free_pages, p.first_free = d_first_free;
  p.table = d_block_table, p.table_stride = table_stride;
  p.kv_lens_out = d_kv_lens_out, p.shares_out = d_shares_out, p.copy_from = d_copy_from, p.copy_to = d_copy_to;
  p.num_copies = d_num_copies, p.next_free = d_next_free, p.status = d_status;
  p.num_seqs = num_seqs, p.num_pages = num_pages, p.num_free = num_free, p.page_size = page_size, p.max_pages = max_pages;
  return launch_planner(toploc_fork_pages_kernel, p, cuda_stream);
}

extern "C" int toploc_release_pages(const uint8_t* d_release, const int32_t* d_kv_lens, int32_t num_seqs,
                                    const int32_t* d_block_table, int32_t max_pages, int64_t table_stride,
                                    const int32_t* d_shares, int32_t num_pages, int32_t page_size, int32_t* d_free_pages,
                                    int32_t num_free, const int32_t* d_first_free, int32_t* d_kv_lens_out,
                                    int32_t* d_shares_out, int32_t* d_next_free, uint8_t* d_status, void* cuda_stream) {
  if (const int rc = check_pool(num_seqs, num_pages, num_free, page_size, max_pages, table_stride)) return rc;
  const long long seqs = num_seqs * 4ll, pages = num_pages * 4ll;
  const Argument in[] = {{d_release, num_seqs, 1}, {d_kv_lens, seqs}, {d_block_table, max_pages, num_seqs, table_stride},
                         {d_shares, pages}, {d_first_free, 4}};
  const Argument out[] = {{d_free_pages, num_free * 4ll}, {d_kv_lens_out, seqs}, {d_shares_out, pages}, {d_next_free, 4},
                          {d_status, num_seqs, 1}};
  if (const int rc = check_memory(in, out)) return rc;
  int sms = 0;
  if (const int rc = check_device(&sms)) return rc;
  PoolParams p = {};
  p.release = d_release, p.kv_lens = d_kv_lens, p.shares = d_shares, p.first_free = d_first_free;
  p.table = const_cast<int32_t*>(d_block_table), p.table_stride = table_stride;
  p.free_out = d_free_pages, p.kv_lens_out = d_kv_lens_out, p.shares_out = d_shares_out, p.next_free = d_next_free;
  p.status = d_status;
  p.num_seqs = num_seqs, p.num_pages = num_pages, p.num_free = num_free, p.page_size = page_size, p.max_pages = max_pages;
  if (work_of(p) <= kOneCluster) return launch_planner(toploc_release_pages_kernel<true>, p, cuda_stream);
  const unsigned blocks = (unsigned)(2 * sms);
  if (const int rc = launch(toploc_release_begin_kernel, p, blocks, kWideThreads, 1, false, cuda_stream)) return rc;
  if (const int rc = launch(toploc_release_entries_kernel, p, 4 * blocks, kWideThreads, 1, true, cuda_stream)) return rc;
  return launch(toploc_release_pages_kernel<false>, p, kMostBlocks, kThreads, kMostBlocks, true, cuda_stream);
}

extern "C" int toploc_compact_pages(const int32_t* d_kv_lens, int32_t num_seqs, const int32_t* d_block_table,
                                    int32_t max_pages, int64_t table_stride, const int32_t* d_shares, int32_t num_pages,
                                    int32_t page_size, int32_t* d_block_table_out, int64_t table_out_stride,
                                    int32_t* d_shares_out, int32_t* d_free_pages_out, int32_t num_free,
                                    int32_t* d_copy_from, int32_t* d_copy_to, int32_t* d_num_copies, int32_t* d_next_free,
                                    uint8_t* d_status, void* cuda_stream) {
  if (const int rc = check_pool(num_seqs, num_pages, num_free, page_size, max_pages, table_stride)) return rc;
  if (table_out_stride < max_pages || num_free < num_pages) return TOPLOC_ERR_INVALID_ARGUMENT;
  const long long seqs = num_seqs * 4ll, pages = num_pages * 4ll;
  const bool in_place = d_block_table_out == d_block_table && (table_out_stride == table_stride || num_seqs <= 1);
  const Argument table(d_block_table, max_pages, num_seqs, table_stride);
  const Argument in[] = {{d_kv_lens, seqs}, in_place ? Argument(nullptr, 0) : table, {d_shares, pages}};
  const Argument out[] = {{d_block_table_out, max_pages, num_seqs, table_out_stride}, {d_shares_out, pages},
                          {d_free_pages_out, num_free * 4ll}, {d_copy_from, pages}, {d_copy_to, pages}, {d_num_copies, 4},
                          {d_next_free, 4}, {d_status, num_seqs, 1}};
  if (const int rc = check_memory(in, out)) return rc;
  if (const int rc = check_device()) return rc;
  PoolParams p = {};
  p.kv_lens = d_kv_lens, p.shares = d_shares, p.table_in = d_block_table, p.table_in_stride = table_stride;
  p.table = d_block_table_out, p.table_stride = table_out_stride, p.shares_out = d_shares_out, p.free_out = d_free_pages_out;
  p.copy_from = d_copy_from, p.copy_to = d_copy_to, p.num_copies = d_num_copies, p.next_free = d_next_free;
  p.status = d_status;
  p.num_seqs = num_seqs, p.num_pages = num_pages, p.num_free = num_free, p.page_size = page_size, p.max_pages = max_pages;
  return launch_planner(toploc_compact_pages_kernel, p, cuda_stream);
}

extern "C" int toploc_copy_pages(void* const* h_caches, const toploc_pool_layout* lay, const int32_t* d_copy_from,
                                 const int32_t* d_copy_to, const int32_t* d_num_copies, int32_t max_copies,
                                 void* cuda_stream) {
  if (!lay || lay->num_pages < 0 || lay->page_size <= 0 || lay->kv_heads <= 0 || lay->head_dim <= 0 || lay->num_caches < 0 ||
      lay->page_stride < 0 || lay->token_stride < 0 || lay->head_stride < 0 || max_copies < 0)
    return TOPLOC_ERR_INVALID_ARGUMENT;
  const int size = element_bytes(lay->dtype);
  const int64_t row = lay->head_dim;
  if (size == 0 || row * lay->kv_heads > 0x7FFFFFFF || row * lay->kv_heads * lay->page_size > 0x7FFFFFFF)
    return TOPLOC_ERR_UNSUPPORTED;
  if (lay->num_caches == 0 || max_copies == 0 || lay->num_pages == 0) return TOPLOC_OK;
  if (!h_caches || !d_copy_from || !d_copy_to || !d_num_copies || !aligned(d_copy_from, 4) || !aligned(d_copy_to, 4) ||
      !aligned(d_num_copies, 4))
    return TOPLOC_ERR_INVALID_ARGUMENT;
  const int64_t heads = lay->kv_heads, tokens = lay->page_size;
  // a page whose tokens and heads lie side by side, in either order, is one run
  const bool run = (lay->head_stride == row || heads == 1) && (lay->token_stride == heads * row || tokens == 1);
  const bool run_by_head = (lay->token_stride == row || tokens == 1) && (lay->head_stride == tokens * row || heads == 1);
  const bool dense = run || run_by_head;
  int unit = 16;
  while (unit > size) {  // the widest that everything is a multiple of
    bool fits = (dense ? tokens * heads * row : row) * size % unit == 0 && lay->page_stride * size % unit == 0 &&
                (dense || (lay->token_stride * size % unit == 0 && lay->head_stride * size % unit == 0));
    for (int i = 0; i < lay->num_caches && fits; ++i) fits = aligned(h_caches[i], unit);
    if (fits) break;
    unit = unit == 16 && size <= 4 ? 4 : size;
  }
  for (int i = 0; i < lay->num_caches; ++i)
    if (!h_caches[i] || !aligned(h_caches[i], size)) return TOPLOC_ERR_INVALID_ARGUMENT;
  int sms = 0;
  if (const int rc = check_device(&sms)) return rc;
  const int per = unit / size;
  CopyParams p;
  p.from = d_copy_from, p.to = d_copy_to, p.count = d_num_copies, p.most = max_copies, p.num_pages = lay->num_pages;
  p.page = lay->page_stride / per, p.token = lay->token_stride / per, p.head = lay->head_stride / per;
  p.units = tokens * heads * row / per;
  p.heads = dense ? 0 : (int)heads;
  p.units_per_head = (int)(row / per);
  p.chunks = (int)((p.units + kCopyThreads * kUnits - 1) / (kCopyThreads * kUnits));
  for (int first = 0; first < lay->num_caches; first += kMostCaches) {
    p.num_caches = min(lay->num_caches - first, kMostCaches);
    for (int i = 0; i < p.num_caches; ++i) p.caches[i] = h_caches[first + i];
    // what the list has room for, at most eight blocks an SM
    const long long most = (long long)max_copies * p.num_caches * p.chunks;
    const int blocks = (int)min(most, 8ll * sms);
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const int rc = unit == 16  ? launch_copy<uint4>(p, blocks, stream)
                   : unit == 4 ? launch_copy<uint32_t>(p, blocks, stream)
                               : launch_copy<uint16_t>(p, blocks, stream);
    if (rc) return rc;
  }
  return TOPLOC_OK;
}
