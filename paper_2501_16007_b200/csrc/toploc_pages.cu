// Pages of the key-value cache: the plan of a step (block table, slots, positions) and the write of
// the step's keys and values.
//
// The plan is two prefix sums over the sequences (tokens, then pages) and one write per token.  It is
// bound by latency: a step of 64 sequences moves 2 KB, a thousand prompts 25 MB.  So it is one launch,
// and no block waits for another: every block runs both prefix sums over all sequences itself (they
// are a few KB from L2), then takes an even share of the sequences (offsets, lengths, status, table
// rows) and an even share of the tokens (slots, positions).  A token's page is read from the table
// where it was there before and from the free list where it is new, so no block reads what another
// writes.
#include "model_common.cuh"

namespace {

using namespace toploc_model;

constexpr int kPlanThreads = 256;

struct PlanParams {
  const int32_t* cached;
  const int32_t* fresh;  // new tokens
  const int32_t* free_pages;
  const int32_t* first_free;
  int32_t* table;
  int32_t* offsets;
  int32_t* kv_lens;
  int64_t* slots;
  int32_t* positions;
  int32_t* next_free;
  uint8_t* status;
  long long table_stride, max_tokens;
  int num_seqs, num_free, page_size, max_pages;
  bool wide;  // slots and positions at 16-byte aligned places
};

// One sequence as the plan sees it, given the tokens and the pages in front of it.
struct PlannedSeq {
  long long first_token;  // rows in front of it
  long long first_page;   // entry of the free list its pages start at
  int tokens;
  int cached;
  int pages_before, pages_needed;
  int status;
};

// (32-bit: a 64-bit division takes several times as long, and the plan does a dozen one after the other)
__device__ __forceinline__ int pages_for(int tokens, int page_size) {
  return (int)(((unsigned)tokens + (unsigned)page_size - 1u) / (unsigned)page_size);
}

// The lengths alone: tokens, pages asked for, and the conditions that do not depend on the pool.
__device__ __forceinline__ PlannedSeq look_at(const PlanParams& p, int i, long long first_token) {
  PlannedSeq s;
  s.cached = p.cached[i];
  const int t = p.fresh[i];
  s.tokens = max(t, 0);
  s.first_token = first_token;
  s.first_page = 0;
  s.pages_before = 0;
  s.pages_needed = 0;
  s.status = TOPLOC_SEQ_OK;
  const long long kv = (long long)s.cached + s.tokens;
  if (s.cached < 0 || t < 0 || kv > 0x7FFFFFFF) {
    s.status = TOPLOC_SEQ_BAD_LENGTH;
  } else if (first_token + s.tokens > p.max_tokens) {
    s.status = TOPLOC_SEQ_BATCH_FULL;
  } else {
    const int after = pages_for((int)kv, p.page_size);
    if (after > p.max_pages) {
      s.status = TOPLOC_SEQ_TABLE_FULL;
    } else {
      s.pages_before = pages_for(s.cached, p.page_size);
      s.pages_needed = after - s.pages_before;
    }
  }
  return s;
}

__device__ __forceinline__ void place(const PlanParams& p, PlannedSeq& s, long long first_page) {
  s.first_page = first_page;
  if (s.status == TOPLOC_SEQ_OK && s.pages_needed > 0 && first_page + s.pages_needed > p.num_free)
    s.status = TOPLOC_SEQ_NO_PAGES;
}

// Exclusive prefix sum over the block's threads; *total gets the sum.
__device__ __forceinline__ long long block_scan(long long v, long long* warp_sums, long long* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long incl = v;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const long long up = __shfl_up_sync(0xFFFFFFFFu, incl, off);
    if (lane >= off) incl += up;
  }
  if (lane == 31) warp_sums[warp] = incl;
  __syncthreads();
  long long before = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 32; ++w) {
    if (w < warp) before += warp_sums[w];
    sum += warp_sums[w];
  }
  __syncthreads();
  *total = sum;
  return before + incl - v;
}

__global__ void __launch_bounds__(kPlanThreads) toploc_plan_pages_kernel(const PlanParams p) {
  __shared__ long long warp_sums[kPlanThreads / 32];
  // tokens and pages in front of every thread's run of sequences
  __shared__ long long run_token[kPlanThreads + 1], run_page[kPlanThreads];
  const int tid = threadIdx.x;
  const int per = (p.num_seqs + kPlanThreads - 1) / kPlanThreads;
  const int begin = min(tid * per, p.num_seqs), end = min(begin + per, p.num_seqs);

  long long tokens = 0, total_tokens, total_pages;
  for (int i = begin; i < end; ++i) tokens += max(p.fresh[i], 0);
  const long long my_token = block_scan(tokens, warp_sums, &total_tokens);
  long long pages = 0, at = my_token;
  for (int i = begin; i < end; ++i) {
    const PlannedSeq s = look_at(p, i, at);
    pages += s.pages_needed;
    at += s.tokens;
  }
  // (no page fits behind a negative head: every sequence that needs one is in the same state)
  const long long head = p.first_free[0] < 0 ? p.num_free : p.first_free[0];
  const long long my_page = head + block_scan(pages, warp_sums, &total_pages);
  run_token[tid] = my_token;
  run_page[tid] = my_page;
  if (tid == 0) run_token[kPlanThreads] = total_tokens;
  __syncthreads();

  // the thread's own sequences, dealt to the blocks by run
  long long taken = 0;
  {
    long long token = my_token, page = my_page;
    for (int i = begin; i < end; ++i) {
      PlannedSeq s = look_at(p, i, token);
      const int need = s.pages_needed;
      place(p, s, page);
      if (s.status == TOPLOC_SEQ_OK) taken += need;
      if (i % (int)gridDim.x == (int)blockIdx.x) {
        p.offsets[i] = (int)min(token, p.max_tokens);
        p.kv_lens[i] = s.status == TOPLOC_SEQ_OK ? s.cached + s.tokens : 0;
        p.status[i] = (uint8_t)s.status;
      }
      token += s.tokens;
      page += need;
    }
  }
  long long total_taken;
  block_scan(taken, warp_sums, &total_taken);
  if (blockIdx.x == 0 && tid == 0) {
    p.offsets[p.num_seqs] = (int)min(total_tokens, p.max_tokens);
    p.next_free[0] = (int)(p.first_free[0] + total_taken);
  }

  // table rows: a warp per sequence of the block's share
  const int warps = gridDim.x * (kPlanThreads / 32), warp = blockIdx.x * (kPlanThreads / 32) + (tid >> 5);
  for (int i = warp; i < p.num_seqs; i += warps) {
    const int run = i / per;
    long long token = run_token[run], page = run_page[run];
    for (int j = run * per; j < i; ++j) {
      const PlannedSeq s = look_at(p, j, token);
      token += s.tokens;
      page += s.pages_needed;
    }
    PlannedSeq s = look_at(p, i, token);
    place(p, s, page);
    if (s.status != TOPLOC_SEQ_OK) continue;
    int32_t* row = p.table + i * p.table_stride + s.pages_before;
    for (int j = tid & 31; j < s.pages_needed; j += 32) row[j] = p.free_pages[page + j];
  }

  // slots and positions: four consecutive rows a thread, which as a rule are one sequence's and in one page
  PlannedSeq s;
  s.first_token = 0;
  s.tokens = 0;
  s.status = TOPLOC_SEQ_OK;
  int seq = 0;
  const long long rows = min(total_tokens, p.max_tokens);
  const long long step = (long long)gridDim.x * kPlanThreads * 4;
  for (long long r0 = ((long long)blockIdx.x * kPlanThreads + tid) * 4; r0 < p.max_tokens; r0 += step) {
    long long slot[4];
    int position[4];
    int page_end = 0;  // positions of this sequence from the last one on up to here lie in the last slot's page
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const long long r = r0 + e;
      slot[e] = -1;
      position[e] = 0;
      if (r >= rows) continue;
      if (r >= s.first_token + s.tokens) {  // find the row's sequence: its run, then within the run
        int lo = 0, hi = kPlanThreads;      // run_token[lo] <= r < run_token[hi]
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (run_token[mid] <= r) lo = mid; else hi = mid;
        }
        long long token = run_token[lo], page = run_page[lo];
        for (seq = lo * per; seq < p.num_seqs; ++seq) {
          s = look_at(p, seq, token);
          if (r < token + s.tokens) break;
          token += s.tokens;
          page += s.pages_needed;
        }
        place(p, s, page);
        page_end = 0;
      }
      const int pos = (int)((long long)s.cached + (r - s.first_token));
      position[e] = pos;
      if (s.status != TOPLOC_SEQ_OK) continue;
      if (e > 0 && pos < page_end) {
        if (slot[e - 1] >= 0) slot[e] = slot[e - 1] + 1;
        continue;
      }
      const int col = (int)((unsigned)pos / (unsigned)p.page_size);
      const int held = col < s.pages_before ? p.table[seq * p.table_stride + col]
                                            : p.free_pages[s.first_page + (col - s.pages_before)];
      if (held >= 0) slot[e] = (long long)held * p.page_size + (pos - col * p.page_size);
      page_end = (int)min((long long)(col + 1) * p.page_size, 0x7FFFFFFFll);
    }
    if (r0 + 4 <= p.max_tokens && p.wide) {
      *reinterpret_cast<longlong2*>(p.slots + r0) = make_longlong2(slot[0], slot[1]);
      *reinterpret_cast<longlong2*>(p.slots + r0 + 2) = make_longlong2(slot[2], slot[3]);
      *reinterpret_cast<int4*>(p.positions + r0) = make_int4(position[0], position[1], position[2], position[3]);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (r0 + e < p.max_tokens) {
          p.slots[r0 + e] = slot[e];
          p.positions[r0 + e] = position[e];
        }
      }
    }
  }
}

struct WriteParams {
  const unsigned char* src[2];
  unsigned char* cache[2];
  long long src_token[2], src_head[2], page[2], token[2], head[2];  // strides in units
  const int64_t* slots;
  long long num_tokens, num_slots;
  int heads, units_per_head, page_size;
};

// One unit (16 bytes, or an element) per thread and step; keys and values in one launch (gridDim.y).
template <typename Unit>
__global__ void __launch_bounds__(256) toploc_cache_write_kernel(const WriteParams p) {
  const int which = blockIdx.y;
  const Unit* src = reinterpret_cast<const Unit*>(p.src[which]);
  Unit* cache = reinterpret_cast<Unit*>(p.cache[which]);
  const long long per_token = (long long)p.heads * p.units_per_head;
  const long long total = p.num_tokens * per_token, step = (long long)gridDim.x * blockDim.x;
  for (long long u = (long long)blockIdx.x * blockDim.x + threadIdx.x; u < total; u += step) {
    const long long t = u / per_token;
    const int rest = (int)(u - t * per_token);
    const int head = rest / p.units_per_head, at = rest - head * p.units_per_head;
    const long long slot = p.slots[t];
    if (slot < 0 || slot >= p.num_slots) continue;
    const long long page = slot / p.page_size, in_page = slot - page * p.page_size;
    cache[page * p.page[which] + in_page * p.token[which] + head * p.head[which] + at] =
        src[t * p.src_token[which] + head * p.src_head[which] + at];
  }
}

}  // namespace

extern "C" const char* toploc_sequence_status_string(int s) {
  switch (s) {
    case TOPLOC_SEQ_OK: return "ok";
    case TOPLOC_SEQ_BAD_LENGTH: return "length negative or beyond its bound";
    case TOPLOC_SEQ_NO_PAGES: return "free list exhausted";
    case TOPLOC_SEQ_TABLE_FULL: return "more pages than the block table holds";
    case TOPLOC_SEQ_BATCH_FULL: return "tokens end beyond the token buffers";
    case TOPLOC_SEQ_BAD_PAGE: return "block table entry outside the cache";
    case TOPLOC_SEQ_WAIT_EXPIRED: return "a wait inside the kernel ran out";
    case TOPLOC_SEQ_BAD_PARENT: return "forked from no sequence, or from one that is forked itself";
    case TOPLOC_SEQ_IN_USE: return "forked into a sequence that holds tokens";
    case TOPLOC_SEQ_NO_ROOM: return "free list without room for all pages that came back";
  }
  return "unknown sequence status";
}

extern "C" int toploc_plan_pages(const int32_t* d_cached_lens, const int32_t* d_new_lens, int32_t num_seqs,
                                 const int32_t* d_free_pages, int32_t num_free, const int32_t* d_first_free,
                                 int32_t page_size, int32_t* d_block_table, int32_t max_pages, int64_t table_stride,
                                 int32_t* d_seq_offsets, int32_t* d_kv_lens, int64_t* d_slots, int32_t* d_positions,
                                 int64_t max_tokens, int32_t* d_next_free, uint8_t* d_status, void* cuda_stream) {
  if (num_seqs < 0 || num_free < 0 || page_size <= 0 || max_pages < 0 || table_stride < max_pages || max_tokens < 0)
    return TOPLOC_ERR_INVALID_ARGUMENT;
  if (num_seqs > (1 << 24) || max_tokens > 0x7FFFFFFF) return TOPLOC_ERR_UNSUPPORTED;
  if (!d_first_free || !d_seq_offsets || !d_next_free || d_next_free == d_first_free ||
      (num_seqs > 0 && (!d_cached_lens || !d_new_lens || !d_kv_lens || !d_status)) ||
      (num_seqs > 0 && max_pages > 0 && !d_block_table) || (num_free > 0 && !d_free_pages) ||
      (max_tokens > 0 && (!d_slots || !d_positions)))
    return TOPLOC_ERR_INVALID_ARGUMENT;
  for (const void* q : {(const void*)d_cached_lens, (const void*)d_new_lens, (const void*)d_free_pages,
                        (const void*)d_first_free, (const void*)d_block_table, (const void*)d_seq_offsets,
                        (const void*)d_kv_lens, (const void*)d_positions, (const void*)d_next_free})
    if (!aligned(q, 4)) return TOPLOC_ERR_INVALID_ARGUMENT;
  if (!aligned(d_slots, 8)) return TOPLOC_ERR_INVALID_ARGUMENT;
  // every block reads the inputs several times while others write: nothing that is written may lie in them
  const Rows inputs[] = {{d_cached_lens, num_seqs * 4ll}, {d_new_lens, num_seqs * 4ll}, {d_free_pages, num_free * 4ll},
                         {d_first_free, 4}};
  const Rows outputs[] = {{d_block_table, max_pages * 4ll, num_seqs, min((long long)table_stride, 1ll << 56) * 4},
                          {d_seq_offsets, (num_seqs + 1ll) * 4}, {d_kv_lens, num_seqs * 4ll}, {d_slots, max_tokens * 8},
                          {d_positions, max_tokens * 4}, {d_next_free, 4}, {d_status, num_seqs}};
  for (const Rows& in : inputs)
    for (const Rows& out : outputs)
      if (overlap(in, out)) return TOPLOC_ERR_INVALID_ARGUMENT;
  int sms = 0;
  if (const int rc = check_device(&sms)) return rc;
  const PlanParams p = {d_cached_lens, d_new_lens, d_free_pages, d_first_free, d_block_table, d_seq_offsets, d_kv_lens,
                        d_slots, d_positions, d_next_free, d_status, table_stride, max_tokens, num_seqs, num_free,
                        page_size, max_pages, aligned(d_slots, 16) && aligned(d_positions, 16)};
  // four rows a thread and a warp per sequence, up to four blocks an SM (each repeats the prefix sums)
  const long long wanted = max((long long)(max_tokens + 4 * kPlanThreads - 1) / (4 * kPlanThreads),
                               (long long)(num_seqs + kPlanThreads / 32 - 1) / (kPlanThreads / 32));
  const int blocks = (int)max(1ll, min(wanted, 4ll * sms));
  toploc_plan_pages_kernel<<<blocks, kPlanThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(p);
  return launched();
}

extern "C" int toploc_cache_write(const void* d_k, const void* d_v, int64_t k_token_stride, int64_t k_head_stride,
                                  int64_t v_token_stride, int64_t v_head_stride, const int64_t* d_slots,
                                  int64_t num_tokens, int32_t dtype, int32_t kv_heads, int32_t head_dim,
                                  void* d_k_cache, void* d_v_cache, const toploc_kv_layout* kv, void* cuda_stream) {
  const int size = element_bytes(dtype);
  if (!kv || num_tokens < 0 || kv_heads <= 0 || head_dim <= 0 || kv->page_size <= 0 || kv->num_pages < 0)
    return TOPLOC_ERR_INVALID_ARGUMENT;
  // (a thread's place inside a token is a 32-bit number)
  if (size == 0 || (int64_t)kv_heads * head_dim > 0x7FFFFFFF) return TOPLOC_ERR_UNSUPPORTED;
  if (num_tokens == 0) return TOPLOC_OK;
  if (!d_k || !d_v || !d_slots || !d_k_cache || !d_v_cache || !aligned(d_slots, 8)) return TOPLOC_ERR_INVALID_ARGUMENT;
  const int64_t strides[10] = {k_token_stride, k_head_stride, kv->k_page_stride, kv->k_token_stride, kv->k_head_stride,
                               v_token_stride, v_head_stride, kv->v_page_stride, kv->v_token_stride, kv->v_head_stride};
  bool vectors = (int64_t)head_dim * size % 16 == 0;
  for (const int64_t s : strides) {
    if (s < 0) return TOPLOC_ERR_INVALID_ARGUMENT;
    vectors = vectors && s * size % 16 == 0;
  }
  for (const void* q : {d_k, d_v, (const void*)d_k_cache, (const void*)d_v_cache}) {
    if (!aligned(q, size)) return TOPLOC_ERR_INVALID_ARGUMENT;
    vectors = vectors && aligned(q, 16);
  }
  int sms = 0;
  if (const int rc = check_device(&sms)) return rc;
  const int unit = vectors ? 16 : size, per = unit / size;
  WriteParams p;
  p.src[0] = static_cast<const unsigned char*>(d_k);
  p.src[1] = static_cast<const unsigned char*>(d_v);
  p.cache[0] = static_cast<unsigned char*>(d_k_cache);
  p.cache[1] = static_cast<unsigned char*>(d_v_cache);
  for (int w = 0; w < 2; ++w) {
    p.src_token[w] = strides[5 * w] / per;
    p.src_head[w] = strides[5 * w + 1] / per;
    p.page[w] = strides[5 * w + 2] / per;
    p.token[w] = strides[5 * w + 3] / per;
    p.head[w] = strides[5 * w + 4] / per;
  }
  p.slots = d_slots;
  p.num_tokens = num_tokens;
  p.num_slots = (long long)kv->num_pages * kv->page_size;
  p.heads = kv_heads;
  p.units_per_head = head_dim / per;
  p.page_size = kv->page_size;
  const long long units = num_tokens * kv_heads * p.units_per_head;
  const dim3 grid((unsigned)max(1ll, min((units + 255) / 256, 4ll * sms)), 2);
  const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  if (unit == 16)
    toploc_cache_write_kernel<uint4><<<grid, 256, 0, stream>>>(p);
  else if (unit == 4)
    toploc_cache_write_kernel<uint32_t><<<grid, 256, 0, stream>>>(p);
  else
    toploc_cache_write_kernel<uint16_t><<<grid, 256, 0, stream>>>(p);
  return launched();
}
