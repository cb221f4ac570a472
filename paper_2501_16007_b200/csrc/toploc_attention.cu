// Attention of new tokens over a paged cache, and over packed prompts.
//
//   out_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(scale q_i . k_j - m_i),  j up to the row's own key
//
// One pass over the keys with a running maximum m and sum l: when a tile raises m, what has been summed
// so far shrinks by exp(m_old - m_new).  The query heads of a key head are rows of one matrix, (token,
// head in group) row by row, so that every key and value is read once for all of them.
#include "attention_common.cuh"

namespace {

using namespace toploc_model;

constexpr int kRows = 32;   // rows of a block
constexpr int kKeys = 32;   // keys of a tile, one per lane
constexpr int kWarpRows = kRows / 4;

// The keys of part `split` of a sequence: a multiple of 128 keys each.
__device__ __forceinline__ void split_range(int keys, int splits, int split, int* begin, int* end) {
  const int unit = ((keys + splits - 1) / splits + 128 - 1) / 128 * 128;
  *begin = (int)min((long long)unit * split, (long long)keys);
  *end = (int)min((long long)*begin + unit, (long long)keys);
}

// ---- the kernel on the fp32 units: every type, layout and head size ------------------------------
//
// A block of four warps takes 32 rows of one key head against tiles of 32 keys in shared memory (fp32).
// Scores: a lane per key, eight rows of the warp at a time, so a vector of the key serves eight rows.
// Second product: a lane per channel.  Bound by the fp32 units (4 * head_dim flops a score), with about
// one shared-memory read in four instructions.
template <typename T, int CHUNKS>
__global__ void __launch_bounds__(128) toploc_attention_fp32_kernel(const AttentionParams p) {
  extern __shared__ __align__(16) float smem[];
  const int d = p.head_dim, ld = d + 4;
  float* sq = smem;
  float* sk = sq + kRows * ld;
  float* sv = sk + kKeys * ld;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int b = blockIdx.x;
  const int split = b % p.splits; b /= p.splits;
  const int tile = b % p.row_tiles; b /= p.row_tiles;
  const int head = b % p.kv_heads;
  const int seq = b / p.kv_heads;
  const SeqRange s = sequence(p, seq);
  if (s.bad && p.status && tid == 0) p.status[seq] = TOPLOC_SEQ_BAD_LENGTH;
  const int rows = s.rows * p.group;
  const int row0 = tile * kRows;
  if (row0 >= rows) return;
  int begin, end;
  split_range(s.keys, p.splits, split, &begin, &end);
  const int behind = s.keys - s.rows;  // keys in front of the first new token (negative: rows without keys)
  end = min(end, behind + min(row0 + kRows - 1, rows - 1) / p.group + 1);

  for (int e = tid; e < kRows * d; e += 128) {
    const int r = e / d, c = e - r * d, row = row0 + r;
    float v = 0.f;
    if (row < rows) {
      const int t = row / p.group, h = head * p.group + row - t * p.group;
      v = to_float(static_cast<const T*>(p.q)[(s.first + t) * p.q_token + h * p.q_head + c]) * p.scale_log2;
    }
    sq[r * ld + c] = v;
  }
  float m[kWarpRows], l[kWarpRows], o[kWarpRows][CHUNKS];
  int last[kWarpRows];  // newest key each row sees
#pragma unroll
  for (int r = 0; r < kWarpRows; ++r) {
    m[r] = -INFINITY;
    l[r] = 0.f;
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) o[r][c] = 0.f;
    const int row = row0 + warp * kWarpRows + r;
    last[r] = row < rows ? behind + row / p.group : -1;
  }
  for (int key0 = begin; key0 < end; key0 += kKeys) {
    __syncthreads();
    for (int e = tid; e < kKeys * d; e += 128) {
      const int j = e / d, c = e - j * d, key = key0 + j;
      float kf = 0.f, vf = 0.f;  // keys past the end: zeros, so that nothing foreign meets a weight of zero
      if (key < end) {
        long long page = 0;
        int at = s.first + key;
        if (p.kv_lens) {
          const int col = key / p.page_size;
          at = key - col * p.page_size;
          page = p.table[seq * p.table_stride + col];
          if (page < 0 || page >= p.num_pages) {
            if (p.status) p.status[seq] = TOPLOC_SEQ_BAD_PAGE;
            page = -1;
          }
        }
        if (page >= 0) {
          kf = to_float(static_cast<const T*>(p.k)[page * p.k_page + at * p.k_token + head * p.k_head + c]);
          vf = to_float(static_cast<const T*>(p.v)[page * p.v_page + at * p.v_token + head * p.v_head + c]);
        }
      }
      sk[j * ld + c] = kf;
      sv[j * ld + c] = vf;
    }
    __syncthreads();
    float acc[kWarpRows];
#pragma unroll
    for (int r = 0; r < kWarpRows; ++r) acc[r] = 0.f;
    for (int c = 0; c < d; c += 4) {
      const float4 kk = *reinterpret_cast<const float4*>(sk + lane * ld + c);
#pragma unroll
      for (int r = 0; r < kWarpRows; ++r) {
        const float4 qq = *reinterpret_cast<const float4*>(sq + (warp * kWarpRows + r) * ld + c);
        acc[r] = fmaf(qq.x, kk.x, fmaf(qq.y, kk.y, fmaf(qq.z, kk.z, fmaf(qq.w, kk.w, acc[r]))));
      }
    }
#pragma unroll
    for (int r = 0; r < kWarpRows; ++r) {
      const bool visible = key0 + lane <= last[r] && key0 + lane < end;
      const float score = visible ? acc[r] : -INFINITY;
      float top = score;
      bool nan = score != score;
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, off));
      const float m_new = fmaxf(m[r], top);
      const float ref = m_new == -INFINITY ? 0.f : m_new;
      const float w = nan ? score : exp2f(score - ref);
      const float shrink = exp2f(m[r] - ref);  // 0 for the first keys
      float sum = w;
#pragma unroll
      for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, off);
      l[r] = fmaf(l[r], shrink, sum);
      m[r] = m_new;
      acc[r] = w;
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) o[r][c] *= shrink;
    }
    const int count = min(kKeys, end - key0);
    for (int j = 0; j < count; ++j) {
      float vv[CHUNKS];
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c) vv[c] = lane + 32 * c < d ? sv[j * ld + lane + 32 * c] : 0.f;
#pragma unroll
      for (int r = 0; r < kWarpRows; ++r) {
        const float w = __shfl_sync(0xFFFFFFFFu, acc[r], j);
        if (w != 0.f) {  // the same for the whole warp; a hidden value, NaN or not, is never touched
#pragma unroll
          for (int c = 0; c < CHUNKS; ++c) o[r][c] = fmaf(w, vv[c], o[r][c]);
        }
      }
    }
  }
#pragma unroll
  for (int r = 0; r < kWarpRows; ++r) {
    const int row = row0 + warp * kWarpRows + r;
    if (row >= rows) break;
    const int t = row / p.group, h = head * p.group + row - t * p.group;
    const float inv = l[r] == 0.f ? 0.f : 1.f / l[r];
    const long long at = (long long)(s.first + t) * p.q_heads + h;
    const float lse2 = l[r] == 0.f ? -INFINITY : m[r] + log2f(l[r]);
    if (p.splits == 1) {
      T* out = static_cast<T*>(p.out) + (s.first + t) * p.out_token + h * p.out_head;
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c)
        if (lane + 32 * c < d) store_as(out + lane + 32 * c, o[r][c] * inv);
      if (p.lse && lane == 0) p.lse[at] = lse2 * kLn2;
    } else {
      const long long slot = split * p.total_tokens * p.q_heads + at;
#pragma unroll
      for (int c = 0; c < CHUNKS; ++c)
        if (lane + 32 * c < d) p.part_out[slot * d + lane + 32 * c] = o[r][c] * inv;
      if (lane == 0) p.part_lse[slot] = lse2;
    }
  }
}

// ---- joining the parts -----------------------------------------------------------------------------
//
// Part i has out_i = sum p v / sum p and lse_i over its keys; the whole is sum_i w_i out_i / sum_i w_i
// with w_i = 2^(lse_i - max).  A warp per row, parts in order: the result does not depend on timing.
template <typename T>
__global__ void __launch_bounds__(128) toploc_attention_join_kernel(const AttentionParams p, int blocks_a_seq) {
  const int lane = threadIdx.x & 31, seq = blockIdx.x / blocks_a_seq;
  const SeqRange s = sequence(p, seq);  // the rows that the kernel before has written, no others
  const int r = (blockIdx.x - seq * blocks_a_seq) * 4 + (threadIdx.x >> 5);
  if (r >= s.rows * p.q_heads) return;
  const long long token = s.first + r / p.q_heads;
  const int h = r % p.q_heads;
  const long long at = token * p.q_heads + h, all = p.total_tokens * p.q_heads;
  float top = -INFINITY;
  for (int i = 0; i < p.splits; ++i) top = fmaxf(top, p.part_lse[i * all + at]);
  const float ref = top == -INFINITY ? 0.f : top;
  float sum = 0.f;
  for (int i = 0; i < p.splits; ++i) sum += exp2f(p.part_lse[i * all + at] - ref);
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  T* out = static_cast<T*>(p.out) + token * p.out_token + h * p.out_head;
  for (int c = lane; c < p.head_dim; c += 32) {
    float o = 0.f;
    for (int i = 0; i < p.splits; ++i) {
      const float w = exp2f(p.part_lse[i * all + at] - ref);
      if (w != 0.f) o = fmaf(w, p.part_out[(i * all + at) * p.head_dim + c], o);
    }
    store_as(out + c, o * inv);
  }
  if (p.lse && lane == 0) p.lse[at] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

// Parts the keys of a paged cache are split into (fp32 units), by the bounds the host knows.
int splits_of(const toploc_attention_layout* lay, const toploc_kv_layout* kv) {
  if (kv->page_size <= 0) return 1;
  const long long packed = (long long)lay->max_new_tokens * (lay->q_heads / lay->kv_heads);
  const long long items = (packed + kRows - 1) / kRows * lay->kv_heads * lay->num_seqs;
  if (items == 0) return 1;
  const long long most = (long long)kv->max_pages * kv->page_size;
  return (int)max(1ll, min(min((4ll * kSms + items - 1) / items, most / 256), 64ll));
}

int check_layout(const toploc_attention_layout* lay, const toploc_kv_layout* kv) {
  if (!lay || !kv || lay->num_seqs < 0 || lay->max_new_tokens < 0 || lay->total_tokens < 0 || lay->q_heads <= 0 ||
      lay->kv_heads <= 0 || lay->head_dim <= 0 || !(lay->scale > 0.f) || !(lay->scale < INFINITY) || kv->page_size < 0 ||
      lay->wait_tries < 0 || lay->q_heads % lay->kv_heads != 0)
    return TOPLOC_ERR_INVALID_ARGUMENT;
  if (kv->page_size > 0 && (kv->num_pages < 0 || kv->max_pages < 0 || kv->table_stride < kv->max_pages))
    return TOPLOC_ERR_INVALID_ARGUMENT;
  for (const int64_t s : {lay->q_token_stride, lay->q_head_stride, lay->out_token_stride, lay->out_head_stride,
                          kv->k_token_stride, kv->k_head_stride, kv->v_token_stride, kv->v_head_stride,
                          kv->page_size > 0 ? kv->k_page_stride : 0, kv->page_size > 0 ? kv->v_page_stride : 0})
    if (s < 0) return TOPLOC_ERR_INVALID_ARGUMENT;
  if (element_bytes(lay->dtype) == 0 || lay->head_dim % 8 != 0 || lay->head_dim > 256 ||
      lay->q_heads / lay->kv_heads > 128 || lay->total_tokens > 0x7FFFFFFF || lay->num_seqs > (1 << 24) ||
      (long long)lay->max_new_tokens * (lay->q_heads / lay->kv_heads) > 0x7FFFFFFF - 256 ||
      (kv->page_size > 0 && (long long)kv->max_pages * kv->page_size > 0x7FFFFFFF - 256))
    return TOPLOC_ERR_UNSUPPORTED;
  return TOPLOC_OK;
}

bool tensor_core_types(const toploc_attention_layout* lay) {
  return lay->dtype == TOPLOC_DTYPE_BF16 && (lay->head_dim == 64 || lay->head_dim == 128);
}

size_t workspace_bytes_of(const toploc_attention_layout* lay, const toploc_kv_layout* kv, bool tensor_cores) {
  if (lay->num_seqs == 0 || lay->total_tokens == 0 || lay->max_new_tokens == 0) return 0;
  if (tensor_cores) return tensor_core_workspace_bytes(lay, kv);
  const int splits = splits_of(lay, kv);
  return splits <= 1 ? 0 : (size_t)splits * lay->total_tokens * lay->q_heads * (lay->head_dim + 1) * 4;
}

template <typename T, int CHUNKS>
int launch_fp32(const AttentionParams& p, cudaStream_t stream) {
  const auto bytes = [](int head_dim) { return (kRows + 2 * kKeys) * (head_dim + 4) * 4; };
  static std::atomic<uint64_t> allowed{0};
  if (const int rc = allow_shared(reinterpret_cast<const void*>(toploc_attention_fp32_kernel<T, CHUNKS>),
                                  bytes(32 * CHUNKS), allowed))
    return rc;
  const long long blocks = (long long)p.num_seqs * p.kv_heads * p.row_tiles * p.splits;
  if (blocks > 0x7FFFFFFF) return TOPLOC_ERR_UNSUPPORTED;
  toploc_attention_fp32_kernel<T, CHUNKS><<<(unsigned)blocks, 128, bytes(p.head_dim), stream>>>(p);
  return launched();
}

template <typename T>
int launch_all(AttentionParams& p, cudaStream_t stream) {
  p.row_tiles = (int)(((long long)p.max_new * p.group + kRows - 1) / kRows);
  const int rc = p.head_dim <= 64 ? launch_fp32<T, 2>(p, stream)
           : p.head_dim <= 128 ? launch_fp32<T, 4>(p, stream) : launch_fp32<T, 8>(p, stream);
  if (rc != TOPLOC_OK || p.splits == 1) return rc;
  // (splits_of: where keys are split, all sequences together bring few rows)
  const int blocks_a_seq = (p.max_new * p.q_heads + 3) / 4;
  toploc_attention_join_kernel<T><<<(unsigned)(p.num_seqs * blocks_a_seq), 128, 0, stream>>>(p, blocks_a_seq);
  return launched();
}

int attention(const void* d_q, const void* d_k, const void* d_v, const toploc_attention_layout* lay,
              const toploc_kv_layout* kv, const int32_t* table, const int32_t* offsets, const int32_t* kv_lens,
              void* d_out, float* lse, uint8_t* status, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  const int size = element_bytes(lay->dtype);
  if (!aligned(d_q, size) || !aligned(d_k, size) || !aligned(d_v, size) || !aligned(d_out, size) || !aligned(lse, 4) ||
      !aligned(table, 4) || !aligned(offsets, 4) || !aligned(kv_lens, 4))
    return TOPLOC_ERR_INVALID_ARGUMENT;
  if (const int rc = check_device()) return rc;
  AttentionParams p = {};
  p.q = d_q; p.k = d_k; p.v = d_v; p.out = d_out; p.lse = lse; p.status = status;
  p.table = table; p.offsets = offsets; p.kv_lens = kv_lens;
  p.total_tokens = lay->total_tokens;
  p.q_token = lay->q_token_stride; p.q_head = lay->q_head_stride;
  p.out_token = lay->out_token_stride; p.out_head = lay->out_head_stride;
  p.k_page = kv->k_page_stride; p.k_token = kv->k_token_stride; p.k_head = kv->k_head_stride;
  p.v_page = kv->v_page_stride; p.v_token = kv->v_token_stride; p.v_head = kv->v_head_stride;
  p.table_stride = kv->table_stride;
  p.scale_log2 = lay->scale * kLog2e;
  p.head_dim = lay->head_dim; p.q_heads = lay->q_heads; p.kv_heads = lay->kv_heads;
  p.group = lay->q_heads / lay->kv_heads;
  p.num_seqs = lay->num_seqs; p.max_new = lay->max_new_tokens;
  p.page_size = kv->page_size; p.num_pages = kv->num_pages; p.max_pages = kv->max_pages;
  p.most_keys = kv->page_size > 0 ? kv->max_pages * kv->page_size : 0;  // (check_layout: fits)
  const bool tensor_cores = tensor_cores_take(lay, kv, d_q, d_k, d_v, d_out);
  const size_t need = workspace_bytes_of(lay, kv, tensor_cores);
  if (need > 0 && (!workspace || workspace_bytes < need)) return TOPLOC_ERR_WORKSPACE;
  if (need > 0 && !aligned(workspace, 32)) return TOPLOC_ERR_INVALID_ARGUMENT;
  const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  if (tensor_cores) return launch_tensor_cores(p, lay, kv, workspace, stream);
  p.splits = splits_of(lay, kv);
  if (p.splits > 1) {
    p.part_out = static_cast<float*>(workspace);
    p.part_lse = p.part_out + (long long)p.splits * p.total_tokens * p.q_heads * p.head_dim;
  }
  return lay->dtype == TOPLOC_DTYPE_BF16 ? launch_all<__nv_bfloat16>(p, stream) : launch_all<float>(p, stream);
}

}  // namespace

extern "C" size_t toploc_attention_workspace_bytes(const toploc_attention_layout* lay, const toploc_kv_layout* kv) {
  if (check_layout(lay, kv) != TOPLOC_OK) return 0;
  // (which kernel takes the call also depends on the pointers: room for either)
  return max(workspace_bytes_of(lay, kv, false), tensor_core_types(lay) ? workspace_bytes_of(lay, kv, true) : 0);
}

extern "C" int toploc_attention_paged(const void* d_q, const void* d_k_cache, const void* d_v_cache,
                                      const toploc_attention_layout* lay, const toploc_kv_layout* kv,
                                      const int32_t* d_block_table, const int32_t* d_seq_offsets,
                                      const int32_t* d_kv_lens, void* d_out, float* d_lse_opt, uint8_t* d_status_opt,
                                      void* d_workspace, size_t workspace_bytes, void* cuda_stream) {
  if (const int rc = check_layout(lay, kv)) return rc;
  if (kv->page_size == 0) return TOPLOC_ERR_INVALID_ARGUMENT;
  if (lay->num_seqs == 0 || lay->max_new_tokens == 0 || lay->total_tokens == 0) return TOPLOC_OK;
  if (!d_q || !d_k_cache || !d_v_cache || !d_seq_offsets || !d_kv_lens || !d_out || (!d_block_table && kv->max_pages > 0))
    return TOPLOC_ERR_INVALID_ARGUMENT;
  return attention(d_q, d_k_cache, d_v_cache, lay, kv, d_block_table, d_seq_offsets, d_kv_lens, d_out, d_lse_opt,
                   d_status_opt, d_workspace, workspace_bytes, cuda_stream);
}

extern "C" int toploc_attention_prompt(const void* d_q, const void* d_k, const void* d_v,
                                       const toploc_attention_layout* lay, const toploc_kv_layout* kv,
                                       const int32_t* d_seq_offsets, void* d_out, float* d_lse_opt,
                                       uint8_t* d_status_opt, void* d_workspace, size_t workspace_bytes,
                                       void* cuda_stream) {
  if (const int rc = check_layout(lay, kv)) return rc;
  if (kv->page_size != 0) return TOPLOC_ERR_INVALID_ARGUMENT;
  if (lay->num_seqs == 0 || lay->max_new_tokens == 0 || lay->total_tokens == 0) return TOPLOC_OK;
  if (!d_q || !d_k || !d_v || !d_seq_offsets || !d_out) return TOPLOC_ERR_INVALID_ARGUMENT;
  return attention(d_q, d_k, d_v, lay, kv, nullptr, d_seq_offsets, nullptr, d_out, d_lse_opt, d_status_opt, d_workspace,
                   workspace_bytes, cuda_stream);
}
