// What the attention kernels share: the call as the device sees it, and how a sequence's keys are split.
#pragma once

#include "model_common.cuh"

namespace toploc_model {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kSms = 148;      // of a B200: sizes the workspace and the split, whatever device answers
constexpr int kKeyTile = 128;  // keys of a tile of the tensor-core kernel

struct AttentionParams {
  const void* q;
  const void* k;
  const void* v;
  void* out;
  float* lse;
  uint8_t* status;
  float* part_out;  // results over a part of the keys, and their lse (base 2)
  float* part_lse;
  const int32_t* table;
  const int32_t* offsets;
  const int32_t* kv_lens;  // NULL: a prompt attends over its own rows
  long long total_tokens;
  long long q_token, q_head, out_token, out_head;
  long long k_page, k_token, k_head, v_page, v_token, v_head, table_stride;
  float scale_log2;
  int head_dim, q_heads, kv_heads, group, num_seqs, max_new;
  int page_size, num_pages, max_pages, most_keys;
  int row_tiles, splits;
};

// A sequence's rows and keys, held to what the call promised.
struct SeqRange {
  int first, rows, keys;
  bool bad;
};

// (32 bits are enough: total_tokens, and most_keys = max_pages * page_size, are held below 2^31 by the entry points)
__device__ __forceinline__ SeqRange sequence(const AttentionParams& p, int i) {
  const int a = p.offsets[i], b = p.offsets[i + 1], total = (int)p.total_tokens;
  SeqRange s;
  s.first = max(a, 0);
  const int rows = b > s.first ? min(b, total) - s.first : 0;
  s.bad = a < 0 || b < a || b > total || rows > p.max_new;
  s.rows = max(min(rows, p.max_new), 0);
  s.keys = s.rows;
  if (p.kv_lens != nullptr) {
    const int kv = p.kv_lens[i];
    s.bad = s.bad || kv < 0 || kv > p.most_keys;
    s.keys = max(min(kv, p.most_keys), 0);
  }
  return s;
}

// ---- the tensor-core kernel (toploc_attention_tc.cu) --------------------------------------------

// Whether the tensor-core kernel takes these types, pointers and strides.
bool tensor_cores_take(const toploc_attention_layout* lay, const toploc_kv_layout* kv, const void* q, const void* k,
                       const void* v, const void* out);
size_t tensor_core_workspace_bytes(const toploc_attention_layout* lay, const toploc_kv_layout* kv);
int launch_tensor_cores(AttentionParams& p, const toploc_attention_layout* lay, const toploc_kv_layout* kv, void* workspace,
                        cudaStream_t stream);

}  // namespace toploc_model
