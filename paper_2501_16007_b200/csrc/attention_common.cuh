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
  int page_size, num_pages, max_pages;
  int row_tiles, splits;
};

// A sequence's rows and keys, held to what the call promised.
struct SeqRange {
  int first, rows, keys;
  bool bad;
};

__device__ __forceinline__ SeqRange sequence(const AttentionParams& p, int i) {
  SeqRange s;
  const int a = p.offsets[i], b = p.offsets[i + 1];
  s.first = max(a, 0);
  long long rows = min((long long)b, p.total_tokens) - s.first;
  s.bad = a < 0 || b < a || b > p.total_tokens || rows > p.max_new;
  rows = max(0ll, min(rows, (long long)p.max_new));
  s.rows = (int)rows;
  if (p.kv_lens == nullptr) {
    s.keys = s.rows;
  } else {
    const int kv = p.kv_lens[i];
    const long long most = (long long)p.max_pages * p.page_size;
    s.bad = s.bad || kv < 0 || kv > most;
    s.keys = (int)max(0ll, min((long long)kv, most));
  }
  return s;
}

// ---- the tensor-core kernel (toploc_attention_tc.cu) --------------------------------------------

// Whether the tensor-core kernel takes these types, pointers and strides.
bool tensor_cores_take(const toploc_attention_layout* lay, const toploc_kv_layout* kv, const void* q, const void* k,
                       const void* v, const void* out);
size_t tensor_core_workspace_bytes(const toploc_attention_layout* lay);
int launch_tensor_cores(AttentionParams& p, const toploc_attention_layout* lay, const toploc_kv_layout* kv, void* workspace,
                        cudaStream_t stream);

}  // namespace toploc_model
