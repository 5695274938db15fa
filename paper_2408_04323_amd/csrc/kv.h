// Shared declarations of the key/value cache operators (scoot_kv_*).
#pragma once

#include <cstdint>

#include "internal.h"

namespace scoot {

struct KvAssignArgs {
  const int32_t* context_len;
  const int32_t* new_len;
  int32_t* block_table;
  const int32_t* free_blocks;
  int32_t* query_start;
  int32_t* seq_len;
  int32_t* positions;
  int64_t* slots;
  int32_t* counts;
  int64_t table_stride, max_tokens;
  int num_seqs, max_blocks, num_free, block_shift;
};

struct KvWriteArgs {
  const void* src[2];  // keys, values
  void* cache[2];
  const int64_t* slots;
  int64_t token_stride[2], head_stride[2];  // elements
  int64_t num_tokens, num_slots;            // num_slots = num_blocks * block_size
  float scale[2];
  int num_heads, head_dim, block_shift;
};

// Vectors turned by their positions, and keys and values into the cache.
struct KvAppendArgs {
  const void* q;  // turned into out: queries, or any vectors
  void* out;
  const void* src[2];  // keys, values
  void* cache[2];
  float* scales[2];  // of every block and key head; null: scale[]
  const int64_t* slots;
  const int32_t* positions;
  const double* freqs;
  double magnitude;
  int64_t q_token_stride, q_head_stride, out_token_stride, out_head_stride;  // elements
  int64_t token_stride[2], head_stride[2];
  int64_t num_tokens, num_slots;  // num_slots = num_blocks * block_size
  float scale[2];
  int num_heads, num_kv_heads;  // either may be 0
  int head_dim, turned, block_shift;  // the first `turned` elements of a head are turned
  bool interleaved, reverse;
};

struct KvAttnArgs {
  const void* q;
  void* out;
  const void* k_cache;
  const void* v_cache;
  const int32_t* block_table;
  const int32_t* query_start;
  const int32_t* seq_len;
  int64_t q_token_stride, q_head_stride, out_token_stride, out_head_stride, table_stride;  // elements
  int64_t num_tokens, num_blocks, max_new_len, max_seq_len;
  int num_heads, num_kv_heads, head_dim, num_seqs, max_blocks, block_shift, window;
  float score_scale;  // scale * k_scale * log2(e): weights are powers of two
  float v_scale;
  const float* k_scales;  // of every block and key head, in the place of the one scale; or null
  const float* v_scales;
  void* workspace;
};

int launch_kv_assign(const KvAssignArgs& a, void* stream);
int launch_kv_write(const KvWriteArgs& a, scoot_kv_type type, scoot_kv_type cache_type, void* stream);
// Keys and values go along if there are key heads; type and cache_type as for writes.
int launch_kv_append(const KvAppendArgs& a, scoot_kv_type type, scoot_kv_type cache_type, void* stream);
uint64_t kv_attention_workspace_bytes(int64_t num_tokens, int num_heads, int num_kv_heads, int head_dim, int num_seqs,
                                      int64_t max_new_len, int64_t max_seq_len, int window);
int launch_kv_attention(const KvAttnArgs& a, scoot_kv_type type, scoot_kv_type cache_type, void* stream);

}  // namespace scoot
