// C ABI of the key/value cache operators: argument checks.  See include/scoot.h.
#include <hip/hip_runtime.h>

#include <cmath>
#include <new>

#include "kv.h"

using namespace scoot;

namespace {
bool vector_type(scoot_kv_type t) { return t == SCOOT_KV_F16 || t == SCOOT_KV_BF16; }
bool block_ok(int bs) { return bs >= 8 && bs <= 256 && (bs & (bs - 1)) == 0; }
int shift_of(int bs) { return __builtin_ctz((unsigned)bs); }
bool scale_ok(float s) { return s > 0.0f && std::isfinite(s); }
bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
constexpr int64_t kMaxTokens = ((int64_t)1 << 31) - 1;
// Of a request, where attention counts keys in 32 bits, up to the end of a strip that the last one lies in.
constexpr int64_t kMaxKeys = ((int64_t)1 << 31) - 256;
constexpr int kMaxSeqs = 1 << 20;
constexpr int kMaxHeads = 1024;
constexpr int64_t kMaxBlocks = ((int64_t)1 << 31) - 1;  // tables hold 32-bit block numbers
// Every stride times every index stays in 64 bits.
bool stride_ok(int64_t s) { return s >= 0 && s <= ((int64_t)1 << 31); }

int check_cache(scoot_kv_type type, scoot_kv_type cache_type, int num_kv_heads, int64_t num_blocks, int block_size,
                float k_scale, float v_scale) {
  if (!vector_type(type)) return fail_static(SCOOT_ERR_INVALID_ARG, "kv cache: type must be F16 or BF16");
  if (cache_type != type && cache_type != SCOOT_KV_F8)
    return fail_static(SCOOT_ERR_INVALID_ARG, "kv cache: cache_type must be the vectors' type or F8");
  if (num_kv_heads < 1 || num_kv_heads > kMaxHeads)
    return fail_static(SCOOT_ERR_INVALID_ARG, "kv cache: num_kv_heads must be in 1..1024");
  if (!block_ok(block_size))
    return fail_static(SCOOT_ERR_INVALID_ARG, "kv cache: block_size must be a power of two in 8..256");
  if (num_blocks < 0 || num_blocks > kMaxBlocks) return fail_static(SCOOT_ERR_INVALID_ARG, "kv cache: num_blocks out of range");
  if (!scale_ok(k_scale) || !scale_ok(v_scale))
    return fail_static(SCOOT_ERR_INVALID_ARG, "kv cache: scales must be positive and finite");
  if (cache_type != SCOOT_KV_F8 && (k_scale != 1.0f || v_scale != 1.0f))
    return fail_static(SCOOT_ERR_INVALID_ARG, "kv cache: scales other than 1 need an 8-bit cache");
  return SCOOT_OK;
}

// No exception leaves a C entry.
template <typename F>
int guarded(F launch) {
  try {
    return launch();
  } catch (const std::bad_alloc&) {
    return fail_static(SCOOT_ERR_NO_MEMORY, "kv cache: host allocation failed");
  }
}

int check_attention_sizes(int64_t num_tokens, int num_heads, int num_kv_heads, int head_dim, int num_seqs,
                          int64_t max_new_len, int64_t max_seq_len, int window) {
  if (num_tokens < 0 || num_tokens > kMaxTokens)
    return fail_static(SCOOT_ERR_INVALID_ARG, "kv attention: num_tokens out of range");
  if (num_seqs < 0 || num_seqs > kMaxSeqs) return fail_static(SCOOT_ERR_INVALID_ARG, "kv attention: num_seqs must be in 0..2^20");
  if (num_kv_heads < 1 || num_heads < 1 || num_heads > kMaxHeads || num_heads % num_kv_heads != 0)
    return fail_static(SCOOT_ERR_INVALID_ARG, "kv attention: num_heads must be a multiple of num_kv_heads, at most 1024");
  if (head_dim != 64 && head_dim != 128 && head_dim != 192 && head_dim != 256)
    return fail_static(SCOOT_ERR_UNSUPPORTED, "kv attention: head_dim must be 64, 128, 192 or 256");
  if (max_new_len < 0 || max_seq_len < 0 || max_new_len > kMaxTokens || max_seq_len > kMaxTokens)
    return fail_static(SCOOT_ERR_INVALID_ARG, "kv attention: max_new_len and max_seq_len must be in 0..2^31-1");
  if (window < 0) return fail_static(SCOOT_ERR_INVALID_ARG, "kv attention: window must be >= 0");
  return SCOOT_OK;
}
}  // namespace

extern "C" {

int scoot_kv_assign(const int32_t* context_len, const int32_t* new_len, int num_seqs, int block_size,
                    int32_t* block_table, int max_blocks, int64_t table_stride, const int32_t* free_blocks,
                    int num_free, int64_t max_tokens, int32_t* query_start, int32_t* seq_len, int32_t* positions,
                    int64_t* slots, int32_t* counts, void* stream) {
  clear_error();
  if (num_seqs < 0 || num_seqs > kMaxSeqs) return fail_static(SCOOT_ERR_INVALID_ARG, "kv assign: num_seqs must be in 0..2^20");
  if (!block_ok(block_size))
    return fail_static(SCOOT_ERR_INVALID_ARG, "kv assign: block_size must be a power of two in 8..256");
  if (max_blocks < 0 || max_blocks > (int)(kMaxTokens / block_size) || num_free < 0 || max_tokens < 0 || max_tokens > kMaxTokens)
    return fail_static(SCOOT_ERR_INVALID_ARG, "kv assign: max_blocks, num_free or max_tokens out of range");
  if (table_stride < max_blocks || !stride_ok(table_stride))
    return fail_static(SCOOT_ERR_INVALID_ARG, "kv assign: table_stride must be at least max_blocks");
  if (!query_start || !counts || (num_seqs > 0 && (!context_len || !new_len || !seq_len)) ||
      (num_seqs > 0 && max_blocks > 0 && !block_table) || (num_free > 0 && !free_blocks) ||
      (max_tokens > 0 && (!positions || !slots)))
    return fail_static(SCOOT_ERR_INVALID_ARG, "kv assign: null pointer");
  KvAssignArgs a{};
  a.context_len = context_len;
  a.new_len = new_len;
  a.block_table = block_table;
  a.free_blocks = free_blocks;
  a.query_start = query_start;
  a.seq_len = seq_len;
  a.positions = positions;
  a.slots = slots;
  a.counts = counts;
  a.table_stride = table_stride;
  a.max_tokens = max_tokens;
  a.num_seqs = num_seqs;
  a.max_blocks = max_blocks;
  a.num_free = num_free;
  a.block_shift = shift_of(block_size);
  return guarded([&] { return launch_kv_assign(a, stream); });
}

int scoot_kv_write(const void* k, const void* v, scoot_kv_type type, int64_t num_tokens, int num_kv_heads,
                   int head_dim, int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride,
                   int64_t v_head_stride, const int64_t* slots, void* k_cache, void* v_cache,
                   scoot_kv_type cache_type, int64_t num_blocks, int block_size, float k_scale, float v_scale,
                   void* stream) {
  clear_error();
  int rc = check_cache(type, cache_type, num_kv_heads, num_blocks, block_size, k_scale, v_scale);
  if (rc != SCOOT_OK) return rc;
  if (head_dim < 8 || head_dim > 1024 || head_dim % 8 != 0)
    return fail_static(SCOOT_ERR_UNSUPPORTED, "kv write: head_dim must be a multiple of 8, at most 1024");
  if (num_tokens < 0 || num_tokens > kMaxTokens) return fail_static(SCOOT_ERR_INVALID_ARG, "kv write: num_tokens out of range");
  if (!stride_ok(k_token_stride) || !stride_ok(k_head_stride) || !stride_ok(v_token_stride) || !stride_ok(v_head_stride))
    return fail_static(SCOOT_ERR_INVALID_ARG, "kv write: stride out of range");
  if (num_tokens == 0 || num_blocks == 0) return SCOOT_OK;
  if (!k || !v || !slots || !k_cache || !v_cache) return fail_static(SCOOT_ERR_INVALID_ARG, "kv write: null pointer");
  if (((uintptr_t)k | (uintptr_t)v) & 1) return fail_static(SCOOT_ERR_INVALID_ARG, "kv write: vectors not aligned to their elements");
  if (!aligned16(k_cache) || !aligned16(v_cache))
    return fail_static(SCOOT_ERR_INVALID_ARG, "kv write: the cache must be 16-byte aligned");
  KvWriteArgs a{};
  a.src[0] = k;
  a.src[1] = v;
  a.cache[0] = k_cache;
  a.cache[1] = v_cache;
  a.slots = slots;
  a.token_stride[0] = k_token_stride;
  a.token_stride[1] = v_token_stride;
  a.head_stride[0] = k_head_stride;
  a.head_stride[1] = v_head_stride;
  a.num_tokens = num_tokens;
  a.num_slots = num_blocks * block_size;
  a.scale[0] = k_scale;
  a.scale[1] = v_scale;
  a.num_heads = num_kv_heads;
  a.head_dim = head_dim;
  a.block_shift = shift_of(block_size);
  return guarded([&] { return launch_kv_write(a, type, cache_type, stream); });
}

int scoot_kv_attention_workspace(int64_t num_tokens, int num_heads, int num_kv_heads, int head_dim, int num_seqs,
                                 int64_t max_new_len, int64_t max_seq_len, int window, uint64_t* bytes) {
  clear_error();
  if (!bytes) return fail_static(SCOOT_ERR_INVALID_ARG, "kv attention: null output");
  const int rc = check_attention_sizes(num_tokens, num_heads, num_kv_heads, head_dim, num_seqs, max_new_len, max_seq_len, window);
  if (rc != SCOOT_OK) return rc;
  *bytes = kv_attention_workspace_bytes(num_tokens, num_heads, num_kv_heads, head_dim, num_seqs, max_new_len, max_seq_len, window);
  return SCOOT_OK;
}

int scoot_kv_attention(const void* q, scoot_kv_type type, int64_t num_tokens, int num_heads, int num_kv_heads,
                       int head_dim, int64_t q_token_stride, int64_t q_head_stride, const void* k_cache,
                       const void* v_cache, scoot_kv_type cache_type, int64_t num_blocks, int block_size,
                       const int32_t* block_table, int max_blocks, int64_t table_stride, const int32_t* query_start,
                       const int32_t* seq_len, int num_seqs, int64_t max_new_len, int64_t max_seq_len, float scale,
                       int window, float k_scale, float v_scale, void* out, int64_t out_token_stride,
                       int64_t out_head_stride, void* workspace, uint64_t workspace_bytes, void* stream) {
  clear_error();
  int rc = check_cache(type, cache_type, num_kv_heads, num_blocks, block_size, k_scale, v_scale);
  if (rc == SCOOT_OK)
    rc = check_attention_sizes(num_tokens, num_heads, num_kv_heads, head_dim, num_seqs, max_new_len, max_seq_len, window);
  if (rc != SCOOT_OK) return rc;
  if (!std::isfinite(scale) || scale < 0.0f)
    return fail_static(SCOOT_ERR_INVALID_ARG, "kv attention: scale must be finite and not negative");
  const float score_scale = scale * k_scale * 1.44269504088896340736f;  // log2(e): weights are powers of two
  if (!std::isfinite(score_scale))
    return fail_static(SCOOT_ERR_INVALID_ARG, "kv attention: scale * k_scale is too large");
  if (max_blocks < 0 || max_blocks > (int)(kMaxKeys / block_size) || table_stride < max_blocks || !stride_ok(table_stride))
    return fail_static(SCOOT_ERR_INVALID_ARG, "kv attention: max_blocks or table_stride out of range");
  if (!stride_ok(q_token_stride) || !stride_ok(q_head_stride) || !stride_ok(out_token_stride) || !stride_ok(out_head_stride))
    return fail_static(SCOOT_ERR_INVALID_ARG, "kv attention: stride out of range");
  if (num_tokens == 0 || num_seqs == 0) return SCOOT_OK;
  if (!q || !out || !query_start || !seq_len || (max_blocks > 0 && !block_table) || (num_blocks > 0 && (!k_cache || !v_cache)))
    return fail_static(SCOOT_ERR_INVALID_ARG, "kv attention: null pointer");
  if (!aligned16(q) || !aligned16(out) || !aligned16(k_cache) || !aligned16(v_cache) ||
      ((q_token_stride | q_head_stride | out_token_stride | out_head_stride) & 7))
    return fail_static(SCOOT_ERR_INVALID_ARG, "kv attention: q, out and the cache must be 16-byte aligned, rows included");
  const uint64_t need =
      kv_attention_workspace_bytes(num_tokens, num_heads, num_kv_heads, head_dim, num_seqs, max_new_len, max_seq_len, window);
  if (need > 0 && (!workspace || workspace_bytes < need || !aligned16(workspace)))
    return fail_static(SCOOT_ERR_INVALID_ARG, "kv attention: workspace missing, too small or not 16-byte aligned");
  KvAttnArgs a{};
  a.q = q;
  a.out = out;
  a.k_cache = k_cache;
  a.v_cache = v_cache;
  a.block_table = block_table;
  a.query_start = query_start;
  a.seq_len = seq_len;
  a.q_token_stride = q_token_stride;
  a.q_head_stride = q_head_stride;
  a.out_token_stride = out_token_stride;
  a.out_head_stride = out_head_stride;
  a.table_stride = table_stride;
  a.num_tokens = num_tokens;
  a.num_blocks = num_blocks;
  a.max_new_len = max_new_len;
  a.max_seq_len = max_seq_len;
  a.num_heads = num_heads;
  a.num_kv_heads = num_kv_heads;
  a.head_dim = head_dim;
  a.num_seqs = num_seqs;
  a.max_blocks = num_blocks > 0 ? max_blocks : 0;  // a cache without blocks holds no tokens
  a.block_shift = shift_of(block_size);
  a.window = window;
  // The smallest positive float in the place of 0: it leaves nothing of a score, and -inf stays -inf.
  a.score_scale = std::max(score_scale, 1.4e-45f);
  a.v_scale = v_scale;
  a.workspace = workspace;
  return guarded([&] { return launch_kv_attention(a, type, cache_type, stream); });
}

}  // extern "C"
