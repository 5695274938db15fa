// Attention over the block cache: a call's plan, workspace and limits, and the way to the launches of its head dimension.
#include "kv_attn.h"

namespace scoot {
namespace kvattn {
// Instantiated in k_kv_attn_<dim>.hip.
template <>
int launch_dim<64>(const KvAttnArgs&, const Plan&, scoot_kv_type, bool, float*, float*, hipStream_t);
template <>
int launch_dim<128>(const KvAttnArgs&, const Plan&, scoot_kv_type, bool, float*, float*, hipStream_t);
template <>
int launch_dim<192>(const KvAttnArgs&, const Plan&, scoot_kv_type, bool, float*, float*, hipStream_t);
template <>
int launch_dim<256>(const KvAttnArgs&, const Plan&, scoot_kv_type, bool, float*, float*, hipStream_t);
}  // namespace kvattn
namespace {
using namespace kvattn;

int64_t slots(const Plan& p, int num_kv_heads) {
  return p.splits > 1 ? p.items * p.splits * num_kv_heads * (p.tile_rows ? p.tile_rows : kFew) : 0;
}
}  // namespace

uint64_t kv_attention_workspace_bytes(int64_t num_tokens, int num_heads, int num_kv_heads, int head_dim, int num_seqs,
                                      int64_t max_new_len, int64_t max_seq_len, int window) {
  int64_t most = 0;  // of a 16-bit and an 8-bit cache
  for (int bytes = 1; bytes <= 2; ++bytes)
    most = std::max(most, slots(plan(num_tokens, num_heads, num_kv_heads, head_dim, bytes, num_seqs, max_new_len, max_seq_len, window),
                                num_kv_heads));
  return (uint64_t)most * (head_dim + 2) * 4;
}

int launch_kv_attention(const KvAttnArgs& a, scoot_kv_type type, scoot_kv_type cache_type, void* stream) {
  const Plan p = plan(a.num_tokens, a.num_heads, a.num_kv_heads, a.head_dim, cache_type == SCOOT_KV_F8 ? 1 : 2, a.num_seqs,
                      a.max_new_len, a.max_seq_len, a.window);
  // A launch has less than 2^32 threads: a workgroup per part of an item and key head; in a join, per 4 rows at least.
  const int64_t groups = p.items * a.num_kv_heads;
  const int64_t joins = p.splits > 1 ? groups * (p.tile_rows ? p.tile_rows : kFew) / 4 * kThreads : 0;
  if (std::max(groups * p.splits * 64 * p.waves, joins) > 0xffffffffLL)
    return fail_static(SCOOT_ERR_UNSUPPORTED, "kv attention: too many rows for one call");
  float* parts = (float*)a.workspace;
  float* stats = parts + slots(p, a.num_kv_heads) * a.head_dim;
  const hipStream_t s = (hipStream_t)stream;
  const bool f8 = cache_type == SCOOT_KV_F8;
  switch (a.head_dim) {
    case 64: return launch_dim<64>(a, p, type, f8, parts, stats, s);
    case 128: return launch_dim<128>(a, p, type, f8, parts, stats, s);
    case 192: return launch_dim<192>(a, p, type, f8, parts, stats, s);
    default: return launch_dim<256>(a, p, type, f8, parts, stats, s);
  }
}

}  // namespace scoot
