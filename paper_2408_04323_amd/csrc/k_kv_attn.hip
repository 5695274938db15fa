// How an attention call over the block cache is split, and its launches.
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

constexpr int64_t kUnits = 256;   // compute units
constexpr int kPartOf = 128;      // parts are multiples of this many keys: a strip of 32 for each of four waves
constexpr int kMinPart = 512;     // and not smaller than this: a part costs about as much as 256 keys to join
constexpr int kAlone = 2048;      // keys that eight waves of one workgroup do not share with another

// Requests of at most 16 rows (new tokens x heads per key head) are items of
// their own; once some have more, tiles of 128 (64) rows are.  Where the items do
// not fill the chip (tiles), or not four times over (few rows, whose lengths
// differ most), their keys are split into parts.
Plan plan(int64_t num_tokens, int num_heads, int num_kv_heads, int head_dim, int element_bytes, int num_seqs, int64_t max_new_len,
          int64_t max_seq_len, int window) {
  Plan p{};
  const int64_t G = num_heads / num_kv_heads;
  const int64_t longest = std::min<int64_t>(max_new_len, num_tokens);
  const bool tiles = longest * G > kFew;
  p.tile_rows = tiles ? tile_rows(head_dim) : 0;
  p.items = tiles ? num_tokens * G / p.tile_rows + num_seqs : num_seqs;
  int64_t keys = max_seq_len;
  if (window > 0) keys = std::min<int64_t>(keys, (int64_t)window + (tiles ? p.tile_rows / G : longest) + 32);
  keys = std::max<int64_t>(keys, 1);
  const int64_t groups = std::max<int64_t>(1, p.items * num_kv_heads);
  const int64_t resident = kUnits * (tiles && head_dim <= 64 ? 3 : 2);
  int64_t want = std::max<int64_t>(1, (tiles ? resident : 4 * resident) / groups);
  // Few items of few rows: eight waves each.
  p.waves = !tiles && groups <= kUnits && head_dim * element_bytes <= kWideRow ? 8 : kWaves;
  if (p.waves == 8) want = keys <= kAlone ? 1 : std::max<int64_t>(1, 2 * kUnits / groups);
  int64_t part = (keys + want - 1) / want;
  part = std::max<int64_t>(kMinPart * (p.waves / kWaves), (part + kPartOf - 1) / kPartOf * kPartOf);
  p.part = (int)std::min<int64_t>(part, (int64_t)1 << 30);
  p.splits = (int)((keys + p.part - 1) / p.part);
  p.deep = groups * p.splits <= kUnits;
  return p;
}

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
  if (p.items * std::max(p.splits, tile_rows(64) / 4) * a.num_kv_heads > 0x7fffffff)
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
