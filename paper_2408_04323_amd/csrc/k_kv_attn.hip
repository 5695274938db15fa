// Attention of a step's tokens over the block cache (scoot_kv_attention).
#include <hip/hip_runtime.h>

#include "kv.h"

namespace scoot {
namespace {

// One wave per token and query head: a key at a time, the lanes share the head
// dimension, the softmax's maximum and sum run along.
constexpr int kWaves = 4;

template <typename T>
__device__ __forceinline__ float load1(const T* p) {
  return (float)*p;
}
__device__ __forceinline__ float load1(const uint8_t* p) { return __builtin_amdgcn_cvt_f32_fp8((int)*p, 0); }

template <typename T, typename C, int D>
__global__ __launch_bounds__(64 * kWaves) void kv_attention_simple(KvAttnArgs a) {
  constexpr int E = D / 64;
  const int lane = threadIdx.x & 63;
  const int64_t item = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  const int64_t t = item / a.num_heads;
  const int h = (int)(item - t * a.num_heads);
  if (t >= a.num_tokens) return;
  if (t < a.query_start[0] || t >= a.query_start[a.num_seqs]) return;
  int lo = 0, hi = a.num_seqs;  // query_start[lo] <= t < query_start[hi]
  while (hi - lo > 1) {
    const int m = (lo + hi) >> 1;
    if (a.query_start[m] <= t) lo = m;
    else hi = m;
  }
  const int64_t cap = (int64_t)a.max_blocks << a.block_shift;
  int64_t len = a.seq_len[lo];
  int64_t end = a.query_start[lo + 1];
  const int64_t pos = len - (end - t);
  int64_t last = pos < cap - 1 ? pos : cap - 1;
  int64_t p0 = a.window > 0 && pos - a.window + 1 > 0 ? pos - a.window + 1 : 0;
  const int kvh = h / (a.num_heads / a.num_kv_heads);
  const T* q = (const T*)a.q + t * a.q_token_stride + h * a.q_head_stride;
  float qv[E], o[E] = {};
  for (int e = 0; e < E; ++e) qv[e] = (float)q[lane + 64 * e];
  float m = -INFINITY, l = 0.0f;
  const int bs = 1 << a.block_shift;
  for (int64_t p = p0; p <= last; ++p) {
    const int64_t block = a.block_table[(int64_t)lo * a.table_stride + (p >> a.block_shift)];
    if (block < 0 || block >= a.num_blocks) continue;
    const int64_t row = (((block * a.num_kv_heads + kvh) << a.block_shift) + (p & (bs - 1))) * D;
    float s = 0.0f;
    for (int e = 0; e < E; ++e) s += qv[e] * load1((const C*)a.k_cache + row + lane + 64 * e);
    for (int w = 32; w > 0; w >>= 1) s += __shfl_xor(s, w);
    s *= a.score_scale;
    const float mn = fmaxf(m, s), f = exp2f(m - mn), w = exp2f(s - mn);
    m = mn;
    l = l * f + w;
    for (int e = 0; e < E; ++e) o[e] = o[e] * f + w * load1((const C*)a.v_cache + row + lane + 64 * e);
  }
  T* out = (T*)a.out + t * a.out_token_stride + h * a.out_head_stride;
  const float inv = l == 0.0f ? 0.0f : a.v_scale / l;
  for (int e = 0; e < E; ++e) out[lane + 64 * e] = (T)(l == 0.0f ? 0.0f : o[e] * inv);
}

int launched(const char* what) {
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return fail(SCOOT_ERR_DEVICE, std::string(what) + ": " + hipGetErrorString(err));
  return SCOOT_OK;
}

template <typename T, typename C>
int launch_dim(const KvAttnArgs& a, hipStream_t s) {
  const int64_t items = a.num_tokens * a.num_heads;
  const dim3 grid((unsigned)((items + kWaves - 1) / kWaves)), block(64 * kWaves);
  if (a.head_dim == 64) hipLaunchKernelGGL((kv_attention_simple<T, C, 64>), grid, block, 0, s, a);
  else if (a.head_dim == 128) hipLaunchKernelGGL((kv_attention_simple<T, C, 128>), grid, block, 0, s, a);
  else if (a.head_dim == 192) hipLaunchKernelGGL((kv_attention_simple<T, C, 192>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((kv_attention_simple<T, C, 256>), grid, block, 0, s, a);
  return launched("kv attention launch");
}

}  // namespace

uint64_t kv_attention_workspace_bytes(int64_t, int, int, int, int, int64_t, int64_t, int) { return 0; }

int launch_kv_attention(const KvAttnArgs& a, scoot_kv_type type, scoot_kv_type cache_type, void* stream) {
  const hipStream_t s = (hipStream_t)stream;
  const bool f8 = cache_type == SCOOT_KV_F8;
  if (type == SCOOT_KV_F16) return f8 ? launch_dim<_Float16, uint8_t>(a, s) : launch_dim<_Float16, _Float16>(a, s);
  return f8 ? launch_dim<__bf16, uint8_t>(a, s) : launch_dim<__bf16, __bf16>(a, s);
}

}  // namespace scoot
