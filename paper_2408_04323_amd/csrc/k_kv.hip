// Slots of a step's tokens in the block cache, and the writes to them
// (scoot_kv_assign, scoot_kv_write).
#include <hip/hip_runtime.h>

#include "kv.h"

namespace scoot {
namespace {

// ---------------------------------------------------------------- assignment
//
// With n_i new tokens, c_i cached ones and blocks of B: request i holds
// u_i = ceil(c_i / B) blocks and needs d_i = ceil((c_i + n_i) / B) - u_i more
// (0 if its tokens or blocks do not fit).  Prefix sums of n and d give its
// first token and its first free block; token t of request i stands at
// position p = c_i + t - start_i in block p / B, which is the table's entry if
// p / B < u_i and free block first_i + p / B - u_i otherwise.
//
// Latency bounds this: some kilobytes, a chain of dependent loads.  So one
// launch: every workgroup makes the prefix sums of all requests for itself (64
// KiB of lengths at 8192 requests, out of L2), keeps them in LDS, and then
// serves its own share of the tokens, each found by a binary search in LDS.
// The token that opens a new block writes the table's entry, so no workgroup
// waits for another.
constexpr int kAssignThreads = 1024;
constexpr int kAssignPer = 4;  // requests per thread and tile
constexpr int kAssignTile = kAssignThreads * kAssignPer;
constexpr int kAssignTokens = 2048;  // tokens per workgroup, as long as that makes at most kAssignGroups of them
constexpr int kAssignGroups = 256;

__device__ __forceinline__ int sat32(int64_t v) { return v > 0x7fffffff ? 0x7fffffff : (int)v; }

struct Sums {
  int64_t tokens, blocks;
};

// Exclusive prefix sums over the workgroup's threads, and the totals.
__device__ __forceinline__ Sums scan_workgroup(Sums v, Sums* total, Sums* wave_sum) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Sums x = v;
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t t = __shfl_up((long long)x.tokens, o), b = __shfl_up((long long)x.blocks, o);
    if (lane >= o) {
      x.tokens += t;
      x.blocks += b;
    }
  }
  if (lane == 63) wave_sum[wave] = x;
  __syncthreads();
  Sums before{0, 0}, all{0, 0};
  for (int w = 0; w < kAssignThreads / 64; ++w) {
    if (w < wave) {
      before.tokens += wave_sum[w].tokens;
      before.blocks += wave_sum[w].blocks;
    }
    all.tokens += wave_sum[w].tokens;
    all.blocks += wave_sum[w].blocks;
  }
  *total = all;
  return {before.tokens + x.tokens - v.tokens, before.blocks + x.blocks - v.blocks};
}

__global__ __launch_bounds__(kAssignThreads) void kv_assign_kernel(KvAssignArgs a, int64_t per_group) {
  __shared__ Sums wave_sum[kAssignThreads / 64];
  __shared__ int start[kAssignTile + 1];  // first token of a request, from the tile's first one
  __shared__ int ctx[kAssignTile];        // cached tokens; -1: not admitted
  __shared__ int first[kAssignTile];      // first of its new blocks in the free list
  __shared__ int n_admitted;
  __shared__ int taken;

  const int tid = threadIdx.x;
  const int bs = 1 << a.block_shift;
  const int64_t t_lo = (int64_t)blockIdx.x * per_group;
  const int64_t t_hi = t_lo + per_group < a.max_tokens ? t_lo + per_group : a.max_tokens;
  if (tid == 0) n_admitted = taken = 0;
  Sums base{0, 0};
  for (int r0 = 0, tile = 0; r0 < a.num_seqs; r0 += kAssignTile, ++tile) {
    const bool writes = tile % (int)gridDim.x == (int)blockIdx.x;  // this workgroup stores the tile's lengths
    int c[kAssignPer], n[kAssignPer];
    // First the tokens alone decide which requests ask for blocks.
    int64_t tok = 0;
    for (int j = 0; j < kAssignPer; ++j) {
      const int r = r0 + tid * kAssignPer + j;
      c[j] = r < a.num_seqs ? max(a.context_len[r], 0) : 0;
      n[j] = r < a.num_seqs ? max(a.new_len[r], 0) : 0;
      tok += n[j];
    }
    Sums total;
    const Sums st = scan_workgroup({tok, 0}, &total, wave_sum);
    __syncthreads();
    int64_t end = base.tokens + st.tokens, blk = 0;
    int64_t need[kAssignPer];
    bool fits[kAssignPer];
    for (int j = 0; j < kAssignPer; ++j) {
      end += n[j];
      const int64_t used = ((int64_t)c[j] + bs - 1) >> a.block_shift;
      const int64_t all = ((int64_t)c[j] + n[j] + bs - 1) >> a.block_shift;
      fits[j] = end <= a.max_tokens && all <= a.max_blocks;
      need[j] = fits[j] ? all - used : 0;
      blk += need[j];
    }
    Sums total_b;
    const Sums sb = scan_workgroup({0, blk}, &total_b, wave_sum);
    int64_t tstart = base.tokens + st.tokens, bstart = base.blocks + sb.blocks;
    int ok_count = 0, last_taken = 0;
    for (int j = 0; j < kAssignPer; ++j) {
      const int i = tid * kAssignPer + j, r = r0 + i;
      const bool ok = r < a.num_seqs && fits[j] && (need[j] == 0 || bstart + need[j] <= a.num_free);
      start[i] = sat32(tstart - base.tokens);
      ctx[i] = ok ? c[j] : -1;
      first[i] = sat32(bstart);
      if (ok) {
        ++ok_count;
        if (need[j] > 0) last_taken = sat32(bstart + need[j]);
      }
      if (writes && r < a.num_seqs) {
        a.query_start[r] = sat32(tstart);
        a.seq_len[r] = ok ? sat32((int64_t)c[j] + n[j]) : 0;
      }
      tstart += n[j];
      bstart += need[j];
    }
    if (tid == 0) start[kAssignTile] = sat32(total.tokens);
    if (blockIdx.x == 0 && ok_count) {
      atomicAdd(&n_admitted, ok_count);
      atomicMax(&taken, last_taken);
    }
    __syncthreads();

    // Tokens of this workgroup that belong to this tile's requests.
    const int64_t lo = t_lo > base.tokens ? t_lo : base.tokens;
    const int64_t tile_end = base.tokens + total.tokens;
    const int64_t hi = t_hi < tile_end ? t_hi : tile_end;
    for (int64_t t = lo + tid; t < hi; t += kAssignThreads) {
      const int at = (int)(t - base.tokens);
      int i = 0, e = kAssignTile;  // start[i] <= at < start[e]
      while (e - i > 1) {
        const int m = (i + e) >> 1;
        if (start[m] <= at) i = m;
        else e = m;
      }
      int pos = -1;
      int64_t slot = -1;
      if (ctx[i] >= 0) {
        const int r = r0 + i;
        pos = ctx[i] + at - start[i];
        const int b = pos >> a.block_shift;
        const int used = (int)(((int64_t)ctx[i] + bs - 1) >> a.block_shift);
        int32_t* entry = a.block_table + (int64_t)r * a.table_stride + b;
        int block;
        if (b < used) {
          block = *entry;
        } else {
          block = a.free_blocks[first[i] + b - used];
          if ((pos & (bs - 1)) == 0) *entry = block;
        }
        if (block >= 0) slot = ((int64_t)block << a.block_shift) + (pos & (bs - 1));
      }
      a.positions[t] = pos;
      a.slots[t] = slot;
    }
    base.tokens += total.tokens;
    base.blocks += total_b.blocks;
    __syncthreads();
  }
  for (int64_t t = (t_lo > base.tokens ? t_lo : base.tokens) + tid; t < t_hi; t += kAssignThreads) {
    a.positions[t] = -1;
    a.slots[t] = -1;
  }
  if (blockIdx.x == 0 && tid == 0) {
    a.query_start[a.num_seqs] = sat32(base.tokens);
    a.counts[0] = sat32(base.tokens);
    a.counts[1] = n_admitted;
    a.counts[2] = taken;
    a.counts[3] = sat32(base.blocks);
  }
}

// --------------------------------------------------------------------- writes
//
// A thread moves eight elements of one token's key (or value) head; the
// cache's rows are the vectors' rows, so both sides are whole cache lines.
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
template <typename T>
struct Vec8;
template <>
struct Vec8<_Float16> {
  typedef h8 type;
};
template <>
struct Vec8<__bf16> {
  typedef b8 type;
};

// Nearest 8-bit float (e4m3) of x / scale, limited to the largest finite one; NaN stays NaN.
__device__ __forceinline__ float limit_f8(float x, float scale) {
  x /= scale;
  return x > 448.0f ? 448.0f : x < -448.0f ? -448.0f : x;
}

constexpr int kWriteThreads = 256;

template <typename T, bool F8, bool ALIGNED>
__global__ __launch_bounds__(kWriteThreads) void kv_write_kernel(KvWriteArgs a) {
  const uint32_t chunks = (uint32_t)a.head_dim / 8, per_token = chunks * (uint32_t)a.num_heads;
  const int64_t total = a.num_tokens * per_token;
  for (int64_t i = (int64_t)blockIdx.x * kWriteThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kWriteThreads) {
    const int64_t t = i / per_token;
    const uint32_t r = (uint32_t)(i - t * per_token), h = r / chunks, c = r - h * chunks;
    const int64_t slot = a.slots[t];
    if (slot < 0 || slot >= a.num_slots) continue;
    const int64_t block = slot >> a.block_shift, at = slot & ((1 << a.block_shift) - 1);
    const int64_t to = ((((block * a.num_heads + h) << a.block_shift) + at) * a.head_dim) + c * 8;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const T* p = (const T*)a.src[s] + t * a.token_stride[s] + h * a.head_stride[s] + c * 8;
      typename Vec8<T>::type x;
      if (ALIGNED) {
        x = *(const typename Vec8<T>::type*)p;
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = p[j];
      }
      if (F8) {
        int w[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float f[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) f[k] = limit_f8((float)x[4 * j + k], a.scale[s]);
          w[j] = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
          w[j] = __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], w[j], true);
        }
        *(int2*)((uint8_t*)a.cache[s] + to) = make_int2(w[0], w[1]);
      } else {
        *(typename Vec8<T>::type*)((T*)a.cache[s] + to) = x;
      }
    }
  }
}

int launched(const char* what) {
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return fail(SCOOT_ERR_DEVICE, std::string(what) + ": " + hipGetErrorString(err));
  return SCOOT_OK;
}

template <typename T, bool F8>
void write_launch(const KvWriteArgs& a, bool aligned, dim3 grid, hipStream_t s) {
  if (aligned)
    hipLaunchKernelGGL((kv_write_kernel<T, F8, true>), grid, dim3(kWriteThreads), 0, s, a);
  else
    hipLaunchKernelGGL((kv_write_kernel<T, F8, false>), grid, dim3(kWriteThreads), 0, s, a);
}

}  // namespace

int launch_kv_assign(const KvAssignArgs& a, void* stream) {
  const int64_t most = (a.max_tokens + kAssignTokens - 1) / kAssignTokens;
  const int groups = (int)std::max<int64_t>(1, std::min<int64_t>(most, kAssignGroups));
  const int64_t per_group = (a.max_tokens + groups - 1) / groups;
  hipLaunchKernelGGL(kv_assign_kernel, dim3(groups), dim3(kAssignThreads), 0, (hipStream_t)stream, a, per_group);
  return launched("kv assign launch");
}

int launch_kv_write(const KvWriteArgs& a, scoot_kv_type type, scoot_kv_type cache_type, void* stream) {
  const int64_t total = a.num_tokens * (a.head_dim / 8) * a.num_heads;
  const dim3 grid((unsigned)std::min<int64_t>((total + kWriteThreads - 1) / kWriteThreads, 1 << 20));
  const hipStream_t s = (hipStream_t)stream;
  bool aligned = true;  // every row starts on 16 bytes
  for (int i = 0; i < 2; ++i)
    aligned = aligned && ((uintptr_t)a.src[i] & 15) == 0 && ((a.token_stride[i] | a.head_stride[i]) & 7) == 0;
  const bool f8 = cache_type == SCOOT_KV_F8;
  if (type == SCOOT_KV_F16) {
    if (f8) write_launch<_Float16, true>(a, aligned, grid, s);
    else write_launch<_Float16, false>(a, aligned, grid, s);
  } else {
    if (f8) write_launch<__bf16, true>(a, aligned, grid, s);
    else write_launch<__bf16, false>(a, aligned, grid, s);
  }
  return launched("kv write launch");
}

}  // namespace scoot
