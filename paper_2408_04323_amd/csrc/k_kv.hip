// Slots of a step's tokens in the block cache, and the writes to them
// (scoot_kv_assign, scoot_kv_write).
#include <hip/hip_runtime.h>

#include "kv.h"
#include "kv_vec.h"

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
// waits for another.  The sums are 32-bit ones that stay at their largest
// value, past every limit they are compared with.
//
// Few requests (and so mostly few tokens) go to workgroups of 256 threads, a
// quarter of the waves to start and to bring together (calls in a row, 256 and
// 1024 threads: 64 requests 4.7 and 5.1 us, 1000 4.6 and 5.6, 2000 5.3 and 5.6, 8192 12.0
// and 8.5; the limit is what one tile holds).  Lengths come four at a time, those
// of the next tile during the sums of this one: 8192 requests 11.8 -> 8.4 us, 20,000
// 22.8 -> 15.3.  Tiles of eight requests per thread were slower (18.5 and 37: LDS
// banks).  64 requests take 3.7 us without the host's side.  Workgroups: 100
// requests of up to 2000 new tokens 6.0 us with 128, 4.9 with 256, 4.7 with 512.
constexpr int kAssignPer = 4;     // requests per thread and tile
constexpr int kAssignFew = 1024;  // requests that one tile of 256 threads holds
constexpr int kAssignGroups = 256;

__device__ __forceinline__ int sat31(uint32_t v) { return v > 0x7fffffffu ? 0x7fffffff : (int)v; }
__device__ __forceinline__ uint32_t add_sat(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }

template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t moved(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
// Inclusive sums over a wave's lanes.
__device__ __forceinline__ uint32_t scan_wave(uint32_t v) {
  v = add_sat(v, moved<0x111, 0xf>(v));  // from 1, 2, 4, 8 lanes below within a row of 16,
  v = add_sat(v, moved<0x112, 0xf>(v));
  v = add_sat(v, moved<0x114, 0xf>(v));
  v = add_sat(v, moved<0x118, 0xf>(v));
  v = add_sat(v, moved<0x142, 0xa>(v));  // the last lane of the row below to the rows 1 and 3,
  return add_sat(v, moved<0x143, 0xc>(v));  // and that of the lower half to the upper one
}
// Exclusive sums over a workgroup's threads, and the total.
template <int THREADS>
__device__ __forceinline__ uint32_t scan_group(uint32_t v, uint32_t* sums, uint32_t& total) {
  constexpr int kWaves = THREADS / 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t x = scan_wave(v);
  if (lane == 63) sums[wave] = x;
  __syncthreads();
  const uint32_t w = scan_wave(lane < kWaves ? sums[lane] : 0);
  __syncthreads();
  total = (uint32_t)__builtin_amdgcn_readlane((int)w, kWaves - 1);
  const uint32_t before = wave ? (uint32_t)__builtin_amdgcn_readlane((int)w, wave - 1) : 0;
  const uint32_t below = moved<0x138, 0xf>(x);  // from the lane below, over the whole wave
  return add_sat(before, lane ? below : 0);
}

template <int THREADS>
__global__ __launch_bounds__(THREADS) void kv_assign_kernel(KvAssignArgs a, uint32_t per_group) {
  constexpr int kTile = THREADS * kAssignPer;
  __shared__ uint32_t sums[THREADS / 64];
  __shared__ uint32_t start[kTile];      // first token of a request, from the tile's first one
  __shared__ int ctx[kTile];             // cached tokens; -1: not admitted
  __shared__ uint32_t first[kTile];      // first of its new blocks in the free list

  const int tid = threadIdx.x;
  const uint32_t bs = 1u << a.block_shift;
  const uint32_t max_tokens = (uint32_t)a.max_tokens, num_free = (uint32_t)a.num_free;
  const uint32_t t_lo = min(blockIdx.x * per_group, max_tokens);
  const uint32_t t_hi = max_tokens - t_lo < per_group ? max_tokens : t_lo + per_group;
  uint32_t tokens = 0, blocks = 0;    // of the tiles before
  uint32_t admitted = 0, taken = 0;   // of this thread's requests
  int next_c[kAssignPer], next_n[kAssignPer];  // the thread's lengths of the next tile
  const bool quads = (((uintptr_t)a.context_len | (uintptr_t)a.new_len) & 15) == 0;
  const auto load = [&](int r0) {
    const int r = r0 + tid * kAssignPer;
    static_assert(kAssignPer == 4, "a 16-byte load");
    if (quads && r + kAssignPer <= a.num_seqs) {
      const int4 x = *(const int4*)(a.context_len + r), y = *(const int4*)(a.new_len + r);
      next_c[0] = x.x, next_c[1] = x.y, next_c[2] = x.z, next_c[3] = x.w;
      next_n[0] = y.x, next_n[1] = y.y, next_n[2] = y.z, next_n[3] = y.w;
    } else {
#pragma unroll
      for (int j = 0; j < kAssignPer; ++j) {
        next_c[j] = r + j < a.num_seqs ? a.context_len[r + j] : 0;
        next_n[j] = r + j < a.num_seqs ? a.new_len[r + j] : 0;
      }
    }
  };
  load(0);
  for (int r0 = 0, tile = 0; r0 < a.num_seqs; r0 += kTile, ++tile) {
    const bool writes = tile % (int)gridDim.x == (int)blockIdx.x;  // this workgroup stores the tile's lengths
    uint32_t c[kAssignPer], n[kAssignPer], tok = 0;
#pragma unroll
    for (int j = 0; j < kAssignPer; ++j) {
      c[j] = max(next_c[j], 0);
      n[j] = max(next_n[j], 0);
      tok = add_sat(tok, n[j]);
    }
    if (r0 + kTile < a.num_seqs) load(r0 + kTile);  // on its way during this tile's sums
    uint32_t tile_tokens, tile_blocks;
    const uint32_t t0 = scan_group<THREADS>(tok, sums, tile_tokens);  // from the tile's first token
    // The tokens alone decide which requests ask for blocks.
    uint32_t end = add_sat(tokens, t0), blk = 0, need[kAssignPer];
    bool fits[kAssignPer];
#pragma unroll
    for (int j = 0; j < kAssignPer; ++j) {
      end = add_sat(end, n[j]);
      const uint32_t len = c[j] + n[j];  // below 2^32
      const uint32_t used = (c[j] + bs - 1) >> a.block_shift, all = (len >> a.block_shift) + ((len & (bs - 1)) != 0);
      fits[j] = end <= max_tokens && all <= (uint32_t)a.max_blocks;
      need[j] = fits[j] ? all - used : 0;
      blk = add_sat(blk, need[j]);
    }
    uint32_t b0 = add_sat(blocks, scan_group<THREADS>(blk, sums, tile_blocks)), at = t0;
#pragma unroll
    for (int j = 0; j < kAssignPer; ++j) {
      const int i = tid * kAssignPer + j, r = r0 + i;
      const uint32_t upto = add_sat(b0, need[j]);
      const bool ok = r < a.num_seqs && fits[j] && (need[j] == 0 || upto <= num_free);
      start[i] = at;
      ctx[i] = ok ? (int)c[j] : -1;
      first[i] = b0;
      admitted += ok;
      if (ok && need[j] > 0) taken = upto;
      if (writes && r < a.num_seqs) {
        a.query_start[r] = sat31(add_sat(tokens, at));
        a.seq_len[r] = ok ? (int)(c[j] + n[j]) : 0;
      }
      at = add_sat(at, n[j]);
      b0 = upto;
    }
    __syncthreads();

    // Tokens of this workgroup that belong to this tile's requests.
    const uint32_t tile_end = add_sat(tokens, tile_tokens);
    const uint32_t hi = t_hi < tile_end ? t_hi : tile_end;
    for (uint32_t t = min(max(t_lo, tokens), hi) + tid; t < hi; t += THREADS) {  // hi is below 2^31
      const uint32_t my = t - tokens;
      int i = 0;  // the last request with start <= my; kTile is a power of two
#pragma unroll
      for (int step = kTile / 2; step > 0; step /= 2)
        if (start[i + step] <= my) i += step;
      int pos = -1;
      int64_t slot = -1;
      if (ctx[i] >= 0) {
        pos = ctx[i] + (int)(my - start[i]);
        const int b = pos >> a.block_shift, used = (int)((ctx[i] + bs - 1) >> a.block_shift);
        int32_t* entry = a.block_table + (int64_t)(r0 + i) * a.table_stride + b;
        const int block = b < used ? *entry : a.free_blocks[first[i] + b - used];
        if (b >= used && (pos & (bs - 1)) == 0) *entry = block;
        if (block >= 0) slot = ((int64_t)block << a.block_shift) + (pos & (bs - 1));
      }
      a.positions[t] = pos;
      a.slots[t] = slot;
    }
    tokens = tile_end;
    blocks = add_sat(blocks, tile_blocks);
    __syncthreads();
  }
  for (uint32_t t = min(max(t_lo, tokens), t_hi) + tid; t < t_hi; t += THREADS) {
    a.positions[t] = -1;
    a.slots[t] = -1;
  }
  if (blockIdx.x == 0) {
    uint32_t all;
    scan_group<THREADS>(admitted, sums, all);
    // The free blocks are taken in order: the last request that got one tells how many.
    for (int o = 1; o < 64; o <<= 1) taken = max(taken, (uint32_t)__shfl_xor((int)taken, o));
    if ((tid & 63) == 0) sums[tid >> 6] = taken;
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < THREADS / 64; ++w) taken = max(taken, sums[w]);
      a.query_start[a.num_seqs] = sat31(tokens);
      a.counts[0] = sat31(tokens);
      a.counts[1] = (int)all;
      a.counts[2] = (int)taken;
      a.counts[3] = sat31(blocks);
    }
  }
}

// --------------------------------------------------------------------- writes
//
// A workgroup takes one head of a few consecutive tokens, a thread eight
// elements of the key and of the value.  The cache's rows are the vectors'
// rows, and tokens in order mostly lie next to each other, so a wave reads
// whole lines and writes 512 bytes (8-bit) or a KiB without a gap.  Bytes
// bound this: both sides once; 45,993 tokens into 8 bits take 18.6 us (4.8 TB/s,
// a large copy's rate).
constexpr int kWriteThreads = 256;  // at most: (elements of a head / 8) x tokens

template <typename T, bool F8, bool ALIGNED>
__global__ __launch_bounds__(kWriteThreads) void kv_write_kernel(KvWriteArgs a) {
  const int64_t t = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  if (t >= a.num_tokens) return;
  const int64_t slot = a.slots[t];
  if (slot < 0 || slot >= a.num_slots) return;
  const uint32_t h = blockIdx.y, c = threadIdx.x;
  const int64_t block = slot >> a.block_shift, at = slot & ((1 << a.block_shift) - 1);
  const int64_t to = (((block * a.num_heads + h) << a.block_shift) + at) * a.head_dim + c * 8;
  typename Vec8<T>::type x[2];
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const T* p = (const T*)a.src[s] + t * a.token_stride[s] + h * a.head_stride[s] + c * 8;
    if (ALIGNED) {
      x[s] = *(const typename Vec8<T>::type*)p;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[s][j] = p[j];
    }
  }
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    if (F8) {
      float f[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = limit_f8((float)x[s][j], a.scale[s]);
      *(int2*)((uint8_t*)a.cache[s] + to) = to_f8(f);
    } else {
      *(typename Vec8<T>::type*)((T*)a.cache[s] + to) = x[s];
    }
  }
}

template <typename T, bool F8>
void write_launch(const KvWriteArgs& a, bool aligned, hipStream_t s) {
  const int chunks = a.head_dim / 8, tokens = kWriteThreads / chunks;  // head_dim <= 1024: two tokens at least
  const dim3 grid((unsigned)((a.num_tokens + tokens - 1) / tokens), (unsigned)a.num_heads), block(chunks, tokens);
  if (aligned)
    hipLaunchKernelGGL((kv_write_kernel<T, F8, true>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((kv_write_kernel<T, F8, false>), grid, block, 0, s, a);
}

}  // namespace

int launch_kv_assign(const KvAssignArgs& a, void* stream) {
  const int threads = a.num_seqs <= kAssignFew ? 256 : 1024;
  const int64_t most = (a.max_tokens + threads - 1) / threads;
  const int groups = (int)std::max<int64_t>(1, std::min<int64_t>(most, kAssignGroups));
  const uint32_t per_group = (uint32_t)((a.max_tokens + groups - 1) / groups);
  const hipStream_t s = (hipStream_t)stream;
  if (threads == 256)
    hipLaunchKernelGGL((kv_assign_kernel<256>), dim3(groups), dim3(256), 0, s, a, per_group);
  else
    hipLaunchKernelGGL((kv_assign_kernel<1024>), dim3(groups), dim3(1024), 0, s, a, per_group);
  return launched("kv assign launch");
}

int launch_kv_write(const KvWriteArgs& a, scoot_kv_type type, scoot_kv_type cache_type, void* stream) {
  const hipStream_t s = (hipStream_t)stream;
  bool aligned = true;  // every row starts on 16 bytes
  for (int i = 0; i < 2; ++i)
    aligned = aligned && ((uintptr_t)a.src[i] & 15) == 0 && ((a.token_stride[i] | a.head_stride[i]) & 7) == 0;
  const bool f8 = cache_type == SCOOT_KV_F8;
  if (type == SCOOT_KV_F16) {
    if (f8) write_launch<_Float16, true>(a, aligned, s);
    else write_launch<_Float16, false>(a, aligned, s);
  } else {
    if (f8) write_launch<__bf16, true>(a, aligned, s);
    else write_launch<__bf16, false>(a, aligned, s);
  }
  return launched("kv write launch");
}

}  // namespace scoot
