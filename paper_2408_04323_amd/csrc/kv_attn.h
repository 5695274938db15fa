// Attention over the block cache: the kernels and their launches, for one head
// dimension per translation unit (k_kv_attn_<dim>.hip).  kv_plan.h says how a
// call is split, k_kv_attn.hip takes it to its head dimension.
//
// Mathematics.  A row is one query of one head; the G query heads that share a
// key head are rows of the same tile, row = token * G + head.  With scores s_t
// = q . k_t the rows keep m, l and o over the keys seen so far: for every 32
// keys, w_t = 2^(c s_t - m), l += sum w_t, o += sum w_t v_t.  m stays near the
// row's largest score: only when a lane's weights of these keys add up to more
// than 2^14 it moves up, to 6 below their largest, and l and o are multiplied by
// 2^(old m - m).  So no weight overflows, one at least is 64 or more, and most
// keys take no maximum and leave o alone.  Parts of the keys that were handled
// by different waves or workgroups are joined by the same factors.
//
// Rounding: scores, m, l and o are in float; a weight is rounded once, to the 16
// bits that the matrix instructions take, and l adds the rounded weights, so that
// a row of equal values gives that value.  Values whose mean is not small against
// their spread hide this rounding; with values of zero mean the result's error,
// most of which is its own rounding to 16 bits, is 1.3 to 1.4 times that of
// weights in float (bfloat16 0.0023 of the result for 0.0017, half precision 0.00029
// for 0.00021), and 1.01 times with an 8-bit cache, whose weights are in half
// precision.  Weights in two 16-bit parts would be exact enough and double the
// second product.
//
// Matrix instructions (32 x 32 x 16).  S^T = K Q^T with the keys as rows and the
// queries as columns, then O^T += V^T W^T: a lane's sixteen scores belong to
// one query, so maxima and sums are lane-local up to one exchange between the
// wave's halves, and, with the rows of K assigned as in key_of_row(), the
// lane's weights are, rounded to 16 bits, already the second product's operand.
// Q stays in registers for the whole tile.  V^T is read out of row-major LDS
// by the transposing reads (16 lanes exchange a 4 x 16 or 8 x 16 tile).
//
// Keys and values go from memory straight into LDS, 1 KiB per instruction,
// their 16-byte pieces permuted on the way so that both kinds of reads spread
// over the banks.
//
// Registers decide the waves per SIMD: three for tiles of 64 dimensions, two for
// 128, one for 192 and 256, where o and q take 144 and 192 of a lane's 512.  A
// wave alone keeps both units busy by itself: the weights of 32 keys are made
// between the matrix instructions of the next products, and a strip's loads go
// between those of the first scores (in a row they hold the wave up: 192 427 ->
// 396 us).  Late chunks over 30,000 keys, heads of 64, 128, 192, 256: 0.95, 1.14,
// 0.90, 0.88 PFLOP/s (192 and 256 with two waves and half of the registers each,
// o shared: 0.58 and 0.44).
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "kv.h"
#include "kv_plan.h"

namespace scoot {
namespace kvattn {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef int i4 __attribute__((ext_vector_type(4)));
typedef int i2 __attribute__((ext_vector_type(2)));
typedef short s4 __attribute__((ext_vector_type(4)));

#define SCOOT_LDS __attribute__((address_space(3)))
#define SCOOT_CONST __attribute__((address_space(4)))

constexpr int kThreads = 64 * kWaves;
constexpr float kNoScore = -3.40282347e38f;  // m before any key was seen; finite, so that m - m is 0, and below no finite score
constexpr int kReadsAhead = 4;               // operands of the matrix instructions on their way out of LDS
constexpr float kMost = 16384.0f;            // m moves once a lane's weights of 32 keys add up to more,
constexpr float kBelow = 6.0f;               // to this much below their largest: half precision holds 64 as well as 1, and
                                             // weights down to 2^-30 of the largest, which counts where many keys are small

constexpr float kLimit = 14.0f;              // of a weight's exponent where it moved: no other weight is above kMost

constexpr int gcd256(int x) { return x % 256 == 0 ? 256 : x % 128 == 0 ? 128 : 64; }

// Sizes of a cache row in LDS.
template <typename T_, bool F8_, int D_>
struct Shape {
  typedef T_ T;
  static constexpr bool F8 = F8_;
  static constexpr int D = D_;
  static constexpr int EB = F8 ? 1 : 2;
  static constexpr int RB = D * EB;                 // bytes of a row
  static constexpr int PC = RB / 16;                // 16-byte pieces of a row
  static constexpr int g = 256 / gcd256(RB);        // rows this far apart start on the same bank
  static constexpr int NJ = RB / 64;                // loads of 1 KiB for 16 rows
  static constexpr int ST = kStripKeys;             // keys per strip of a shared tile
  static constexpr int kStrip = strip_bytes(RB);    // of K and V
  // The second product runs in the cache's 16-bit type; 8-bit values are exact in half precision, which rounds the
  // weights eight times finer than bfloat16.
  typedef typename std::conditional<F8, _Float16, T>::type W;
};

// How the pieces of a row are permuted on the way into LDS.  A read instruction
// takes one piece of 16 keys (K) or U pieces of 8 or 16 keys (V) per 256 bytes
// that LDS delivers in a cycle; these keys, counted by kid() and vid(), must
// hit different banks.  Keys g apart start on the same bank, so there the
// piece (the unit of U pieces) is exchanged by XOR with the count.
template <typename S>
struct Tile32Order {  // 32 x 32 x 16 products
  static constexpr int KM = 16 / S::g;
  static constexpr int U = 2 * S::EB, VM = (8 / S::EB) / S::g;
  static __device__ __forceinline__ constexpr int k(int key) { return key / S::g % KM; }
  static __device__ __forceinline__ constexpr int v(int key) { return key / S::g % VM; }
};
template <typename S>
struct Tile16Order {  // 16 x 16 x 32 products
  static constexpr int KM = 16 / S::g;
  static constexpr int U = S::EB, VM = (16 / S::EB) / S::g;
  static constexpr uint32_t kNext = 128 / S::g;  // what the order of the next 16 keys differs by, in bytes
  static __device__ __forceinline__ constexpr int k(int key) { return ((key & 3) | (key >> 1 & 12)) / S::g % KM; }
  static __device__ __forceinline__ constexpr int v(int key) {
    return (S::F8 ? key & 15 : (key & 3) | (key >> 1 & 4)) / S::g % VM;
  }
};

template <typename T>
struct Vec {
  typedef h8 v8;
};
template <>
struct Vec<__bf16> {
  typedef b8 v8;
};

__device__ __forceinline__ f16v mfma(h8 a, h8 b, f16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f16v mfma(b8 a, b8 b, f16v c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f4 mfma(h8 a, h8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f4 mfma(b8 a, b8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// The key, of a strip's 32, that row r of the first product's left operand
// holds: rows 4h .. 4h + 3 and 8 + 4h .. (the scores of the wave's half h) are
// keys 8h .. 8h + 7.
__device__ __forceinline__ int key_of_row(int r) { return (r & 19) | ((r & 4) << 1) | ((r & 8) >> 1); }

template <int N>
__device__ __forceinline__ void wait_vm() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// All vector loads, in a form that the compiler takes note of: it then waits for none of them later, in a loop where
// that would be a wait for the loads to LDS, too.
__device__ __forceinline__ void settle() { __builtin_amdgcn_s_waitcnt(0x0f70); }
// A value that the compiler does not take apart: an address of LDS, to which constants are added as the
// instruction's offset.
__device__ __forceinline__ uint32_t pinned(uint32_t v) {
  asm("" : "+v"(v));
  return v;
}
// A value as of here: what is made of it is not made ahead of a loop and kept.
__device__ __forceinline__ uint32_t here(uint32_t v) {
  asm volatile("" : "+v"(v));
  return v;
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// 64 lanes x 16 bytes from base + off to LDS at `to`, lane after lane; counted
// by vmcnt.  The compiler does not know of the write: whoever reads it waits
// first.  Written out because the compiler, for the builtin, waits for all
// loads in flight before any read of LDS.  m0 is named as changed, so that the
// compiler's own uses of it stay in order with these; it warns that it does
// not keep the register's value, and nothing here needs that.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_lds(uint32_t to, uint64_t base, uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void load_lds(uint32_t to, uint64_t addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(addr) : "memory", "m0");
}
#pragma clang diagnostic pop

// What a workgroup works on: rows of a request from row0 on (a tile's, or 16), one key
// head, keys [k0, k1) of the tile's, as split `split` of `splits`.
struct Item {
  int64_t q0;       // token of the request's row 0
  int64_t pos0;     // its position
  int rows;         // rows of the request
  int row0;         // first row of the tile
  int len;          // cached tokens that have table entries
  int k0, k1;       // keys of this workgroup; k0 is a multiple of 32
  int splits;       // parts that the tile's keys are in
  int split;
  int seq;
  bool shared;      // the waves share the keys (more than kFew rows), else each wave takes strips of its own
};

__device__ __forceinline__ int64_t clamp64(int64_t v, int64_t lo, int64_t hi) { return v < lo ? lo : v > hi ? hi : v; }

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Finds the item: false if there is none.  All values are the same in every lane.
//
// Tiles need no list: request i, whose tokens start at s_i, owns the numbers
// from floor(s_i G / R) + i on (R rows per tile), which are enough for its
// ceil(n_i G / R) tiles whatever n_i is; the request of a number is searched for 64-fold.
__device__ __forceinline__ bool find_item(const KvAttnArgs& a, const Plan& p, int64_t index, int split, Item& it) {
  const int G = a.num_heads / a.num_kv_heads;
  const SCOOT_CONST int32_t* qs = (const SCOOT_CONST int32_t*)a.query_start;
  int seq;
  int64_t first = 0;
  if (p.tile_rows) {
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = a.num_seqs;
    bool any = true;
    do {
      const int step = (hi - lo + 63) / 64;
      const int64_t i = lo + (int64_t)lane * step;
      bool below = false;
      if (i < hi) below = clamp64(a.query_start[i], 0, a.num_tokens) * G / p.tile_rows + i <= index;
      const int n = __popcll(__builtin_amdgcn_ballot_w64(below));
      if (n == 0) {
        any = false;
        break;
      }
      lo += (n - 1) * step;
      if (hi > lo + step) hi = lo + step;
    } while (hi - lo > 1);
    if (!any) return false;
    seq = uniform(lo);
    first = clamp64(qs[seq], 0, a.num_tokens) * G / p.tile_rows + seq;
  } else {
    seq = uniform((int)index);
  }
  const int64_t s = qs[seq], e = qs[seq + 1];
  const int64_t t0 = clamp64(s, 0, a.num_tokens), t1 = clamp64(e, 0, a.num_tokens);
  if (t1 <= t0) return false;
  const int64_t rows = (t1 - t0) * G;
  const int64_t len = ((const SCOOT_CONST int32_t*)a.seq_len)[seq];
  it.q0 = t0;
  it.pos0 = len - (e - t0);
  it.rows = rows > 0x7fffffff ? 0x7fffffff : (int)rows;
  it.seq = seq;
  it.len = (int)clamp64(len, 0, (int64_t)a.max_blocks << a.block_shift);
  it.shared = p.tile_rows && rows > kFew;
  int last_row = it.rows - 1;
  int splits = p.splits;
  if (it.shared) {
    const int tiles = (int)(((int64_t)it.rows + p.tile_rows - 1) / p.tile_rows);
    const int64_t t = index - first;
    if (t < 0 || t >= tiles) return false;  // negative: query_start does not ascend
    it.row0 = (tiles - 1 - (int)t) * p.tile_rows;  // the tiles that see most come first
    if (last_row - it.row0 >= p.tile_rows) last_row = it.row0 + p.tile_rows - 1;
  } else {
    if (p.tile_rows && index != first) return false;
    it.row0 = 0;
    if (it.rows > kFew) splits = 1;  // more rows than the caller announced: one workgroup, tile after tile
  }
  // The tile's keys, and this split's part of them.
  const int64_t top = it.pos0 + last_row / G;
  const int end = (int)clamp64(top + 1, 0, it.len);
  int begin = 0;
  if (a.window > 0) begin = (int)clamp64(it.pos0 + it.row0 / G - a.window + 1, 0, end) & ~31;
  const int parts = end > begin ? (int)(((int64_t)end - begin + p.part - 1) / p.part) : 1;
  it.splits = parts < splits ? parts : splits;
  it.split = split;
  if (split >= it.splits) return false;
  it.k0 = begin + split * p.part;
  it.k1 = split == it.splits - 1 ? end : it.k0 + p.part;
  return true;
}

// Blocks of the cache, as scalars.
template <typename S>
struct Cache {
  const SCOOT_CONST int32_t* table;
  const int32_t* entries;  // the same, for vector loads
  uint64_t k, v;
  uint32_t block_bytes;  // of all heads; at most 1024 heads of 256 keys of 512 bytes
  uint32_t num_blocks;
  int shift, last;       // last entry of the row

  __device__ __forceinline__ void setup(const KvAttnArgs& a, int seq, int head) {
    entries = a.block_table + (int64_t)seq * a.table_stride;
    table = (const SCOOT_CONST int32_t*)entries;
    const uint32_t head_bytes = (uint32_t)S::RB << a.block_shift;
    block_bytes = head_bytes * (uint32_t)a.num_kv_heads;
    k = (uint64_t)a.k_cache + (uint64_t)head * head_bytes;
    v = (uint64_t)a.v_cache + (uint64_t)head * head_bytes;
    num_blocks = (uint32_t)a.num_blocks;
    shift = a.block_shift;
    last = a.max_blocks - 1;
  }
  // The entry of eight keys from `key` on (inside one block), for at().
  __device__ __forceinline__ uint32_t entry(int key) const {
    const int e = key >> shift;
    return (uint32_t)table[e < last ? e : last];
  }
  // Byte offset of these keys.  An entry that names no block reads block 0, and the mask drops it.
  __device__ __forceinline__ uint64_t at(int key, uint32_t e) const {
    return (uint64_t)(e < num_blocks ? e : 0) * block_bytes + (uint32_t)(key & ((1 << shift) - 1)) * S::RB;
  }
  // Which of the four groups of eight keys from `key` on have no block.
  __device__ __forceinline__ int holes(int key) const {
    int h = 0;
    for (int j = 0; j < 4; ++j) {
      const int e = (key + 8 * j) >> shift;
      if (e > last || (uint32_t)table[e] >= num_blocks) h |= 1 << j;
    }
    return h;
  }
};

// Addresses of a wave's next 64 strips, one strip per lane: N groups of eight
// keys each, `stride` keys from strip to strip.  (By scalars, a strip would
// cost some forty instructions, and a scalar load is waited for together with
// the reads of LDS.)
template <typename S, int N>
struct Ahead {
  uint32_t lo[N], hi[N];
  uint64_t from;  // keys or values
  int key0, stride, strips, base, end;
  bool holes;     // some group below key `end` of the 64 strips has no block

  __device__ __forceinline__ void fill(const Cache<S>& c, int strip) {
    base = strip;
    const int lane = threadIdx.x & 63;
    const int key = key0 + (strip + lane < strips ? strip + lane : strip) * stride;
    uint32_t e[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int i = (key + 8 * j) >> c.shift;
      e[j] = (uint32_t)c.entries[i < c.last ? i : c.last];
    }
    settle();
    bool hole = false;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      hole |= (key + 8 * j < end) & (e[j] >= c.num_blocks);
      const uint64_t at = from + c.at(key + 8 * j, e[j]);
      lo[j] = (uint32_t)at;
      hi[j] = (uint32_t)(at >> 32);
    }
    holes = __builtin_amdgcn_ballot_w64(hole) != 0;
  }
  __device__ __forceinline__ void start(const Cache<S>& c, uint64_t cache, int first, int keys, int n, int last) {
    from = cache;
    key0 = first;
    stride = keys;
    strips = n;
    end = last;
    holes = false;
    if (n > 0) fill(c, 0);
  }
  // The groups of a strip, which follows the last one asked for.
  __device__ __forceinline__ void get(const Cache<S>& c, int strip, uint64_t (&b)[N]) {
    if (strip - base == 64) fill(c, strip);
#pragma unroll
    for (int j = 0; j < N; ++j)
      b[j] = (uint32_t)__builtin_amdgcn_readlane((int)lo[j], strip - base) |
             (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)hi[j], strip - base) << 32;
  }
};

// Whether `x` holds in any of the workgroup's waves; `flag`: a word of LDS for each.
template <int W>
__device__ __forceinline__ bool any_wave(bool x, int* flag) {
  __syncthreads();
  if ((threadIdx.x & 63) == 0) flag[threadIdx.x >> 6] = x;
  __syncthreads();
  int any = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) any |= flag[w];
  return uniform(any) != 0;
}

// Whether any of the item's keys lies in an entry that names no block.
template <int W>
__device__ __forceinline__ bool any_holes(const KvAttnArgs& a, const Item& it, int* flag) {
  const int32_t* t = a.block_table + (int64_t)it.seq * a.table_stride;
  bool h = false;
  for (int64_t e = (it.k0 >> a.block_shift) + threadIdx.x; (e << a.block_shift) < it.k1; e += 64 * W)
    h = h || (uint32_t)t[e] >= (uint32_t)a.num_blocks;
  return any_wave<W>(__builtin_amdgcn_ballot_w64(h) != 0, flag);
}

// Eight 8-bit floats as 16-bit ones (exact).
template <typename R>
__device__ __forceinline__ typename Vec<R>::v8 widen(int a, int b) {
  typename Vec<R>::v8 r;
  if constexpr (std::is_same<R, _Float16>::value) {
    const h2 x[4] = {__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, false), __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, true),
                     __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, false), __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, true)};
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = x[i / 2][i % 2];
  } else {
    const b2 x[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true),
                     __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true)};
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = x[i / 2][i % 2];
  }
  return r;
}

// The sum l with the weights i and i + 1, as rounded, like the product takes them.
template <typename W>
__device__ __forceinline__ float add_pair(const typename Vec<W>::v8& r, int i, float l) {
  if constexpr (std::is_same<W, _Float16>::value) {
    const h2 p = {r[i], r[i + 1]}, one = {(_Float16)1.0f, (_Float16)1.0f};
    return __builtin_amdgcn_fdot2(p, one, l, false);
  } else {
    const b2 p = {r[i], r[i + 1]}, one = {(__bf16)1.0f, (__bf16)1.0f};
    return __builtin_amdgcn_fdot2_f32_bf16(p, one, l, false);
  }
}

// m for a largest score of s.  The exponents scale s - m are exact, but m is as far off as a float is: from 2^27 on by 16
// and more, so that the weight of the largest score would overflow or vanish.  There m goes below by so much that this
// weight is always above kMost and then limited; scores that are limited with it are within the error of a float sum.
__device__ __forceinline__ float below(float s, float scale) {
  const float x = s * scale, e = __builtin_fabsf(x);
  return x - (e >= 0x1p27f && e < INFINITY ? e * 0x1p-22f : 0.0f) - kBelow;
}
// Not above the limit; NaN stays.
__device__ __forceinline__ float limited(float x, float limit) { return __builtin_elementwise_minimum(x, limit); }

// Eight weights 2^(scale s - m), rounded, and their sum added to l.
template <typename W, bool LIMITED, typename F>
__device__ __forceinline__ typename Vec<W>::v8 eight_weights(F score, float scale, float m, float limit, float& l) {
  typename Vec<W>::v8 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = fmaf(score(i), scale, -m);
    r[i] = (W)__builtin_amdgcn_exp2f(LIMITED ? limited(x, limit) : x);
  }
#pragma unroll
  for (int i = 0; i < 8; i += 2) l = add_pair<W>(r, i, l);
  return r;
}

// Where some rows do not see some keys, 0 * inf must not arise.
//
// Eight keys' values without those past the first `seen`, which no row sees.
template <typename V>
__device__ __forceinline__ V only_seen(V v, int seen) {
  union {
    V v;
    uint32_t w[4];
  } x;
  x.v = v;
#pragma unroll
  for (int i = 0; i < 4; ++i) x.w[i] &= (seen > 2 * i ? 0xffffu : 0u) | (seen > 2 * i + 1 ? 0xffff0000u : 0u);
  return x.v;
}
// ... and without what is not finite.  A key that only some rows see and whose
// value is not finite spoils the others' sums; that shows in the end, and the
// tile is done again with these values left out and added afterwards.
template <typename W>
__device__ __forceinline__ typename Vec<W>::v8 only_finite(typename Vec<W>::v8 v) {
  constexpr uint32_t kExp = (std::is_same<W, _Float16>::value ? 0x7c00u : 0x7f80u) * 0x10001u;
  union {
    typename Vec<W>::v8 v;
    uint32_t w[4];
  } x;
  x.v = v;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    // A full exponent carries into the sign's place; from there all over its half.
    const uint32_t e = ((x.w[i] & kExp) + (0x80008000u - kExp)) & 0x80008000u;
    x.w[i] &= ~(e | (e - (e >> 15)));
  }
  return x.v;
}

// Memory offsets of a lane's loads of 16 keys: its pieces, as they lie in LDS.
// Where a load takes a power of two of keys, the numbers of a load's keys and
// of the keys in it share no bit, and every offset is the first one with some
// bits changed: heads of 256 have no registers for them all (256 decoding
// requests 140 -> 131 us, late chunks 1160 -> 585; heads of 64 in 8 bits 185 -> 188).
template <typename S, typename Order, bool FEW_REGS>
struct Offsets {
  static constexpr bool kLinear = FEW_REGS && 64 % S::PC == 0;
  static constexpr int N = kLinear ? 1 : S::NJ;
  uint32_t k[N], v[N];

  static __device__ __forceinline__ constexpr uint32_t k_of(int key, int p) { return (key & 7) * S::RB + (p ^ Order::k(key)) * 16; }
  static __device__ __forceinline__ constexpr uint32_t v_of(int key, int p) {
    return (key & 7) * S::RB + ((p / Order::U ^ Order::v(key)) * Order::U + p % Order::U) * 16;
  }
  __device__ __forceinline__ void setup() {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int at = 64 * j + (int)(threadIdx.x & 63), key = at / S::PC, p = at % S::PC;
      k[j] = k_of(key, p);
      v[j] = v_of(key, p);
    }
  }
  __device__ __forceinline__ uint32_t of_k(int j) const {
    if constexpr (kLinear) return here(k[0]) ^ k_of(64 * j / S::PC, 0);
    else return k[j];
  }
  __device__ __forceinline__ uint32_t of_v(int j) const {
    if constexpr (kLinear) return here(v[0]) ^ v_of(64 * j / S::PC, 0);
    else return v[j];
  }
};

// The j-th load of 16 keys (two groups of eight, each inside a block) to LDS; off(j): its offset.
template <typename S, uint32_t X = 0, typename F>
__device__ __forceinline__ void load16(F off, uint32_t to, uint64_t b0, uint64_t b1, int j) {
  constexpr int kHalf = 8 * S::PC;  // pieces of eight keys
  if (64 * j + 63 < kHalf)
    load_lds(to + 1024 * j, b0, off(j) ^ X);
  else if (64 * j >= kHalf)
    load_lds(to + 1024 * j, b1, off(j) ^ X);
  else
    load_lds(to + 1024 * j, (64 * j + (int)(threadIdx.x & 63) < kHalf ? b0 : b1) + (off(j) ^ X));
}
template <typename S, uint32_t X = 0, typename F>
__device__ __forceinline__ void load16(F off, uint32_t to, uint64_t b0, uint64_t b1) {
#pragma unroll
  for (int j = 0; j < S::NJ; ++j) load16<S, X>(off, to, b0, b1, j);
}

// What `count` rows from row0 on see: a lane's row (row0 + r) keys lo < k <=
// hi, and over the rows.  Positions grow with the rows.
struct Sight {
  int tok, g;  // token and head of the lane's row
  int hi, lo, hi_min, hi_max, lo_max;

  __device__ __forceinline__ void start(const KvAttnArgs& a, const Item& it, int row0, int r, int count) {
    const int G = a.num_heads / a.num_kv_heads;
    int row = row0 + r;  // rows past the request's last one repeat it; nothing of them is stored
    row = row < it.rows ? row : it.rows - 1;
    tok = row / G;
    g = row - tok * G;
    const int first = uniform((row0 < it.rows ? row0 : it.rows - 1) / G);
    const int last = uniform((row0 + count < it.rows ? row0 + count - 1 : it.rows - 1) / G);
    hi = upto(it, tok);
    lo = after(a, it, tok);
    hi_min = upto(it, first);
    hi_max = upto(it, last);
    lo_max = after(a, it, last);
  }
  static __device__ __forceinline__ int upto(const Item& it, int tok) { return (int)clamp64(it.pos0 + tok, -1, it.len - 1); }
  static __device__ __forceinline__ int after(const KvAttnArgs& a, const Item& it, int tok) {
    return a.window > 0 ? (int)clamp64(it.pos0 + tok - a.window, -1, 0x7fffffff) : -1;
  }
  // Strips of `keys` keys from k0 on that every row sees whole: [u0, u1).
  __device__ __forceinline__ void whole(const Item& it, int strips, int keys, bool holes, int& u0, int& u1) const {
    u0 = u1 = strips;
    if (holes) return;
    u1 = hi_min + 1 > it.k0 ? min((hi_min + 1 - it.k0) / keys, strips) : 0;
    u0 = lo_max + 1 > it.k0 ? (lo_max + 1 - it.k0 + keys - 1) / keys : 0;
  }
};

// Whether the lane's row sees any of the item's keys, in a block that there is.  All lanes take part: 64 entries of the
// table at a time.
__device__ __forceinline__ bool sees_any(const KvAttnArgs& a, const Item& it, const Sight& see) {
  const int32_t* t = a.block_table + (int64_t)it.seq * a.table_stride;
  const int first = max(see.lo + 1, it.k0), last = min(see.hi, it.k1 - 1);
  const int to = min(see.hi_max, it.k1 - 1) >> a.block_shift;
  bool any = false;
#pragma unroll 1
  for (int e0 = it.k0 >> a.block_shift; e0 <= to; e0 += 64) {
    const int e = e0 + (int)(threadIdx.x & 63);
    const uint64_t real = __builtin_amdgcn_ballot_w64(e <= to && (uint32_t)t[e < to ? e : to] < (uint32_t)a.num_blocks);
    const int i = max((first >> a.block_shift) - e0, 0), j = min((last >> a.block_shift) - e0, 63);
    if (first <= last && i <= j) any |= real >> i << (63 - j + i) != 0;
  }
  return any;
}
// Rows whose weights add up to 0 either see nothing, which gives 0, or have scores of -inf alone, whose softmax is no
// number.  Their part of the keys tells by m: kNoScore, or -inf for the latter, which counts if all parts' weights are 0.
__device__ __forceinline__ float told(const KvAttnArgs& a, const Item& it, const Sight& see, float m, float sum) {
  const bool none = sum == 0.0f && min(see.hi, it.k1 - 1) >= max(see.lo + 1, it.k0);
  if (__builtin_expect(__builtin_amdgcn_ballot_w64(none) == 0, 1)) return m;
  return sees_any(a, it, see) && none ? -INFINITY : m;
}
// What the sums of values times weights are multiplied by.
__device__ __forceinline__ float inverse(float v_scale, float sum, bool lost) {
  return sum == 0.0f ? (lost ? __builtin_nanf("") : 0.0f) : v_scale / sum;
}

// Value d of the key's row as it is stored.
template <typename S>
__device__ __forceinline__ float stored(uint64_t row, int d) {
  if constexpr (S::F8) return __builtin_amdgcn_cvt_f32_fp8((int)((const uint8_t*)row)[d], 0);
  else return (float)((const typename S::W*)row)[d];
}

// ------------------------------------------------------------- shared tiles
//
// More than 16 rows: the four waves take 32 rows each and share strips of 64 keys
// through LDS buffers, R of them, the loads R - 1 strips ahead.  The clock falls
// to 1.6 - 1.9 GHz under these products (a library's large product: 1.8), and the matrix
// units are busy 50% of the time with heads of 128 (that product: 68%).
template <typename S>
struct Tile32 {
  typedef typename S::T T;
  typedef typename S::W W;
  typedef typename Vec<T>::v8 T8;
  typedef typename Vec<W>::v8 W8;
  typedef Tile32Order<S> Order;
  static constexpr int KS = S::D / 16;  // steps of the first product
  static constexpr int DT = S::D / 32;  // tiles of O^T
  static constexpr int VN = Order::VM < DT ? Order::VM : DT;

  int lane, half;
  Sight see;
  T8 q[KS];
  f16v o[DT];
  float m, l;
  // LDS offsets of this lane's reads; with few registers the first ones, of which the others differ by some bits.
  static constexpr bool kFewRegs = S::D == 256;
  static constexpr int KN = kFewRegs ? 1 : Order::KM / 2, VM = kFewRegs ? 1 : VN;
  int koff[KN], voff[VM];
  Offsets<S, Order, kFewRegs> dma;

  __device__ __forceinline__ void setup() {
    lane = threadIdx.x & 63;
    half = lane >> 5;
    const int key = key_of_row(lane & 31);
#pragma unroll
    for (int n = 0; n < KN; ++n) koff[n] = key * S::RB + ((2 * n + half) ^ Order::k(key)) * 16;
    const int n16 = lane & 15, dhalf = (lane >> 4) & 1;
    const int row = 8 * half + (S::F8 ? n16 >> 1 : n16 >> 2);
    const int in = S::F8 ? dhalf * 16 + (n16 & 1) * 8 : dhalf * 32 + (n16 & 3) * 8;
#pragma unroll
    for (int n = 0; n < VM; ++n) voff[n] = row * S::RB + (n ^ Order::v(row)) * (16 * Order::U) + in;
    dma.setup();
  }

  __device__ __forceinline__ void start(const KvAttnArgs& a, const Item& it, int row0, int head) {
    see.start(a, it, row0, lane & 31, kRows);
    const int G = a.num_heads / a.num_kv_heads;
    const T* p = (const T*)a.q + (it.q0 + see.tok) * a.q_token_stride + (int64_t)(head * G + see.g) * a.q_head_stride;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int d = S::F8 ? (2 * (s / 2) + half) * 16 + 8 * (s & 1) : (2 * s + half) * 8;
      q[s] = *(const T8*)(p + d);
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
    m = kNoScore;
    l = 0.0f;
  }

  // What a strip's products read out of LDS.  The reads go ahead of the
  // products that use them, and every product is followed by some other work,
  // `between`, that runs while the matrix unit is busy: left alone, the compiler
  // waits for each read and keeps products and weights apart.
  static constexpr int KR = S::F8 ? KS / 2 : KS;  // reads of K for 32 keys
  static constexpr int kAheadK = KR < kReadsAhead ? KR : kReadsAhead;
  static constexpr int KP = KS;      // products per 32 keys: of the scores,
  static constexpr int VP = 2 * DT;  // and of the values
  typedef typename std::conditional<S::F8, i4, T8>::type Piece;
  struct Keys {
    uint32_t at[Order::KM / 2];
    Piece k[kAheadK];
  };
  __device__ __forceinline__ Piece key(const Keys& x, int i) const {
    constexpr int N = Order::KM / 2;
    const int n = i / KR, u = i % KR;
    return *(const SCOOT_LDS Piece*)(x.at[u % N] + n * 32 * S::RB + (u / N) * (16 * Order::KM));
  }
  __device__ __forceinline__ Keys keys(uint32_t lds) const {
    Keys x;
#pragma unroll
    for (int n = 0; n < Order::KM / 2; ++n) x.at[n] = pinned(lds + (kFewRegs ? here(koff[0]) ^ n * 32 : koff[n % KN]));
#pragma unroll
    for (int i = 0; i < kAheadK; ++i) x.k[i] = key(x, i);
    __builtin_amdgcn_sched_barrier(0);
    return x;
  }
  // S^T of the strip's keys 32 n .. 32 n + 31.
  template <int n, typename F>
  __device__ __forceinline__ void scores(Keys& x, f16v& s, F between) const {
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.0f;
#pragma unroll
    for (int u = 0; u < KR; ++u) {
      const int i = n * KR + u;
      const Piece k = x.k[i % kAheadK];
      if constexpr (S::F8) {
        s = mfma(widen<T>(k[0], k[1]), q[2 * u], s);
        between(2 * u);
        __builtin_amdgcn_sched_barrier(0);
        s = mfma(widen<T>(k[2], k[3]), q[2 * u + 1], s);
      } else {
        s = mfma(k, q[u], s);
      }
      if (i + kAheadK < 2 * KR) x.k[i % kAheadK] = key(x, i + kAheadK);
      between(S::F8 ? 2 * u + 1 : u);
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  struct Lds {
    uint32_t at[VN];
  };
  __device__ __forceinline__ Lds values_at(uint32_t lds) const {
    Lds r;
#pragma unroll
    for (int n = 0; n < VN; ++n) r.at[n] = pinned(lds + (kFewRegs ? here(voff[0]) ^ n * 16 * Order::U : voff[n % VM]));
    return r;
  }
  // V^T: lane's element d = 32 dt + lane % 32 of the keys 16 ks + 8 half .. + 7.
  __device__ __forceinline__ W8 values(const Lds& v, int ks, int dt) const {
    const uint32_t at = v.at[dt % VN] + (dt / VN) * (VN * 16 * Order::U) + ks * 16 * S::RB;
    if constexpr (S::F8) {
      const i2 v = __builtin_amdgcn_ds_read_tr8_b64_v2i32((SCOOT_LDS i2*)at);
      return widen<_Float16>(v[0], v[1]);
    } else {
      union {
        s4 h[2];
        W8 v;
      } r;
      r.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SCOOT_LDS s4*)at);
      r.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SCOOT_LDS s4*)(at + 4 * S::RB));
      return r.v;
    }
  }

  // -inf for what a row does not see; `holes`: bits of the strip's groups of eight keys without a block.
  __device__ __forceinline__ void mask(f16v& s, int key0, int holes) const {
    const int first = key0 + 8 * half;
    const int h = see.hi - first, l = see.lo - first;  // no underflow: hi, lo >= -1 and keys are below 2^31
    holes >>= half;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int k = 16 * (i / 8) + (i & 7);
      // bit operations and a select: a branch that differs between lanes here would cost copies of o in the whole loop
      const bool hidden = (k > h) | (k <= l) | ((holes & (i < 8 ? 1 : 4)) != 0);
      s[i] = hidden ? -INFINITY : s[i];
    }
  }

  // Weights of 32 keys.  No maximum is taken as long as the weights stay
  // moderate, which their sum tells; whether a row's m moves depends on that
  // row alone.  weigh() is the i-th of n parts of the work, moderate() its end.
  struct Weights {
    W8 w[2];
    float add;
  };
  template <bool LIMITED = false>
  __device__ __forceinline__ void weigh(const f16v& s, float scale, Weights& x, int i, int n, float limit = 0.0f) const {
    const int from = 2 * (8 * i / n), to = 2 * (8 * (i + 1) / n);
    if (i == 0) x.add = 0.0f;
#pragma unroll
    for (int j = from; j < to; ++j) {
      const float e = fmaf(s[j], scale, -m);
      x.w[j / 8][j % 8] = (W)__builtin_amdgcn_exp2f(LIMITED ? limited(e, limit) : e);
    }
#pragma unroll
    for (int j = from; j < to; j += 2) x.add = add_pair<W>(x.w[j / 8], j % 8, x.add);
  }
  __device__ __forceinline__ void moderate(const f16v& s, float scale, Weights& w) {
    if (__builtin_amdgcn_ballot_w64(!(w.add <= kMost))) {
      float x = s[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) x = fmaxf(x, s[i]);
      auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
      x = below(fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])), scale);
      const uint32_t over = !(w.add <= kMost);
      sw = __builtin_amdgcn_permlane32_swap(over, over, false, false);
      const bool moves = (sw[0] | sw[1]) != 0;
      const float up = moves && x > m ? x : m, f = __builtin_amdgcn_exp2f(m - up);
      m = up;
      l *= f;
#pragma unroll
      for (int d = 0; d < DT; ++d) {
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] *= f;
        __builtin_amdgcn_sched_barrier(0);  // not all of o at once: large ones rest outside the vector units' registers
      }
      weigh<true>(s, scale, w, 0, 1, moves ? kLimit : INFINITY);
    }
    l += w.add;
  }

  template <int n, typename F>
  __device__ __forceinline__ void product(const Lds& lds, const Weights& w, W8 (&v)[kReadsAhead], F between) {
#pragma unroll
    for (int j = 0; j < VP; ++j) {
      const int i = n * VP + j, next = i + kReadsAhead;
      o[j % DT] = mfma(v[i % kReadsAhead], w.w[j / DT], o[j % DT]);
      if (next < 2 * VP) v[i % kReadsAhead] = values(lds, next / DT, next % DT);
      between(j);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // A strip that every row sees whole.  Of the two halves of 64 keys the first one's weights are made between the
  // second one's scores, and the second one's between the first one's values; load(i), i < KP, the i-th part of a
  // strip's loads, goes between the first one's scores.
  template <typename L>
  __device__ __forceinline__ void strip(uint32_t kat, uint32_t vat, float scale, L load) {
    const auto nothing = [](int) {};
    f16v s[2];
    Weights p[2];
    W8 v[kReadsAhead];
    Keys x = keys(kat);
    scores<0>(x, s[0], load);
    const Lds lds = values_at(vat);
    scores<1>(x, s[1], [&](int i) { weigh(s[0], scale, p[0], i, KP); });
#pragma unroll
    for (int i = 0; i < kReadsAhead; ++i) v[i] = values(lds, i / DT, i % DT);
    moderate(s[0], scale, p[0]);
    __builtin_amdgcn_sched_barrier(0);
    product<0>(lds, p[0], v, [&](int i) { weigh(s[1], scale, p[1], i, VP); });
    moderate(s[1], scale, p[1]);
    product<1>(lds, p[1], v, nothing);
  }
  // Any other strip, from key `key0` on; holes(key): as for mask().  In this form for all strips, four prompts of 4096
  // tokens took 422 us instead of 413: the masks' registers are those of the loop above, too.
  template <bool FINITE, typename H>
  __device__ __forceinline__ void strip_seen(uint32_t kat, uint32_t vat, float scale, int key0, H holes) {
    const auto nothing = [](int) {};
    f16v s[2];
    Keys x = keys(kat);
    const bool two = key0 + 32 <= see.hi_max;  // some row sees the second half's keys
    scores<0>(x, s[0], nothing);
    if (two) scores<1>(x, s[1], nothing);
    const Lds lds = values_at(vat);
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      if (n && !two) break;
      mask(s[n], key0 + 32 * n, holes(key0 + 32 * n));
      Weights p;
      weigh(s[n], scale, p, 0, 1);
      moderate(s[n], scale, p);
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          W8 v = only_seen(values(lds, 2 * n + k, d), see.hi_max + 1 - (key0 + 32 * n + 16 * k + 8 * half));
          if constexpr (FINITE) v = only_finite<W>(v);
          o[d] = mfma(v, p.w[k], o[d]);
        }
    }
  }
  __device__ __forceinline__ bool spoilt() const {
    bool x = false;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) x |= !(__builtin_fabsf(o[d][i]) < INFINITY);
    return __builtin_amdgcn_ballot_w64(x) != 0;
  }

  // Adds the values that only_finite() left out, at the keys k0 .. k1 - 1,
  // to the rows that see them: a sum with an infinity or a NaN in it.
  __device__ __forceinline__ void add_lost(const Cache<S>& c, int k0, int k1) {
#pragma unroll 1
    for (int key = k0; key < k1 && key <= see.hi_max; ++key) {
      const uint32_t e = c.entry(key);
      if (e >= c.num_blocks) continue;
      const bool mine = (key <= see.hi) & (key > see.lo);
      const uint64_t row = c.v + c.at(key, e);
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float x = stored<S>(row, 32 * d + 8 * (i / 4) + 4 * half + i % 4);
          o[d][i] += (mine & !(__builtin_fabsf(x) < INFINITY)) ? x : 0.0f;
        }
    }
  }

  __device__ __forceinline__ float row_sum() const {
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    return __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
  }

  // Result rows: into `out`, or unscaled into the workspace (row `at` on).
  __device__ __forceinline__ void store(const KvAttnArgs& a, const Item& it, int row0, int head, int64_t at, float* parts,
                                        float* stats) const {
    const float sum = row_sum(), top = told(a, it, see, m, sum);
    if (row0 + (lane & 31) >= it.rows) return;
    if (it.splits > 1) {
      at += lane & 31;
      if (half == 0) *(float2*)(stats + at * 2) = make_float2(top, sum);
      float* p = parts + at * S::D + 4 * half;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const f4 x = {o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]};
          *(f4*)(p + 32 * d + 2 * i) = x;
        }
      return;
    }
    const float inv = inverse(a.v_scale, sum, top == -INFINITY);  // a row that saw nothing has o = 0, too
    const int G = a.num_heads / a.num_kv_heads;
    T* p = (T*)a.out + (it.q0 + see.tok) * a.out_token_stride + (int64_t)(head * G + see.g) * a.out_head_stride + 4 * half;
    typedef T T4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        T4 x;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = (T)(o[d][i + j] * inv);
        *(T4*)(p + 32 * d + 2 * i) = x;
      }
  }
};

template <typename S, int R>
__device__ __forceinline__ void shared_tile(const KvAttnArgs& a, const Item& it, int head, uint32_t lds, int* flag,
                                            int64_t slot, float* parts, float* stats) {
  const int wave = uniform(threadIdx.x >> 6);
  Tile32<S> w;
  Cache<S> c;
  w.setup();
  c.setup(a, it.seq, head);
  constexpr int kHalf = S::ST * S::RB;  // bytes of a strip's keys
  const int strips = (it.k1 - it.k0 + S::ST - 1) / S::ST;

  // A strip's loads in groups of 16 keys of K or V; every wave takes its share.
  Ahead<S, 2> ahead;
  ahead.start(c, c.k, it.k0 + 16 * wave, S::ST, strips, it.k1);
  const uint64_t to_v = c.v - c.k;
  const auto dma_k = [&](int j) { return w.dma.of_k(j); };
  const auto dma_v = [&](int j) { return w.dma.of_v(j); };
  struct Next {
    uint64_t b[2];
    uint32_t to;
  };
  auto next = [&](int strip) {
    Next n;
    n.to = lds + (strip % R) * S::kStrip + wave * 16 * S::RB;
    ahead.get(c, strip, n.b);
    return n;
  };
  auto part = [&](const Next& n, int i) {
    if (i < S::NJ) load16<S>(dma_k, n.to, n.b[0], n.b[1], i);
    else if (i < 2 * S::NJ) load16<S>(dma_v, n.to + kHalf, to_v + n.b[0], to_v + n.b[1], i - S::NJ);
  };
  auto load = [&](int strip) {
    const Next n = next(strip);
#pragma unroll
    for (int i = 0; i < 2 * S::NJ; ++i) part(n, i);
  };
  auto begin = [&] {
    for (int i = 0; i < R - 1 && i < strips; ++i) load(i);
  };
  begin();
  const int row0 = it.row0 + wave * kRows;
  w.start(a, it, row0, head);
  // The waves' first addresses tell of their entries.
  const bool holes = strips <= 64 ? any_wave<kWaves>(ahead.holes, flag) : any_holes<kWaves>(a, it, flag);
  settle();
  int u0, u1;
  w.see.whole(it, strips, S::ST, holes, u0, u1);

  auto turn = [&](int strip) {
    // This strip has landed, for every wave, and everyone is done with the one before, whose place the next load takes.
    if (R > 2 && strip + R - 2 < strips) wait_vm<(R - 2) * 2 * S::NJ>();
    else wait_vm<0>();
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
  };
  auto pass = [&](auto finite) {
    w.clear();
    int strip = 0;
    while (strip < strips) {
      if (strip >= u0 && strip < u1) {
        __builtin_amdgcn_s_setprio(1);  // over waves that wait or mask: a late chunk of 64-dimensional heads 566 -> 559 us
        for (; strip < min(u1, strips - (R - 1)); ++strip) {
          turn(strip);
          const Next n = next(strip + R - 1);
          const uint32_t at = lds + (strip % R) * S::kStrip;
          w.strip(at, at + kHalf, a.score_scale, [&](int i) { part(n, i); });
        }
        for (; strip < u1; ++strip) {
          turn(strip);
          const uint32_t at = lds + (strip % R) * S::kStrip;
          w.strip(at, at + kHalf, a.score_scale, [](int) {});
        }
        __builtin_amdgcn_s_setprio(0);
      } else {
        turn(strip);
        if (strip + R - 1 < strips) load(strip + R - 1);
        const uint32_t at = lds + (strip % R) * S::kStrip;
        const int key0 = it.k0 + strip * S::ST;
        if (key0 <= w.see.hi_max)
          w.template strip_seen<decltype(finite)::value>(at, at + kHalf, a.score_scale, key0,
                                                         [&](int key) { return holes ? c.holes(key) : 0; });
        ++strip;
      }
    }
  };
  pass(std::false_type{});
  if (any_wave<kWaves>(w.spoilt(), flag)) {
    ahead.start(c, c.k, it.k0 + 16 * wave, S::ST, strips, it.k1);
    begin();
    pass(std::true_type{});
    w.add_lost(c, it.k0, u0 < u1 ? it.k0 + u0 * S::ST : it.k1);  // the strips that went through the mask
    if (u0 < u1) w.add_lost(c, it.k0 + u1 * S::ST, it.k1);
  }
  w.store(a, it, row0, head, slot * kTile + (row0 - it.row0), parts, stats);
}

// --------------------------------------------------------------- few rows
//
// At most 16 rows: bytes bound this, so the products are the smaller ones (16 x
// 16 x 32), and no wave waits for another: each takes strips of 32 keys of its
// own, through LDS of its own, and the results are joined at the end.
template <typename S>
struct Tile16 {
  typedef typename S::T T;
  typedef typename S::W W;
  typedef typename Vec<T>::v8 T8;
  typedef typename Vec<W>::v8 W8;
  typedef Tile16Order<S> Order;
  static constexpr int KS = S::D / 32;  // steps of the first product
  static constexpr int DT = S::D / 16;  // tiles of O^T
  static constexpr int KN = Order::KM / 4;

  int lane, quad;  // quad: the wave's quarter, which holds the scores of eight keys
  Sight see;
  T8 q[KS];
  f4 o[DT];
  float m, l;
  int koff[KN];
  // LDS offsets of V's reads; for 8-bit heads of 256, which would have sixteen, the first one, of which the others differ
  // by some bits.
  static constexpr bool kFewRegs = S::F8 && S::D == 256;
  static constexpr int VN = kFewRegs ? 1 : Order::VM;
  int voff[VN];
  Offsets<S, Order, S::D == 256> dma;

  // Row r of the first product's tile t is key 8 (r / 4) + 4 t + r % 4: quad q gets the keys 8 q .. 8 q + 7.
  __device__ __forceinline__ void setup() {
    lane = threadIdx.x & 63;
    quad = lane >> 4;
    const int n16 = lane & 15;
    const int key = 8 * (n16 >> 2) + (n16 & 3);
#pragma unroll
    for (int n = 0; n < KN; ++n) koff[n] = key * S::RB + ((4 * n + quad) ^ Order::k(key)) * 16;
    const int row = 8 * quad + (S::F8 ? n16 >> 1 : n16 >> 2);
    const int in = S::F8 ? (n16 & 1) * 8 : (n16 & 3) * 8;
#pragma unroll
    for (int n = 0; n < VN; ++n) voff[n] = row * S::RB + (n ^ Order::v(row)) * (16 * Order::U) + in;
    dma.setup();
  }

  // A 16-byte piece holds eight or (in 8 bits) sixteen values of a key: piece 4 s + quad for step s, or for the steps
  // 2 s and 2 s + 1.
  __device__ __forceinline__ void start(const KvAttnArgs& a, const Item& it, int row0, int head) {
    see.start(a, it, row0, lane & 15, kFew);
    const int G = a.num_heads / a.num_kv_heads;
    const T* p = (const T*)a.q + (it.q0 + see.tok) * a.q_token_stride + (int64_t)(head * G + see.g) * a.q_head_stride;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int d = S::F8 ? (4 * (s / 2) + quad) * 16 + 8 * (s & 1) : (4 * s + quad) * 8;
      q[s] = *(const T8*)(p + d);
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[d][i] = 0.0f;
    m = kNoScore;
    l = 0.0f;
  }

  // S^T of 32 keys: s[t][i] is key 8 quad + 4 t + i.
  __device__ __forceinline__ void scores(uint32_t lds, f4 (&s)[2]) const {
    uint32_t from[KN];
#pragma unroll
    for (int n = 0; n < KN; ++n) from[n] = pinned(lds + koff[n]);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[t][i] = 0.0f;
      constexpr int N = S::F8 ? KS / 2 : KS;
#pragma unroll
      for (int u = 0; u < N; ++u) {
        const uint32_t at = from[u % KN] + (u / KN) * (64 * KN) + 4 * t * S::RB;
        if constexpr (S::F8) {
          const i4 k = *(const SCOOT_LDS i4*)at;
#pragma unroll
          for (int e = 0; e < 2; ++e) s[t] = mfma(widen<T>(k[2 * e], k[2 * e + 1]), q[2 * u + e], s[t]);
        } else {
          s[t] = mfma(*(const SCOOT_LDS T8*)at, q[u], s[t]);
        }
      }
    }
  }

  // V^T: lane's element d = 16 dt + lane % 16 of the keys 8 quad .. + 7.
  __device__ __forceinline__ W8 values(uint32_t lds, int dt) const {
    const int n = dt % Order::VM;
    const uint32_t at = lds + (kFewRegs ? here(voff[0]) ^ n * 16 * Order::U : voff[n % VN]) + (dt / Order::VM) * (Order::VM * 16 * Order::U);
    if constexpr (S::F8) {
      const i2 v = __builtin_amdgcn_ds_read_tr8_b64_v2i32((SCOOT_LDS i2*)at);
      return widen<_Float16>(v[0], v[1]);
    } else {
      union {
        s4 h[2];
        W8 v;
      } r;
      r.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SCOOT_LDS s4*)at);
      r.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SCOOT_LDS s4*)(at + 4 * S::RB));
      return r.v;
    }
  }

  __device__ __forceinline__ void mask(f4 (&s)[2], int key0, int holes) const {
    const int first = key0 + 8 * quad;
    const int h = see.hi - first, l = see.lo - first;
    const bool none = (holes >> quad & 1) != 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const bool hidden = (k > h) | (k <= l) | none;
      s[k / 4][k % 4] = hidden ? -INFINITY : s[k / 4][k % 4];
    }
  }

  // As Tile32::weigh() and moderate().
  __device__ __forceinline__ W8 weights(const f4 (&s)[2], float scale) {
    float add = 0.0f;
    W8 w = eight_weights<W, false>([&](int i) { return s[i / 4][i % 4]; }, scale, m, 0.0f, add);
    if (__builtin_amdgcn_ballot_w64(!(add <= kMost))) {
      float x = s[0][0];
#pragma unroll
      for (int k = 1; k < 8; ++k) x = fmaxf(x, s[k / 4][k % 4]);
      auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
      x = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
      sw = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
      x = below(fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])), scale);
      uint32_t over = !(add <= kMost);
      sw = __builtin_amdgcn_permlane32_swap(over, over, false, false);
      over = sw[0] | sw[1];
      sw = __builtin_amdgcn_permlane16_swap(over, over, false, false);
      const bool moves = (sw[0] | sw[1]) != 0;
      const float up = moves && x > m ? x : m, f = __builtin_amdgcn_exp2f(m - up);
      m = up;
      l *= f;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[d][i] *= f;
      add = 0.0f;
      w = eight_weights<W, true>([&](int i) { return s[i / 4][i % 4]; }, scale, m, moves ? kLimit : INFINITY, add);
    }
    l += add;
    return w;
  }

  __device__ __forceinline__ void product(uint32_t lds, W8 w) {
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = mfma(values(lds, d), w, o[d]);
  }
  template <bool FINITE>
  __device__ __forceinline__ void product_seen(uint32_t lds, W8 w, int key0) {
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      W8 v = only_seen(values(lds, d), see.hi_max + 1 - (key0 + 8 * quad));
      if constexpr (FINITE) v = only_finite<W>(v);
      o[d] = mfma(v, w, o[d]);
    }
  }
  __device__ __forceinline__ bool spoilt() const {
    bool x = false;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) x |= !(__builtin_fabsf(o[d][i]) < INFINITY);
    return __builtin_amdgcn_ballot_w64(x) != 0;
  }

  __device__ __forceinline__ void add_lost(const Cache<S>& c, int k0, int k1) {
#pragma unroll 1
    for (int key = k0; key < k1 && key <= see.hi_max; ++key) {
      const uint32_t e = c.entry(key);
      if (e >= c.num_blocks) continue;
      const bool mine = (key <= see.hi) & (key > see.lo);
      const uint64_t row = c.v + c.at(key, e);
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = stored<S>(row, 16 * d + 4 * quad + i);
          o[d][i] += (mine & !(__builtin_fabsf(x) < INFINITY)) ? x : 0.0f;
        }
    }
  }

  __device__ __forceinline__ float row_sum() const {
    auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    const float x = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    sw = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
  }
};

template <typename S, int W>
__device__ __forceinline__ void few_rows(const KvAttnArgs& a, const Item& it, int row0, int head, uint32_t lds, char* smem,
                                         float* ml, int* flag, int64_t slot_row, float* parts, float* stats) {
  typedef typename S::T T;
  const int wave = uniform(threadIdx.x >> 6);
  Tile16<S> w;
  Cache<S> c;
  w.setup();
  c.setup(a, it.seq, head);
  constexpr int kHalf = 32 * S::RB;
  const uint32_t kat = lds + wave * (2 * kHalf), vat = kat + kHalf;
  const int strips = (it.k1 - it.k0 + 31) / 32;

  struct Base {
    uint64_t b[4];
  };
  Ahead<S, 4> ahead;  // its strips: every W-th one
  ahead.start(c, c.k, it.k0 + 32 * wave, 32 * W, (strips - wave + W - 1) / W, it.k1);
  const auto dma_k = [&](int j) { return w.dma.of_k(j); };
  const auto dma_v = [&](int j) { return w.dma.of_v(j); };
  auto load_k = [&](const Base& b) {
    load16<S>(dma_k, kat, b.b[0], b.b[1]);
    load16<S, Tile16Order<S>::kNext>(dma_k, kat + 16 * S::RB, b.b[2], b.b[3]);
  };
  const uint64_t to_v = c.v - c.k;
  auto load_v = [&](const Base& b) {
    load16<S>(dma_v, vat, to_v + b.b[0], to_v + b.b[1]);
    load16<S>(dma_v, vat + 16 * S::RB, to_v + b.b[2], to_v + b.b[3]);
  };

  Base b;
  auto begin = [&] {
    if (wave >= strips) return;
    ahead.get(c, 0, b.b);
    load_k(b);
    load_v(b);
  };
  begin();
  w.start(a, it, row0, head);
  // The first addresses tell of their entries.
  bool holes = ahead.holes;
  if (strips > 64 * W) holes = any_holes<W>(a, it, flag);
  settle();
  int u0, u1;  // strips seen whole by every row
  w.see.whole(it, strips, 32, holes, u0, u1);

  int strip;
  auto step = [&](auto masked, auto finite) {
    constexpr bool kMasked = decltype(masked)::value;
    const bool more = strip + W < strips;
    const int key0 = it.k0 + strip * 32;
    wait_vm<2 * S::NJ>();  // the keys, not the values behind them
    f4 s[2];
    w.scores(kat, s);
    wait_lds();
    if (more) {
      ahead.get(c, strip / W + 1, b.b);
      load_k(b);
    }
    if (kMasked) w.mask(s, key0, holes ? c.holes(key0) : 0);
    const typename Tile16<S>::W8 p = w.weights(s, a.score_scale);
    if (more) wait_vm<2 * S::NJ>();
    else wait_vm<0>();
    if (kMasked) w.template product_seen<decltype(finite)::value>(vat, p, key0);
    else w.product(vat, p);
    wait_lds();
    if (more) load_v(b);
    strip += W;
  };
  auto pass = [&](auto finite) {
    w.clear();
    strip = wave;
    while (strip < strips) {
      if (strip >= u0 && strip < u1) {
        while (strip < u1) step(std::false_type{}, finite);
      } else {
        step(std::true_type{}, finite);
      }
    }
  };
  pass(std::false_type{});
  if (w.spoilt()) {
    ahead.start(c, c.k, it.k0 + 32 * wave, 32 * W, (strips - wave + W - 1) / W, it.k1);
    begin();
    pass(std::true_type{});
    for (strip = wave; strip < strips; strip += W)
      if (strip < u0 || strip >= u1) w.add_lost(c, it.k0 + strip * 32, min(it.k0 + strip * 32 + 32, it.k1));
  }

  // Join the waves, in their order.
  const float sum = w.row_sum(), m = wave < strips ? told(a, it, w.see, w.m, sum) : kNoScore;
  __syncthreads();
  if (w.quad == 0) *(float2*)(ml + (wave * kFew + w.lane) * 2) = make_float2(m, sum);
  constexpr int kRow = S::D + 4;  // floats of a row, off by 16 bytes so that rows start on different banks
  float* mine = (float*)smem + (wave * kFew + (w.lane & 15)) * kRow + 4 * w.quad;
#pragma unroll
  for (int d = 0; d < Tile16<S>::DT; ++d) *(f4*)(mine + 16 * d) = w.o[d];
  __syncthreads();
  const int G = a.num_heads / a.num_kv_heads;
  const int rows = min(kFew, it.rows - row0);
  for (int i = threadIdx.x; i < rows * (S::D / 4); i += 64 * W) {
    const int r = i / (S::D / 4), d = i % (S::D / 4) * 4;
    float top = kNoScore, l = 0.0f;
    f4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int v = 0; v < W; ++v) top = fmaxf(top, ml[(v * kFew + r) * 2]);
#pragma unroll
    for (int v = 0; v < W; ++v) {
      const float f = __builtin_amdgcn_exp2f(ml[(v * kFew + r) * 2] - top);
      l += f * ml[(v * kFew + r) * 2 + 1];
      const f4 x = *(const f4*)((const float*)smem + (v * kFew + r) * kRow + d);
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] += f * x[j];
    }
    bool lost = false;
    if (l == 0.0f)
      for (int v = 0; v < W; ++v) lost |= ml[(v * kFew + r) * 2] == -INFINITY;
    if (it.splits > 1) {
      if (d == 0) *(float2*)(stats + (slot_row + r) * 2) = make_float2(lost ? -INFINITY : top, l);
      *(f4*)(parts + (slot_row + r) * S::D + d) = o;
    } else {
      const float inv = inverse(a.v_scale, l, lost);
      const int row = row0 + r, tok = row / G, g = row - tok * G;
      typedef T T4 __attribute__((ext_vector_type(4)));
      T4 y;
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] = (T)(o[j] * inv);
      *(T4*)((T*)a.out + (it.q0 + tok) * a.out_token_stride + (int64_t)(head * G + g) * a.out_head_stride + d) = y;
    }
  }
  __syncthreads();
}

// LDS of W waves: strips of keys (or what the waves' results are joined
// through), the waves' m and l, and their flags.
template <typename S, int W>
struct FewLds {
  static constexpr int kStrips = W * 64 * S::RB;  // per wave one strip of 32 keys of K and V
  static constexpr int kJoin = W * kFew * (S::D + 4) * 4;
  static constexpr int kStats = kStrips > kJoin ? kStrips : kJoin;
  static constexpr int kEnd = kStats + W * kFew * 8;
};
// R > 0: tiles through R buffers, requests of few rows among them; R = 0: these alone.
template <typename S, int R, int W>
constexpr int kFlagAt = R * S::kStrip > FewLds<S, W>::kEnd ? R * S::kStrip : FewLds<S, W>::kEnd;
template <typename S, int R, int W>
__global__ __launch_bounds__(64 * W, (waves_per_simd(S::D, R))) void attention_kernel(KvAttnArgs a, Plan p, float* parts, float* stats) {
  extern __shared__ __attribute__((aligned(256))) char smem[];
  const uint32_t lds = (uint32_t)(uintptr_t)(SCOOT_LDS char*)smem;
  const uint32_t heads = (uint32_t)a.num_kv_heads;
  const uint32_t head = blockIdx.x % heads, rest = blockIdx.x / heads;
  const uint32_t split = rest % (uint32_t)p.splits, index = rest / (uint32_t)p.splits;
  Item it;
  if (!find_item(a, p, index, (int)split, it)) return;
  const int64_t slot = blockIdx.x;
  int* flag = (int*)(smem + kFlagAt<S, R, W>);
  if constexpr (R > 0) {
    if (it.shared) {
      shared_tile<S, R>(a, it, (int)head, lds, flag, slot, parts, stats);
      return;
    }
  }
  float* ml = (float*)(smem + FewLds<S, W>::kStats);
  for (int row0 = 0; row0 < it.rows; row0 += kFew)
    few_rows<S, W>(a, it, row0, (int)head, lds, smem, ml, flag, slot * (R > 0 ? kTile : kFew), parts, stats);
}

// Joins the parts of a tile's keys: one workgroup per key head and as many rows
// as it has threads for, four dimensions each.  Latency bounds this, so the
// parts are read eight at a time.
template <typename S>
constexpr int kJoinRows = kThreads / (S::D / 4);

template <typename S>
__global__ __launch_bounds__(kThreads) void join_kernel(KvAttnArgs a, Plan p, const float* parts, const float* stats, int chunks) {
  typedef typename S::T T;
  const uint32_t heads = (uint32_t)a.num_kv_heads;
  const int tile = p.tile_rows ? p.tile_rows : kFew;
  const uint32_t head = blockIdx.x % heads, rest = blockIdx.x / heads, index = rest / (uint32_t)chunks;
  constexpr int per = S::D / 4;
  const int r = (int)(rest % (uint32_t)chunks) * kJoinRows<S> + (int)threadIdx.x / per, d = (int)threadIdx.x % per * 4;
  Item it;
  if (!find_item(a, p, index, 0, it) || it.splits < 2) return;
  if ((int)threadIdx.x >= kJoinRows<S> * per || r >= min(tile, it.rows - it.row0)) return;
  const int G = a.num_heads / a.num_kv_heads;
  const int64_t step = (int64_t)heads * tile;  // rows of the workspace from part to part
  const int64_t at = ((int64_t)index * p.splits * heads + head) * tile + r;
  float top = kNoScore, least = INFINITY, sum = 0.0f;
  f4 o = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s0 = 0; s0 < it.splits; s0 += 8) {
    float2 ml[8];
    f4 x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int64_t from = at + min(s0 + j, it.splits - 1) * step;
      ml[j] = *(const float2*)(stats + from * 2);
      x[j] = *(const f4*)(parts + from * S::D + d);
    }
    float up = top;
#pragma unroll
    for (int j = 0; j < 8; ++j) {  // the last part's again is no harm
      up = fmaxf(up, ml[j].x);
      least = fminf(least, ml[j].x);
    }
    const float f = __builtin_amdgcn_exp2f(top - up);
    top = up;
    sum *= f;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] *= f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float g = s0 + j < it.splits ? __builtin_amdgcn_exp2f(ml[j].x - up) : 0.0f;
      sum += s0 + j < it.splits ? ml[j].y * g : 0.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] += s0 + j < it.splits ? x[j][i] * g : 0.0f;
    }
  }
  const float inv = inverse(a.v_scale, sum, least == -INFINITY);
  const int row = it.row0 + r, tok = row / G, g = row - tok * G;
  T* out = (T*)a.out + (it.q0 + tok) * a.out_token_stride + (int64_t)(head * G + g) * a.out_head_stride + d;
  typedef T T4 __attribute__((ext_vector_type(4)));
  T4 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = (T)(o[i] * inv);
  *(T4*)out = y;
}

template <typename S, int R, int W>
int launch_kernel(const KvAttnArgs& a, const Plan& p, float* parts, float* stats, hipStream_t stream) {
  const int rc = allow_full_lds((const void*)attention_kernel<S, R, W>, "kv attention");
  if (rc != SCOOT_OK) return rc;
  hipLaunchKernelGGL((attention_kernel<S, R, W>), dim3((unsigned)(p.items * p.splits * a.num_kv_heads)), dim3(64 * W),
                     (kFlagAt<S, R, W> + 4 * W), stream, a, p, parts, stats);
  return SCOOT_OK;
}

template <typename S>
int launch(const KvAttnArgs& a, const Plan& p, float* parts, float* stats, hipStream_t stream) {
  int rc;
  if (p.tile_rows) {
    rc = launch_kernel<S, buffers(S::D, S::RB), kWaves>(a, p, parts, stats, stream);
  } else {
    if constexpr (S::RB <= kWideRow) {
      if (p.waves == 8) rc = launch_kernel<S, 0, 8>(a, p, parts, stats, stream);
      else rc = launch_kernel<S, 0, kWaves>(a, p, parts, stats, stream);
    } else {
      rc = launch_kernel<S, 0, kWaves>(a, p, parts, stats, stream);
    }
  }
  if (rc != SCOOT_OK) return rc;
  if (p.splits > 1) {
    const int chunks = ((p.tile_rows ? p.tile_rows : kFew) + kJoinRows<S> - 1) / kJoinRows<S>;
    hipLaunchKernelGGL((join_kernel<S>), dim3((unsigned)(p.items * chunks * a.num_kv_heads)), dim3(kThreads), 0, stream, a, p, parts,
                       stats, chunks);
  }
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return fail(SCOOT_ERR_DEVICE, std::string("kv attention launch: ") + hipGetErrorString(err));
  return SCOOT_OK;
}

// One per head dimension, each in a file of its own.
template <int D>
int launch_dim(const KvAttnArgs& a, const Plan& p, scoot_kv_type type, bool f8, float* parts, float* stats, hipStream_t stream);

#define SCOOT_KV_ATTN_DIM(D)                                                                                              \
  namespace scoot {                                                                                                       \
  namespace kvattn {                                                                                                      \
  template <>                                                                                                             \
  int launch_dim<D>(const KvAttnArgs& a, const Plan& p, scoot_kv_type type, bool f8, float* parts, float* stats,          \
                    hipStream_t s) {                                                                                      \
    if (type == SCOOT_KV_F16)                                                                                             \
      return f8 ? launch<Shape<_Float16, true, D>>(a, p, parts, stats, s)                                                 \
                : launch<Shape<_Float16, false, D>>(a, p, parts, stats, s);                                               \
    return f8 ? launch<Shape<__bf16, true, D>>(a, p, parts, stats, s) : launch<Shape<__bf16, false, D>>(a, p, parts, stats, s); \
  }                                                                                                                       \
  }                                                                                                                       \
  }

}  // namespace kvattn
}  // namespace scoot
