// Attention over the block cache: the kernels, for one head dimension per
// translation unit (k_kv_attn_<dim>.hip); k_kv_attn.hip holds the launches.
//
// Mathematics.  A row is one query of one head; the G query heads that share a
// key head are rows of the same tile, row = token * G + head.  With scores s_t
// = q . k_t the rows keep m, l and o over the keys seen so far: for every strip
// of keys, w_t = 2^(c s_t - m), l += sum w_t, o += sum w_t v_t; when a score
// passes m by more than 2^8, m moves up to it and l and o are multiplied by
// 2^(old m - m), so w stays below 2^8 and most strips leave o alone.  Parts of
// the keys that were handled by different waves or workgroups are joined by the
// same factors.
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
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "kv.h"

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

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kRows = 32;                    // rows (queries) of a wave
constexpr int kTileRows = kRows * kWaves;    // rows of a workgroup whose waves share the keys
constexpr float kNoScore = -3.0e38f;         // m before any key was seen; finite, so that m - m is 0
constexpr float kSlack = 8.0f;               // m follows a larger score only past this

constexpr int gcd256(int x) { return x % 256 == 0 ? 256 : x % 128 == 0 ? 128 : 64; }

// Sizes of a cache row and of the permutations of its pieces.  Rows g apart
// start on the same bank (256 bytes of LDS per cycle).
template <typename T_, bool F8_, int D_>
struct Shape {
  typedef T_ T;
  static constexpr bool F8 = F8_;
  static constexpr int D = D_;
  static constexpr int EB = F8 ? 1 : 2;
  static constexpr int RB = D * EB;                 // bytes of a row
  static constexpr int PC = RB / 16;                // 16-byte pieces of a row
  static constexpr int g = 256 / gcd256(RB);
  static constexpr int KM = 16 / g;                 // K: piece ^ (row / g % KM)
  static constexpr int VU = 2 * EB;                 // V: pieces of 32 elements, permuted together:
  static constexpr int VM = (8 / EB) / g;           //    32-element unit ^ (row / g % VM)
  static constexpr int DT = D / 32;                 // tiles of O^T
  static constexpr int KS = D / 16;                 // steps of the first product
  static constexpr int NJ = RB / 64;                // loads of 1 KiB for 16 rows
  static constexpr int ST = D <= 128 ? 64 : 32;     // keys per strip of a shared tile
  static constexpr int SUB = ST / 32;
  static constexpr int kShared = 4 * ST * RB;       // two buffers of K and V
  static constexpr int kPrivate = kWaves * 64 * RB; // per wave one strip of 32 keys of K and V
  static constexpr int kJoin = 2 * kRows * (D + 4) * 4;
  // The second product runs in the cache's 16-bit type; 8-bit values are exact in half precision, which rounds the
  // weights eight times finer than bfloat16.
  typedef typename std::conditional<F8, _Float16, T>::type W;
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

// The key, of a strip's 32, that row r of the first product's left operand
// holds: rows 4h .. 4h + 3 and 8 + 4h .. (the scores of the wave's half h) are
// keys 8h .. 8h + 7.
__device__ __forceinline__ int key_of_row(int r) { return (r & 19) | ((r & 4) << 1) | ((r & 8) >> 1); }

template <int N>
__device__ __forceinline__ void wait_vm() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// 64 lanes x 16 bytes from base + off to LDS at `to`, lane after lane; counted
// by vmcnt.  The compiler does not know of the write: whoever reads it waits
// first.  Written out because the compiler, for the builtin, waits for all
// loads in flight before any read of LDS.
__device__ __forceinline__ void load_lds(uint32_t to, uint64_t base, uint32_t off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void load_lds(uint32_t to, uint64_t addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(to), "v"(addr) : "memory");
}

// What a workgroup works on: rows r0 .. r0 + 127 (or 31) of a request, one key
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
  bool shared;      // the waves share the keys (more than kRows rows), else each wave takes strips of its own
};

struct Plan {
  int64_t items;    // tiles or requests
  int splits;
  int part;         // keys per part, a multiple of 128
  bool mixed;       // tiles of kTileRows rows; else requests
};

__device__ __forceinline__ int64_t clamp64(int64_t v, int64_t lo, int64_t hi) { return v < lo ? lo : v > hi ? hi : v; }

__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Finds the item: false if there is none.  All values are the same in every lane.
//
// Tiles need no list: request i, whose tokens start at s_i, owns the numbers
// from floor(s_i G / 128) + i on, which are enough for its ceil(n_i G / 128)
// tiles whatever n_i is; the request of a number is searched for 64-fold.
__device__ __forceinline__ bool find_item(const KvAttnArgs& a, const Plan& p, int64_t index, int split, Item& it) {
  const int G = a.num_heads / a.num_kv_heads;
  const SCOOT_CONST int32_t* qs = (const SCOOT_CONST int32_t*)a.query_start;
  int seq;
  int64_t first = 0;
  if (p.mixed) {
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = a.num_seqs;
    bool any = true;
    do {
      const int step = (hi - lo + 63) / 64;
      const int64_t i = lo + (int64_t)lane * step;
      bool below = false;
      if (i < hi) below = clamp64(a.query_start[i], 0, a.num_tokens) * G / kTileRows + i <= index;
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
    first = clamp64(qs[seq], 0, a.num_tokens) * G / kTileRows + seq;
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
  it.shared = p.mixed && rows > kRows;
  int last_row = it.rows - 1;
  int splits = p.splits;
  if (it.shared) {
    const int tiles = (it.rows + kTileRows - 1) / kTileRows;
    const int64_t t = index - first;
    if (t >= tiles) return false;
    it.row0 = (tiles - 1 - (int)t) * kTileRows;  // the tiles that see most come first
    if (it.row0 + kTileRows - 1 < last_row) last_row = it.row0 + kTileRows - 1;
  } else {
    if (p.mixed && index != first) return false;
    it.row0 = 0;
    if (it.rows > kRows) splits = 1;  // more rows than the caller announced: one workgroup, tile after tile
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

// One wave's rows and what it knows of the keys.
template <typename S>
struct Wave {
  typedef typename S::T T;
  typedef typename S::W W;
  typedef typename Vec<T>::v8 T8;
  typedef typename Vec<W>::v8 W8;

  int lane, half;
  int hi, lo;              // this lane's row sees keys lo < k <= hi
  int hi_min, hi_max, lo_max;  // over the wave's rows
  T8 q[S::KS];
  f16v o[S::DT];
  float m, l;
  int koff[S::KM / 2];     // LDS offsets of this lane's reads
  int voff[S::VM];
  uint32_t kdma[S::NJ], vdma[S::NJ];  // memory offsets of its loads

  __device__ __forceinline__ void setup() {
    lane = threadIdx.x & 63;
    half = lane >> 5;
    const int key = key_of_row(lane & 31);
#pragma unroll
    for (int n = 0; n < S::KM / 2; ++n) koff[n] = key * S::RB + (((2 * n + half) ^ (key / S::g % S::KM)) * 16);
    const int n16 = lane & 15, dhalf = (lane >> 4) & 1;
    const int row = 8 * half + (S::F8 ? n16 >> 1 : n16 >> 2);
    const int in = S::F8 ? dhalf * 16 + (n16 & 1) * 8 : dhalf * 32 + (n16 & 3) * 8;
#pragma unroll
    for (int n = 0; n < S::VM; ++n) voff[n] = row * S::RB + (n ^ (row / S::g % S::VM)) * (16 * S::VU) + in;
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) {
      const int at = 64 * j + lane, r = at / S::PC, p = at % S::PC;
      kdma[j] = (r & 7) * S::RB + (p ^ (r / S::g % S::KM)) * 16;
      vdma[j] = (r & 7) * S::RB + (((p / S::VU) ^ (r / S::g % S::VM)) * S::VU + p % S::VU) * 16;
    }
  }

  // Rows row0 .. row0 + 31 of the request (those past its last row repeat it; nothing of them is stored).
  __device__ __forceinline__ void start(const KvAttnArgs& a, const Item& it, int row0, int head) {
    const int G = a.num_heads / a.num_kv_heads;
    int row = row0 + (lane & 31);
    row = row < it.rows ? row : it.rows - 1;
    const int tok = row / G, g = row - tok * G;
    const int64_t pos = it.pos0 + tok;
    hi = (int)clamp64(pos, -1, it.len - 1);
    lo = a.window > 0 ? (int)clamp64(pos - a.window, -1, 0x7fffffff) : -1;
    hi_min = hi_max = hi;
    lo_max = lo;
#pragma unroll
    for (int x = 1; x < 32; x <<= 1) {
      hi_min = min(hi_min, __shfl_xor(hi_min, x));
      hi_max = max(hi_max, __shfl_xor(hi_max, x));
      lo_max = max(lo_max, __shfl_xor(lo_max, x));
    }
    hi_min = uniform(hi_min);
    hi_max = uniform(hi_max);
    lo_max = uniform(lo_max);
    const T* p = (const T*)a.q + (it.q0 + tok) * a.q_token_stride + (int64_t)(head * G + g) * a.q_head_stride;
#pragma unroll
    for (int s = 0; s < S::KS; ++s) {
      const int d = S::F8 ? (2 * (s / 2) + half) * 16 + 8 * (s & 1) : (2 * s + half) * 8;
      q[s] = *(const T8*)(p + d);
    }
#pragma unroll
    for (int d = 0; d < S::DT; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
    m = kNoScore;
    l = 0.0f;
  }

  // The loads of 16 keys (two groups of eight, each inside a block) to LDS.
  static __device__ __forceinline__ void load16(const uint32_t (&off)[S::NJ], uint32_t to, uint64_t b0, uint64_t b1) {
#pragma unroll
    for (int j = 0; j < S::NJ; ++j) {
      constexpr int kHalf = 8 * S::PC;  // pieces of eight keys
      if (64 * j + 63 < kHalf)
        load_lds(to + 1024 * j, b0, off[j]);
      else if (64 * j >= kHalf)
        load_lds(to + 1024 * j, b1, off[j]);
      else
        load_lds(to + 1024 * j, (64 * j + (int)(threadIdx.x & 63) < kHalf ? b0 : b1) + off[j]);
    }
  }

  // S^T of 32 keys.
  __device__ __forceinline__ f16v scores(uint32_t lds) const {
    f16v s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.0f;
    constexpr int N = S::KM / 2;
    if constexpr (S::F8) {
#pragma unroll
      for (int u = 0; u < S::KS / 2; ++u) {
        const i4 k = *(const SCOOT_LDS i4*)(lds + koff[u % N] + (u / N) * (16 * S::KM));
#pragma unroll
        for (int e = 0; e < 2; ++e) s = mfma(widen<T>(k[2 * e], k[2 * e + 1]), q[2 * u + e], s);
      }
    } else {
#pragma unroll
      for (int u = 0; u < S::KS; ++u) {
        const T8 k = *(const SCOOT_LDS T8*)(lds + koff[u % N] + (u / N) * (16 * S::KM));
        s = mfma(k, q[u], s);
      }
    }
    return s;
  }

  // Eight 8-bit floats as 16-bit ones (exact).
  template <typename R>
  static __device__ __forceinline__ typename Vec<R>::v8 widen(int a, int b) {
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

  // V^T: lane's element d = 32 dt + lane % 32 of the keys 16 ks + 8 half .. + 7.
  __device__ __forceinline__ W8 values(uint32_t lds, int ks, int dt) const {
    const uint32_t at = lds + voff[dt % S::VM] + (dt / S::VM) * (S::VM * 16 * S::VU) + ks * 16 * S::RB;
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
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int k = 16 * (i / 8) + 8 * half + (i & 7);
      const int key = key0 + k;
      if (key > hi || key <= lo || (holes >> (k / 8) & 1)) s[i] = -INFINITY;
    }
  }

  // Weights of N strips of 32 keys, in place, rounded: m, l and o follow.
  template <int N>
  __device__ __forceinline__ void weights(f16v (&s)[N], float scale, W8 (&w)[2 * N]) {
    float x = s[0][0];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) x = fmaxf(x, s[n][i]);
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * scale;
    if (__builtin_amdgcn_ballot_w64(x > m + kSlack)) {
      const float up = x > m + kSlack ? x : m, f = __builtin_amdgcn_exp2f(m - up);  // no row's m depends on another row
      m = up;
      l *= f;
#pragma unroll
      for (int d = 0; d < S::DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] *= f;
    }
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        W8 r;
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = (W)__builtin_amdgcn_exp2f(fmaf(s[n][8 * k + i], scale, -m));
        w[2 * n + k] = r;
        // The sum takes the weights as rounded, like the product.
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          if constexpr (std::is_same<W, _Float16>::value) {
            const h2 p = {r[i], r[i + 1]}, one = {(_Float16)1.0f, (_Float16)1.0f};
            l = __builtin_amdgcn_fdot2(p, one, l, false);
          } else {
            const b2 p = {r[i], r[i + 1]}, one = {(__bf16)1.0f, (__bf16)1.0f};
            l = __builtin_amdgcn_fdot2_f32_bf16(p, one, l, false);
          }
        }
      }
  }

  template <int N>
  __device__ __forceinline__ void product(uint32_t lds, const W8 (&w)[2 * N]) {
#pragma unroll
    for (int k = 0; k < 2 * N; ++k)
#pragma unroll
      for (int d = 0; d < S::DT; ++d) o[d] = mfma(values(lds, k, d), w[k], o[d]);
  }

  // The same where some rows do not see some keys: 0 * inf must not arise.
  // What is not finite is taken out of the product, and rows with a weight on
  // it get it back as what it is.
  template <int N>
  __device__ __forceinline__ void product_masked(uint32_t lds, const W8 (&w)[2 * N]) {
    constexpr uint32_t kExp = std::is_same<W, _Float16>::value ? 0x7c00u : 0x7f80u;
    constexpr uint32_t kOne = std::is_same<W, _Float16>::value ? 0x3c00u : 0x3f80u;
#pragma unroll
    for (int d = 0; d < S::DT; ++d) {
#pragma unroll
      for (int k = 0; k < 2 * N; ++k) {
        union {
          W8 v;
          uint16_t u[8];
          uint32_t w[4];
        } x, y;
        x.v = values(lds, k, d);
        uint32_t bad = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          // all exponent bits set carries into the sign's place
          const uint32_t e = x.w[i] & (kExp | kExp << 16);
          bad |= (e + ((0x8000u - kExp) * 0x10001u)) & 0x80008000u;
        }
        if (__builtin_amdgcn_ballot_w64(bad != 0)) {
#pragma unroll 1
          for (int kind = 0; kind < 3; ++kind) {  // +inf, -inf, NaN
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const uint32_t u = x.u[i];
              const bool is = kind == 0 ? u == kExp : kind == 1 ? u == (kExp | 0x8000u) : (u & 0x7fffu) > kExp;
              y.u[i] = is ? kOne : 0;
            }
            f16v c;
#pragma unroll
            for (int i = 0; i < 16; ++i) c[i] = 0.0f;
            c = mfma(y.v, w[k], c);
            const float add = kind == 0 ? INFINITY : kind == 1 ? -INFINITY : __uint_as_float(0x7fc00000u);
#pragma unroll
            for (int i = 0; i < 16; ++i)
              if (!(c[i] == 0.0f)) o[d][i] += add;
          }
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if ((x.u[i] & kExp) == kExp) x.u[i] = 0;
        }
        o[d] = mfma(x.v, w[k], o[d]);
      }
    }
  }

  // Whether the strip's keys need a mask, or are not seen at all.
  __device__ __forceinline__ bool unseen(int key0) const { return key0 > hi_max; }
  __device__ __forceinline__ bool partly(int key0, int n) const { return key0 + n - 1 > hi_min || key0 <= lo_max; }

  __device__ __forceinline__ float row_sum() const {
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    return __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
  }
};

// Blocks of the cache, as scalars.
template <typename S>
struct Cache {
  const SCOOT_CONST int32_t* table;
  uint64_t k, v;
  uint64_t block_bytes;  // of all heads
  uint32_t num_blocks;
  int shift, last;       // last entry of the row

  __device__ __forceinline__ void setup(const KvAttnArgs& a, int seq, int head) {
    table = (const SCOOT_CONST int32_t*)(a.block_table + (int64_t)seq * a.table_stride);
    const uint64_t head_bytes = (uint64_t)S::RB << a.block_shift;
    block_bytes = head_bytes * a.num_kv_heads;
    k = (uint64_t)a.k_cache + head * head_bytes;
    v = (uint64_t)a.v_cache + head * head_bytes;
    num_blocks = (uint32_t)a.num_blocks;
    shift = a.block_shift;
    last = a.max_blocks - 1;
  }
  // Byte offset of eight keys from `key` on (inside one block).  An entry that names no block reads block 0, and the
  // mask drops it.
  __device__ __forceinline__ uint64_t at(int key) const {
    int e = key >> shift;
    e = e < last ? e : last;
    uint32_t b = (uint32_t)table[e];
    b = b < num_blocks ? b : 0;
    return b * block_bytes + (uint64_t)(key & ((1 << shift) - 1)) * S::RB;
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

// Result rows of a wave: into `out`, or unscaled into the workspace.
template <typename S>
__device__ __forceinline__ void store_rows(const KvAttnArgs& a, const Wave<S>& w, const Item& it, int row0, int head, float m,
                                           float l, int64_t slot, int slot_row, float* parts, float* stats, int tile_rows) {
  typedef typename S::T T;
  const int G = a.num_heads / a.num_kv_heads;
  const int row = row0 + (w.lane & 31);
  if (row >= it.rows) return;
  if (it.splits > 1) {
    const int64_t at = slot * tile_rows + slot_row + (w.lane & 31);
    if (w.half == 0) *(float2*)(stats + at * 2) = make_float2(m, l);
    float* p = parts + at * S::D;
#pragma unroll
    for (int d = 0; d < S::DT; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const f4 x = {w.o[d][i], w.o[d][i + 1], w.o[d][i + 2], w.o[d][i + 3]};
        *(f4*)(p + 32 * d + 2 * i + 4 * w.half) = x;
      }
    return;
  }
  const float inv = l == 0.0f ? 0.0f : a.v_scale / l;  // a row that saw nothing has o = 0, too
  const int tok = row / G, g = row - tok * G;
  T* p = (T*)a.out + (it.q0 + tok) * a.out_token_stride + (int64_t)(head * G + g) * a.out_head_stride;
  typedef T T4 __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int d = 0; d < S::DT; ++d)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      T4 x;
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = (T)(w.o[d][i + j] * inv);
      *(T4*)(p + 32 * d + 2 * i + 4 * w.half) = x;
    }
}

// Whether any of the item's keys lies in an entry that names no block; `flag`:
// a word of LDS for every wave.
__device__ __forceinline__ bool any_holes(const KvAttnArgs& a, const Item& it, int* flag) {
  const int32_t* t = a.block_table + (int64_t)it.seq * a.table_stride;
  bool h = false;
  for (int64_t e = (it.k0 >> a.block_shift) + threadIdx.x; (e << a.block_shift) < it.k1; e += kThreads)
    h = h || (uint32_t)t[e] >= (uint32_t)a.num_blocks;
  const bool any = __builtin_amdgcn_ballot_w64(h) != 0;
  if ((threadIdx.x & 63) == 0) flag[threadIdx.x >> 6] = any;
  __syncthreads();
  return uniform(flag[0] | flag[1] | flag[2] | flag[3]) != 0;
}

// More than 32 rows: the four waves take 32 rows each and share strips of keys
// through two LDS buffers.
template <typename S>
__device__ __forceinline__ void shared_tile(const KvAttnArgs& a, const Item& it, int head, uint32_t lds, int* flag,
                                            int64_t slot, float* parts, float* stats) {
  const int wave = uniform(threadIdx.x >> 6);
  Wave<S> w;
  Cache<S> c;
  w.setup();
  c.setup(a, it.seq, head);
  constexpr int kHalf = S::ST * S::RB;  // bytes of a strip's keys
  const int strips = (it.k1 - it.k0 + S::ST - 1) / S::ST;

  // A strip's loads in groups of 16 keys of K or V; every wave takes its share.
  auto load = [&](int strip) {
    const uint32_t to = lds + (strip & 1) * (2 * kHalf);
    const int key0 = it.k0 + strip * S::ST;
    if constexpr (S::SUB == 2) {
      const int key = key0 + 16 * wave;
      const uint64_t b0 = c.at(key), b1 = c.at(key + 8);
      Wave<S>::load16(w.kdma, to + wave * 16 * S::RB, c.k + b0, c.k + b1);
      Wave<S>::load16(w.vdma, to + kHalf + wave * 16 * S::RB, c.v + b0, c.v + b1);
    } else {
      const int part = wave & 1;
      const int key = key0 + 16 * part;
      const uint64_t b0 = c.at(key), b1 = c.at(key + 8);
      if (wave < 2) Wave<S>::load16(w.kdma, to + part * 16 * S::RB, c.k + b0, c.k + b1);
      else Wave<S>::load16(w.vdma, to + kHalf + part * 16 * S::RB, c.v + b0, c.v + b1);
    }
  };

  if (strips > 0) load(0);
  w.start(a, it, it.row0 + wave * kRows, head);
  const bool holes = any_holes(a, it, flag);
  for (int strip = 0; strip < strips; ++strip) {
    // This strip has landed, for every wave, and everyone is done with the other buffer.
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (strip + 1 < strips) load(strip + 1);
    const uint32_t at = lds + (strip & 1) * (2 * kHalf);
    const int key0 = it.k0 + strip * S::ST;
    if (w.unseen(key0)) continue;
    f16v s[S::SUB];
#pragma unroll
    for (int n = 0; n < S::SUB; ++n) s[n] = w.scores(at + n * 32 * S::RB);
    typename Wave<S>::W8 p[2 * S::SUB];
    const bool masked = holes || w.partly(key0, S::ST);
    if (masked) {
#pragma unroll
      for (int n = 0; n < S::SUB; ++n) w.mask(s[n], key0 + 32 * n, holes ? c.holes(key0 + 32 * n) : 0);
    }
    w.template weights<S::SUB>(s, a.score_scale, p);
    if (masked) w.template product_masked<S::SUB>(at + kHalf, p);
    else w.template product<S::SUB>(at + kHalf, p);
  }
  store_rows<S>(a, w, it, it.row0 + wave * kRows, head, w.m, w.row_sum(), slot, wave * kRows, parts, stats, kTileRows);
}

// At most 32 rows: every wave takes strips of 32 keys of its own, through LDS
// of its own, and the waves' results are joined at the end.
template <typename S>
__device__ __forceinline__ void private_rows(const KvAttnArgs& a, const Item& it, int row0, int head, uint32_t lds, char* smem, int* flag,
                                             int64_t slot, float* parts, float* stats, int tile_rows) {
  const int wave = uniform(threadIdx.x >> 6);
  Wave<S> w;
  Cache<S> c;
  w.setup();
  c.setup(a, it.seq, head);
  constexpr int kHalf = 32 * S::RB;
  const uint32_t kat = lds + wave * (2 * kHalf), vat = kat + kHalf;
  const int strips = (it.k1 - it.k0 + 31) / 32;

  struct Base {
    uint64_t b[4];
  };
  auto base = [&](int strip) {
    Base r;
#pragma unroll
    for (int j = 0; j < 4; ++j) r.b[j] = c.at(it.k0 + strip * 32 + 8 * j);
    return r;
  };
  auto load = [&](const uint32_t (&off)[S::NJ], uint32_t to, uint64_t from, const Base& b) {
    Wave<S>::load16(off, to, from + b.b[0], from + b.b[1]);
    Wave<S>::load16(off, to + 16 * S::RB, from + b.b[2], from + b.b[3]);
  };

  int strip = wave;
  Base b{};
  if (strip < strips) {
    b = base(strip);
    load(w.kdma, kat, c.k, b);
    load(w.vdma, vat, c.v, b);
  }
  w.start(a, it, row0, head);
  const bool holes = any_holes(a, it, flag);
  for (; strip < strips; strip += kWaves) {
    const bool more = strip + kWaves < strips;
    const int key0 = it.k0 + strip * 32;
    b = base(strip + kWaves);
    wait_vm<2 * S::NJ>();  // the keys, not the values behind them
    f16v s[1] = {w.scores(kat)};
    wait_lds();
    if (more) load(w.kdma, kat, c.k, b);
    const bool masked = holes || w.partly(key0, 32);
    if (masked) w.mask(s[0], key0, holes ? c.holes(key0) : 0);
    typename Wave<S>::W8 p[2];
    w.template weights<1>(s, a.score_scale, p);
    if (more) wait_vm<2 * S::NJ>();
    else wait_vm<0>();
    if (masked) w.template product_masked<1>(vat, p);
    else w.template product<1>(vat, p);
    wait_lds();
    if (more) load(w.vdma, vat, c.v, b);
  }

  // Join the waves: 2, 3 into 0, 1, then 1 into 0.
  float m = w.m, l = w.row_sum();
  float* ml = (float*)(smem + (S::kPrivate > S::kJoin ? S::kPrivate : S::kJoin));
  __syncthreads();
  if (w.half == 0) {
    ml[(wave * 32 + w.lane) * 2] = m;
    ml[(wave * 32 + w.lane) * 2 + 1] = l;
  }
  __syncthreads();
  float top = kNoScore, sum = 0.0f;
#pragma unroll
  for (int v = 0; v < kWaves; ++v) top = fmaxf(top, ml[(v * 32 + (w.lane & 31)) * 2]);
#pragma unroll
  for (int v = 0; v < kWaves; ++v)
    sum += ml[(v * 32 + (w.lane & 31)) * 2 + 1] * __builtin_amdgcn_exp2f(ml[(v * 32 + (w.lane & 31)) * 2] - top);
  const float f = __builtin_amdgcn_exp2f(m - top);
#pragma unroll
  for (int d = 0; d < S::DT; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) w.o[d][i] *= f;
  const bool real = row0 + (w.lane & 31) < it.rows;
  float* mine = (float*)smem + ((wave & 1) * 32 + (w.lane & 31)) * (S::D + 4) + 4 * w.half;
#pragma unroll
  for (int step = 2; step > 0; step >>= 1) {
    if (real && wave >= step && wave < 2 * step) {
#pragma unroll
      for (int d = 0; d < S::DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const f4 x = {w.o[d][i], w.o[d][i + 1], w.o[d][i + 2], w.o[d][i + 3]};
          *(f4*)((step == 2 ? mine : mine - 32 * (S::D + 4)) + 32 * d + 2 * i) = x;
        }
    }
    __syncthreads();
    if (real && wave < step) {
#pragma unroll
      for (int d = 0; d < S::DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const f4 x = *(const f4*)(mine + 32 * d + 2 * i);
#pragma unroll
          for (int j = 0; j < 4; ++j) w.o[d][i + j] += x[j];
        }
    }
    __syncthreads();
  }
  if (wave == 0) store_rows<S>(a, w, it, row0, head, top, sum, slot, 0, parts, stats, tile_rows);
}

// LDS: strips of keys (or what the waves' results are joined through), the
// waves' m and l, and their flags.
template <typename S>
constexpr int kPrivateBytes = (S::kPrivate > S::kJoin ? S::kPrivate : S::kJoin) + kWaves * kRows * 8;
template <typename S, bool MIXED>
constexpr int kFlagAt = MIXED && S::kShared > kPrivateBytes<S> ? S::kShared : kPrivateBytes<S>;

template <typename S, bool MIXED>
__global__ __launch_bounds__(kThreads, S::D <= 128 ? 2 : 1) void attention_kernel(KvAttnArgs a, Plan p, float* parts, float* stats) {
  extern __shared__ __attribute__((aligned(256))) char smem[];
  const uint32_t lds = (uint32_t)(uintptr_t)(SCOOT_LDS char*)smem;
  const uint32_t heads = (uint32_t)a.num_kv_heads;
  const uint32_t head = blockIdx.x % heads, rest = blockIdx.x / heads;
  const uint32_t split = rest % (uint32_t)p.splits, index = rest / (uint32_t)p.splits;
  Item it;
  if (!find_item(a, p, index, (int)split, it)) return;
  const int64_t slot = blockIdx.x;
  if constexpr (MIXED) {
    if (it.shared) {
      shared_tile<S>(a, it, (int)head, lds, (int*)(smem + kFlagAt<S, MIXED>), slot, parts, stats);
      return;
    }
  }
  for (int row0 = 0; row0 < it.rows; row0 += kRows)
    private_rows<S>(a, it, row0, (int)head, lds, smem, (int*)(smem + kFlagAt<S, MIXED>), slot, parts, stats, MIXED ? kTileRows : kRows);
}

// Joins the parts of a tile's keys: one workgroup per tile and key head.
template <typename S>
__global__ __launch_bounds__(kThreads) void join_kernel(KvAttnArgs a, Plan p, const float* parts, const float* stats) {
  typedef typename S::T T;
  const uint32_t heads = (uint32_t)a.num_kv_heads;
  const uint32_t head = blockIdx.x % heads, index = blockIdx.x / heads;
  Item it;
  if (!find_item(a, p, index, 0, it) || it.splits < 2) return;
  const int tile_rows = p.mixed ? kTileRows : kRows;
  const int G = a.num_heads / a.num_kv_heads;
  const int rows = min(tile_rows, it.rows - it.row0);
  constexpr int per = S::D / 4;
  for (int i = threadIdx.x; i < rows * per; i += kThreads) {
    const int r = i / per, d = (i - r * per) * 4;
    float top = kNoScore, sum = 0.0f;
    f4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s = 0; s < it.splits; ++s) {
      const int64_t at = (((int64_t)index * p.splits + s) * heads + head) * tile_rows + r;
      top = fmaxf(top, stats[at * 2]);
    }
    for (int s = 0; s < it.splits; ++s) {
      const int64_t at = (((int64_t)index * p.splits + s) * heads + head) * tile_rows + r;
      const float f = __builtin_amdgcn_exp2f(stats[at * 2] - top);
      sum += f * stats[at * 2 + 1];
      const f4 x = *(const f4*)(parts + at * S::D + d);
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] += f * x[j];
    }
    const float inv = sum == 0.0f ? 0.0f : a.v_scale / sum;
    const int row = it.row0 + r, tok = row / G, g = row - tok * G;
    T* out = (T*)a.out + (it.q0 + tok) * a.out_token_stride + (int64_t)(head * G + g) * a.out_head_stride + d;
    typedef T T4 __attribute__((ext_vector_type(4)));
    T4 x;
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = (T)(o[j] * inv);
    *(T4*)out = x;
  }
}

template <typename S>
int launch(const KvAttnArgs& a, const Plan& p, float* parts, float* stats, hipStream_t stream) {
  const dim3 grid((unsigned)(p.items * p.splits * a.num_kv_heads)), join((unsigned)(p.items * a.num_kv_heads));
  const int bytes = (p.mixed ? kFlagAt<S, true> : kFlagAt<S, false>) + 4 * kWaves;
  const void* f = p.mixed ? (const void*)attention_kernel<S, true> : (const void*)attention_kernel<S, false>;
  const int rc = allow_full_lds(f, "kv attention");
  if (rc != SCOOT_OK) return rc;
  if (p.mixed)
    hipLaunchKernelGGL((attention_kernel<S, true>), grid, dim3(kThreads), bytes, stream, a, p, parts, stats);
  else
    hipLaunchKernelGGL((attention_kernel<S, false>), grid, dim3(kThreads), bytes, stream, a, p, parts, stats);
  if (p.splits > 1) hipLaunchKernelGGL((join_kernel<S>), join, dim3(kThreads), 0, stream, a, p, parts, stats);
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
