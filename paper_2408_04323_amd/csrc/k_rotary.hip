// Rotations by position, and appends to the block cache with the rotation on
// the way (scoot_rotate, scoot_kv_append).
#include <hip/hip_runtime.h>

#include <type_traits>

#include "kv.h"
#include "kv_vec.h"

namespace scoot {
namespace {

// Pair i of a vector at position p is turned by the angle p f_i:
//   a' = a c - b s,  b' = b c + a s,  (c, s) = magnitude (cos, sin)(p f_i),
// s with the other sign in reverse.  The pairs are elements (i, i + turned / 2),
// or neighbours (2 i, 2 i + 1); elements from `turned` on stay.
//
// Angles grow with the position (10^6 radians in a long context, where a float
// is off by 0.06), so they and their cosines are in double; c and s are rounded
// to float, a' and b' made of three roundings each, and then rounded once to the
// type that is stored.

// A number in scalar registers, made where it is used: the compiler would keep all of a series' in vector registers.
__device__ __forceinline__ double term(double x) {
  asm volatile("" : "+s"(x));
  return x;
}

// cos and sin of x in double: x less the nearest multiple n of pi / 2, which is taken away in two parts (exact but for
// 2^-53 of the rest, as fma rounds once), and the Taylor series up to pi / 4, whose next terms are below 2^-54.
__device__ __forceinline__ float2 turn_of(double x, double magnitude, bool reverse) {
  const double n = __builtin_rint(x * 0.63661977236758134308);
  double r = __builtin_fma(-n, 1.57079632679489655800, x);
  r = __builtin_fma(-n, 6.12323399573676603587e-17, r);
  const double z = r * r;
  double s = term(-1.0 / 1307674368000.0);  // 15!
  s = __builtin_fma(s, z, term(1.0 / 6227020800.0));
  s = __builtin_fma(s, z, term(-1.0 / 39916800.0));
  s = __builtin_fma(s, z, term(1.0 / 362880.0));
  s = __builtin_fma(s, z, term(-1.0 / 5040.0));
  s = __builtin_fma(s, z, term(1.0 / 120.0));
  s = __builtin_fma(s, z, term(-1.0 / 6.0));
  s = __builtin_fma(s * z, r, r);
  double c = term(1.0 / 20922789888000.0);  // 16!
  c = __builtin_fma(c, z, term(-1.0 / 87178291200.0));
  c = __builtin_fma(c, z, term(1.0 / 479001600.0));
  c = __builtin_fma(c, z, term(-1.0 / 3628800.0));
  c = __builtin_fma(c, z, term(1.0 / 40320.0));
  c = __builtin_fma(c, z, term(-1.0 / 720.0));
  c = __builtin_fma(c, z, term(1.0 / 24.0));
  c = __builtin_fma(c, z, -0.5);
  c = __builtin_fma(c, z, 1.0);
  const int quarter = (int)(n - 4.0 * __builtin_floor(n * 0.25));
  double cx = quarter & 1 ? s : c, sx = quarter & 1 ? c : s;
  if (quarter == 1 || quarter == 2) cx = -cx;
  if ((quarter >= 2) != reverse) sx = -sx;
  return make_float2((float)(cx * magnitude), (float)(sx * magnitude));
}

// x / scale, limited to just above 448, which becomes 448 as an 8-bit float; NaN stays.  A quotient q of the rounded
// reciprocal, and the exact rest x - q scale, which makes it the rounded quotient: three instructions for the ten of a
// division.  Scales from 2^-100 to 2^100, so that nothing overflows or underflows that counts.
struct Quotient {
  float scale, inverse, most;
  __device__ __forceinline__ explicit Quotient(float s) : scale(s), inverse(1.0f / s), most(s * 448.25f) {}
  __device__ __forceinline__ float operator()(float x) const {
    x = __builtin_elementwise_maximum(__builtin_elementwise_minimum(x, most), -most);
    const float q = x * inverse;
    return __builtin_fmaf(__builtin_fmaf(-q, scale, x), inverse, q);
  }
};

// A thread's unit: two pieces of N elements of a vector (N = 8, or 1 where rows or pairs are not aligned to that), such
// that pairs lie within the unit.  Neighbouring threads have neighbouring pieces, first and second ones, so that each load
// and store takes whole lines: halves pair piece u with that half of the turned elements later, neighbours (of which a
// piece of eight holds four) and elements that stay with that half of theirs later.  Single elements take twice the time:
// 8192 tokens of 32 heads of 96, 24 turned, as halves 34.8 us (2.9 TB/s), as neighbours, whose pairs are in pieces of eight,
// 17.2 (5.8).
template <typename T, int N, bool IL>
struct Unit {
  typedef typename std::conditional<N == 8, typename Vec8<T>::type, T>::type Raw;
  int e0, e1;    // first elements; e1 < 0: no second piece
  bool t0, t1;   // turned

  static int count(int dim, int turned) {
    if (IL) return (dim + 2 * N - 1) / (2 * N);
    return turned / (2 * N) + (dim - turned + 2 * N - 1) / (2 * N);
  }
  __device__ __forceinline__ Unit(int u, int units, int dim, int turned) {
    if (IL && N == 1) {
      e0 = 2 * u;
      e1 = e0 + 1;
      t0 = t1 = e0 < turned;
    } else if (IL) {
      e0 = N * u;
      e1 = N * (u + units);
      t0 = e0 < turned;
      t1 = e1 < turned;
    } else {
      const int pairs = turned / (2 * N);
      t0 = t1 = u < pairs;
      e0 = t0 ? N * u : turned + N * (u - pairs);
      e1 = e0 + (t0 ? turned / 2 : N * (units - pairs));
    }
    if (e1 >= dim) e1 = -1;
  }
  struct Two {
    Raw p[2];
  };
  __device__ __forceinline__ Two load(const T* row) const {
    Two x;
    x.p[0] = *(const Raw*)(row + e0);
    x.p[1] = *(const Raw*)(row + (e1 < 0 ? e0 : e1));
    return x;
  }
  static __device__ __forceinline__ float at(const Two& x, int p, int i) {
    if constexpr (N == 8) return (float)x.p[p][i];
    else return (float)x.p[p];
  }
  // The number of the unit's pair i, where it is turned.
  __device__ __forceinline__ int pair(int i) const {
    if (IL && N == 8) return i < 4 ? e0 / 2 + i : e1 / 2 + i - 4;
    return IL ? e0 / 2 : e0 + i;
  }
  // (c, s) of the unit's pairs out of those of all pairs.
  __device__ __forceinline__ void turns(const float2* cs, float2 (&r)[N]) const {
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = IL && N == 8 && i >= 4 && !t1 ? make_float2(1.0f, 0.0f) : cs[pair(i)];
  }
  // The unit as floats, turned if `turns`; (c, s) of its pairs at cs.
  __device__ __forceinline__ void floats(const Two& x, bool turns, const float2 (&cs)[N], float (&y)[2][N]) const {
#pragma clang fp contract(off)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      y[0][i] = at(x, 0, i);
      y[1][i] = at(x, 1, i);
    }
    if (!turns || !t0) return;
    if constexpr (IL && N == 8) {
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        if (p && !t1) break;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float a = y[p][2 * i], b = y[p][2 * i + 1], c = cs[4 * p + i].x, s = cs[4 * p + i].y;
          y[p][2 * i] = a * c - b * s;
          y[p][2 * i + 1] = b * c + a * s;
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float a = y[0][i], b = y[1][i];
        y[0][i] = a * cs[i].x - b * cs[i].y;
        y[1][i] = b * cs[i].x + a * cs[i].y;
      }
    }
  }
  __device__ __forceinline__ void store(T* row, const float (&y)[2][N]) const {
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int e = p ? e1 : e0;
      if (e < 0) continue;
      if constexpr (N == 8) {
        Raw v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (T)y[p][i];
        *(Raw*)(row + e) = v;
      } else {
        row[e] = (T)y[p][0];
      }
    }
  }
  // by: a value as it is stored, not above 448 but for less than half a step.
  template <typename F>
  __device__ __forceinline__ void store_f8(uint8_t* row, const float (&y)[2][N], F by) const {
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int e = p ? e1 : e0;
      if (e < 0) continue;
      float f[N];
#pragma unroll
      for (int i = 0; i < N; ++i) f[i] = by(y[p][i]);
      if constexpr (N == 8) *(int2*)(row + e) = to_f8(f);
      else row[e] = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[0], 0, false);
    }
  }
};

// i / pairs for rows below 600 and pairs up to 512: the quotient is off by less than 2^-22 of itself, and i + 1/2 is at least
// 1 / (2 pairs) of a row away from the next one.
__device__ __forceinline__ int row_of(int i, int pairs) { return (int)(((float)i + 0.5f) * __builtin_amdgcn_rcpf((float)pairs)); }

constexpr int kThreads = 256;

// How workgroups take the vectors of one kind (queries, keys or values) one by one: `units` units to a vector, of which
// `lanes` threads take one (or several) each; `tokens` tokens and, of each, `heads` heads at a time.
struct Rows {
  int units, lanes, tokens, heads;
  int64_t groups;
};

// -------------------------------------------------------- vectors one by one
//
// A thread keeps its token and its unit, and so the unit's cosines and sines,
// and goes over the heads of one kind.  The workgroup makes each cosine and
// sine of its tokens once.  Bytes bound this: 8494 tokens of 32 heads of 128
// take 28.3 us (4.9 TB/s; a large copy 5.1), 6800 tokens of 32 + 2 * 8 heads,
// keys and values to 8 bits, 34.6 (4.4).
//
// Kinds have workgroups of their own: a loop over all heads of a token needs
// the addresses of three inputs and two outputs, and twice the registers.
//
// s < 0: queries into out; 0, 1: keys or values into their cache.
template <typename T, int N, bool IL, bool CACHE, bool F8>
__device__ __forceinline__ void rows_part(const KvAppendArgs& a, const Rows& w, int64_t group, int s, float2* cs) {
  typedef Unit<T, N, IL> U;
  const int tid = threadIdx.x, turned = s == 1 ? 0 : a.turned, pairs = turned / 2;
  const int r = tid / w.lanes, tl = r / w.heads, h0 = r - tl * w.heads, heads = CACHE ? a.num_kv_heads : a.num_heads;
  const int64_t first = group * w.tokens, t = first + tl;
  bool live = tl < w.tokens && t < a.num_tokens;
  if (live && a.turned) live = a.positions[t] >= 0;
  const T* src;
  char* to;
  int64_t src_step, to_step;  // from head to head: elements, bytes
  if (CACHE) {
    const int64_t slot = live ? a.slots[t] : -1;
    live = live && slot >= 0 && slot < a.num_slots;
    const int64_t block = slot >> a.block_shift, at = slot & ((1 << a.block_shift) - 1);
    const int size = F8 ? 1 : 2;
    src = (const T*)(s ? a.src[1] : a.src[0]) + t * (s ? a.token_stride[1] : a.token_stride[0]);
    src_step = s ? a.head_stride[1] : a.head_stride[0];
    to_step = ((int64_t)a.head_dim << a.block_shift) * size;
    to = (char*)(s ? a.cache[1] : a.cache[0]) + block * heads * to_step + at * a.head_dim * size;
  } else {
    src = (const T*)a.q + t * a.q_token_stride;
    src_step = a.q_head_stride;
    to = (char*)a.out + t * a.out_token_stride * 2;
    to_step = a.out_head_stride * 2;
  }
  const Quotient quotient(s == 1 ? a.scale[1] : a.scale[0]);
  for (int u0 = 0; u0 < w.units; u0 += w.lanes) {  // once, but for long vectors of single elements
    const int u = u0 + tid % w.lanes;
    const U unit(u, w.units, a.head_dim, turned);
    const bool mine = live && u < w.units;
    typename U::Two x = {}, next = {};
    int h = h0;
    if (mine && h < heads) x = unit.load(src + h * src_step);  // on its way meanwhile
    if (u0 == 0 && pairs) {
#pragma unroll 1
      for (int i = tid; i < w.tokens * pairs; i += kThreads) {
        const int row = row_of(i, pairs);
        if (first + row < a.num_tokens)
          cs[i] = turn_of((double)a.positions[first + row] * a.freqs[i - row * pairs], a.magnitude, a.reverse);
      }
      __syncthreads();
    }
    if (!mine) continue;
    float2 turn[N];
    if (unit.t0) unit.turns(cs + tl * pairs, turn);
    for (; h < heads; h += w.heads) {
      if (h + w.heads < heads) next = unit.load(src + (h + w.heads) * src_step);
      float y[2][N];
      unit.floats(x, true, turn, y);
      if (F8) unit.store_f8((uint8_t*)to + h * to_step, y, quotient);
      else unit.store((T*)(to + h * to_step), y);
      x = next;
    }
  }
}

// --------------------------------------------------- blocks with own scales
//
// A scale is a power of two, the smallest E with 448 E no less than any value
// that the block holds of a head: 8-bit floats lose nothing by it but a range of
// two, and where a scale has to grow the values stored before stay what they
// are, unless they fall below the format's normal range.  A block that has
// values already (its first new slot is not its first) keeps its scale if that
// suffices.
//
// The tokens of one block are rows in a row: a run, at most a block's.  A
// workgroup owns the runs that begin among its tokens; it makes their cosines
// and sines once, and then every wave takes one head of the keys or values of a
// run (or several heads where the run is short): largest value, scale, values.
// The rows are read twice, the second time from the L2; kept in registers they
// spill (46,000 tokens of 15 + 2 * 5 heads of 64: 140 us, so 122 at that time).
// Vector instructions bound this beside the bytes: those 46,000 tokens take 67.8
// us, 3.9 TB/s and 26 million instructions of waves, two thirds of the time; 8192
// tokens of 32 + 2 * 8 heads of 128 into blocks of 16 35.1 (5.3 TB/s).
struct Runs {
  int units, lanes;  // of a vector; lanes: a power of two, 64 at most
  int tokens;        // of a workgroup, 32 at most
  int split;         // workgroups that share these tokens' heads
  int chunks, groups;
};

// The exponent of the smallest power of two E with x <= 448 E, 448 = 1.75 * 2^8, from -64 to 64.
__device__ __forceinline__ int exponent_for(float x) {
  const uint32_t b = __float_as_uint(x);
  const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffff) > 0x600000);
  return e < -64 ? -64 : e > 64 ? 64 : e;  // that of 0 and of the smallest floats, too
}

// One head of a run's keys or values.
template <typename T>
struct Task {
  bool mine, turns;
  const T* row;  // of the run's first token
  int64_t step;
  uint8_t* to;  // the block's first value
  float* scale;

  __device__ __forceinline__ Task(const KvAppendArgs& a, int task, int64_t t, int64_t block) {
    const int s = task >= a.num_kv_heads, h = task - (s ? a.num_kv_heads : 0);
    mine = task < 2 * a.num_kv_heads;
    turns = !s && a.turned > 0;
    step = s ? a.token_stride[1] : a.token_stride[0];
    row = (const T*)(s ? a.src[1] : a.src[0]) + t * step + h * (s ? a.head_stride[1] : a.head_stride[0]);
    const int64_t at = block * a.num_kv_heads + h;
    to = (uint8_t*)(s ? a.cache[1] : a.cache[0]) + (at << a.block_shift) * a.head_dim;
    scale = (s ? a.scales[1] : a.scales[0]) + at;
  }
};

// The eight-bit numbers from `at` on, n of them, times `by`; lane `lane` of `lanes`.
__device__ __forceinline__ void scale_again(uint8_t* at, int64_t n, float by, int lane, int lanes) {
#pragma unroll 1
  for (int64_t i = lane * 8; i < n; i += lanes * 8) {
    const int2 v = *(const int2*)(at + i);
    float f[8];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int p = j ? v.y : v.x;
      f[4 * j] = by * __builtin_amdgcn_cvt_f32_fp8(p, 0);
      f[4 * j + 1] = by * __builtin_amdgcn_cvt_f32_fp8(p, 1);
      f[4 * j + 2] = by * __builtin_amdgcn_cvt_f32_fp8(p, 2);
      f[4 * j + 3] = by * __builtin_amdgcn_cvt_f32_fp8(p, 3);
    }
    *(int2*)(at + i) = to_f8(f);
  }
}

// Some heads of the run of n tokens from t on, whose first slot is `slot`; `task`: this lane's, of all heads' keys and then
// values.  A head has `span` lanes, `lanes` for the units of each of its rows, or, with a team, those of all waves; cs:
// cosines and sines of the run's tokens; tops: a float for each wave.
template <typename T, int N, bool IL, bool IN_LDS>
__device__ __forceinline__ void store_heads(const KvAppendArgs& a, const Runs& w, int task, int span, bool team, int64_t t, int64_t slot,
                                            int n, const float2* cs, float* tops) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, pairs = a.turned / 2, bs = 1 << a.block_shift;
  const int in = (lane & (span - 1)) + (team ? wave * span : 0), lanes = team ? span * (kThreads / 64) : span;  // of the head
  const int begin = (int)(slot & (bs - 1));  // values before this one are in the block already
  const Task<T> k(a, task, t, slot >> a.block_shift);
  const int rows = lanes / w.lanes, r0 = in / w.lanes, u0 = in & (w.lanes - 1);
  const int last = r0 < n ? r0 + (n - 1 - r0) / rows * rows : -1;  // of the lane's rows
  const float old = k.mine && begin ? *k.scale : 0.0f;
  const auto turned = [&](const Unit<T, N, IL>& unit, const typename Unit<T, N, IL>::Two& x, int r, float (&y)[2][N]) {
    float2 turn[N];
    if (k.turns && unit.t0) {
      if constexpr (IN_LDS) {
        unit.turns(cs + r * pairs, turn);
      } else {
        const double at = (double)a.positions[t + r];
#pragma unroll 1
        for (int i = 0; i < N; ++i) {
          const int pair = unit.pair(i);
          turn[i] = pair < pairs ? turn_of(at * a.freqs[pair], a.magnitude, false) : make_float2(1.0f, 0.0f);
        }
      }
    }
    unit.floats(x, k.turns, turn, y);
  };
  typedef Unit<T, N, IL> U;
  const bool one = w.units <= w.lanes;
  float y[2][N] = {};  // the last ones are kept, and the first ones stored
  const auto read = [&](const U& unit, int r) { turned(unit, unit.load(k.row + r * k.step), r, y); };
  // The largest value, in magnitude, without NaN; without infinities, too, where there are any: these are limited when
  // stored, and NaN is kept.
  const auto largest = [&](auto finite) {
    float top = 0.0f;
    if (!k.mine) return top;
#pragma unroll 1
    for (int r = r0; r < n; r += rows)
#pragma unroll 1
      for (int u = u0; u < w.units; u += w.lanes) {
        const U unit(u, w.units, a.head_dim, a.turned);
        read(unit, r);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float p = __builtin_fabsf(y[0][i]), q = unit.e1 >= 0 ? __builtin_fabsf(y[1][i]) : 0.0f;
          if (decltype(finite)::value) top = fmaxf(top, fmaxf(p < INFINITY ? p : 0.0f, q < INFINITY ? q : 0.0f));
          else top = fmaxf(top, fmaxf(p, q));
        }
      }
    return top;
  };
  float top = largest(std::false_type{});
  bool simple = top < INFINITY;  // none of the lane's values has to be limited
  if (__builtin_amdgcn_ballot_w64(!simple)) top = largest(std::true_type{});
  for (int o = 1; o < span; o *= 2) top = fmaxf(top, __shfl_xor(top, o));
  if (team) {  // every wave has read the old scale before one writes the new one
    __syncthreads();
    if (lane == 0) tops[wave] = top;
    __syncthreads();
#pragma unroll
    for (int v = 0; v < kThreads / 64; ++v) top = fmaxf(top, tops[v]);
  }
  float scale = __uint_as_float((uint32_t)(exponent_for(top) + 127) << 23);
  const bool before = old >= 0x1p-64f && old <= 0x1p64f, grows = before && scale > old;
  if (before && !grows) scale = old;
  if (!k.mine) return;
  if (in == 0) *k.scale = scale;
  if (grows) scale_again(k.to, (int64_t)begin * a.head_dim, old / scale, in, lanes);
  // All values are within the scale, which is a power of two, as a rule: a product then.
  simple = simple && (__float_as_uint(scale) & 0x7fffffu) == 0 && top <= 448.0f * scale;
  const bool products = __builtin_amdgcn_ballot_w64(!simple) == 0;
  const float inverse = 1.0f / scale;
  const Quotient quotient(scale);
#pragma unroll 1
  for (int r = last; r >= 0; r -= rows)
#pragma unroll 1
    for (int u = u0; u < w.units; u += w.lanes) {
      const U unit(u, w.units, a.head_dim, a.turned);
      if (!one || r != last) read(unit, r);
      uint8_t* to = k.to + (a.slots[t + r] & (bs - 1)) * a.head_dim;
      if (products) unit.store_f8(to, y, [&](float x) { return x * inverse; });
      else unit.store_f8(to, y, quotient);
    }
}

// IN_LDS: the cosines and sines of a workgroup's runs fit the LDS.
template <typename T, int N, bool IL, bool IN_LDS>
__device__ __forceinline__ void runs_part(const KvAppendArgs& a, const Runs& w, int64_t group, float2* cs, float* tops) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, pairs = a.turned / 2, bs = 1 << a.block_shift;
  // Workgroups go to the eight dies in turn: each die gets tokens next to each other, so that runs which begin at every
  // second, fourth, ... workgroup's tokens are spread over the dies.
  const int per = (w.chunks + 7) / 8, part = (int)group / (8 * per), at = (int)group % (8 * per), chunk = at % 8 * per + at / 8;
  if (chunk >= w.chunks) return;
  const int64_t first = (int64_t)chunk * w.tokens;
  const auto slot_of = [&](int64_t t) -> int64_t {  // -1: not stored
    if (t < 0 || t >= a.num_tokens) return -1;
    const int64_t slot = a.slots[t];
    return slot < 0 || slot >= a.num_slots || (a.turned && a.positions[t] < 0) ? -1 : slot;
  };
  // A lane looks at token first + lane.  A run begins where a token is not of the block of the one before, and ends where
  // the next does (or a block's rows after).
  const int64_t mine = slot_of(first + lane), before = slot_of(first - 1);
  const int64_t block = mine < 0 ? -1 : mine >> a.block_shift;
  int64_t prev = __shfl_up(block, 1);
  if (lane == 0) prev = before < 0 ? -1 : before >> a.block_shift;
  const uint64_t starts = __builtin_amdgcn_ballot_w64(block != prev);
  const bool begins = lane < w.tokens && block >= 0 && block != prev;
  const uint64_t runs = __builtin_amdgcn_ballot_w64(begins);
  if (!runs) return;
  const uint64_t next = lane < 63 ? starts >> lane >> 1 : 0;
  int n = next ? __builtin_ctzll(next) + 1 : 64 - lane;  // rows of the run that begins here
  const int last = 63 - __builtin_clzll(runs);
  if (!(starts >> last >> 1)) {  // the last run goes on past what the lanes see
    const int64_t b = __shfl(block, last);
    int more = 64 - last;
    while (more < bs) {
      const int64_t s = slot_of(first + last + more + lane);
      const uint64_t out = __builtin_amdgcn_ballot_w64(s < 0 || s >> a.block_shift != b);
      more += out ? __builtin_ctzll(out) : 64;
      if (out) break;
    }
    if (lane == last) n = more;
  }
  n = min(n, bs);
  // A run is items, each of one or several heads: keys', then values'.  This workgroup takes its part of all items.
  const int tasks = 2 * a.num_kv_heads;
  int span = w.lanes;
  while (span < 64 && span < w.lanes * n) span *= 2;
  const int count = begins ? (tasks * span + 63) / 64 : 0;
  int upto = count;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const int x = __shfl_up(upto, o);
    if (lane >= o) upto += x;
  }
  const int base = upto - count, items = __shfl(upto, 63), lo = part * items / w.split, hi = (part + 1) * items / w.split;
  if (lo >= hi) return;
  // The tokens whose cosines and sines it needs: those of the runs whose keys it has.
  int from = 0;
  if (IN_LDS && pairs) {
    const uint64_t keys = __builtin_amdgcn_ballot_w64(begins && base < hi && base + (a.num_kv_heads * span + 63) / 64 > lo);
    if (keys) {
      const int end = 63 - __builtin_clzll(keys);
      from = __builtin_ctzll(keys);
      const int to = end + __shfl(n, end);
#pragma unroll 1
      for (int i = threadIdx.x; i < (to - from) * pairs; i += kThreads) {
        const int row = row_of(i, pairs);
        cs[i] = turn_of((double)a.positions[first + from + row] * a.freqs[i - row * pairs], a.magnitude, false);
      }
    }
    __syncthreads();
  }
  // All waves work together on items where one would go over more than eight rows of a lane.
  const bool large = begins && n * w.lanes > 8 * 64, some = __builtin_amdgcn_ballot_w64(large) != 0;
#pragma unroll 1
  for (int item = some ? lo : lo + wave; item < hi; item += some ? 1 : kThreads / 64) {
    const int i = 63 - __builtin_clzll(__builtin_amdgcn_ballot_w64(begins && base <= item));
    const bool team = __shfl(large, i);
    if (some && !team && (item & (kThreads / 64 - 1)) != wave) continue;
    const int s = __shfl(span, i);
    store_heads<T, N, IL, IN_LDS>(a, w, (item - __shfl(base, i)) * (64 / s) + lane / s, s, team, first + i, __shfl(mine, i), __shfl(n, i),
                                  cs + (i - from) * pairs, tops);
  }
}

constexpr int kTops = kThreads / 64 * 4;  // bytes of the waves' largest values, in front of cosines and sines
enum Storage { kAsIs, kOneScale, kScales, kScalesWide };  // wide: without the cosines and sines of a block's tokens in LDS
struct Plan {
  Rows q, k, v;
  Runs runs;
};
// Waves per SIMD that the registers are to suffice for: one more would put some of them into memory, which costs 1.3 to 2.2
// times the time.
template <Storage S>
constexpr int kWavesPerSimd = S >= kScales ? 4 : 5;
template <typename T, int N, bool IL, Storage S>
__global__ __launch_bounds__(kThreads, kWavesPerSimd<S>) void append_kernel(KvAppendArgs a, Plan p) {
  extern __shared__ float2 cs[];
  int64_t group = blockIdx.x;
  if constexpr (S >= kScales) {
    if (group < p.runs.groups) {
      runs_part<T, N, IL, S == kScales>(a, p.runs, group, cs + kTops / 8, (float*)cs);
      return;
    }
    group -= p.runs.groups;
  } else {
    if (group < p.k.groups + p.v.groups) {
      const int s = group >= p.k.groups;
      rows_part<T, N, IL, true, S == kOneScale>(a, s ? p.v : p.k, group - (s ? p.k.groups : 0), s, cs);
      return;
    }
    group -= p.k.groups + p.v.groups;
  }
  rows_part<T, N, IL, false, false>(a, p.q, group, -1, cs);
}

int power_of_two(int x) {
  int p = 1;
  while (p < x) p *= 2;
  return p;
}

// How `vectors` of `units` units of every token are taken: the tokens and heads at a time with the shortest time, which goes
// with the heads after each other (and one for the start) and the workgroups that do not fit at once.  4137 tokens of 12
// heads of 192: three after each other in 828 workgroups 8.3 us, two in 1379 9.7, one in 4137 12.0; 12,518 of 24 of 64: three
// in 1565 13.4, six in 783 15.0, two in 3130 15.2; 64 tokens of 40 of 128: two 4.5, ten 7.1.
Rows rows_for(int units, int vectors, int64_t tokens) {
  Rows r{};
  r.units = units;
  r.lanes = std::min(units, kThreads);
  r.tokens = r.heads = 1;
  if (vectors == 0) return r;
  const int per = kThreads / r.lanes;
  double least = 0;
  for (int h = std::min(vectors, per); h >= 1; --h) {
    const int t = std::min(16, per / h), turns = (vectors + h - 1) / h;
    const int64_t groups = (tokens + t - 1) / t;
    const double time = (turns + 1) * std::max(0.8, (double)groups / (kWavesPerSimd<kAsIs> * 256));
    if (r.groups == 0 || time < least) {
      least = time;
      r.tokens = t;
      r.heads = h;
      r.groups = groups;
    }
  }
  return r;
}

constexpr int kLdsBytes = 160 * 1024;

template <typename T, int N, bool IL>
int append_launch(const KvAppendArgs& a, bool f8, hipStream_t s) {
  const bool blocks = a.scales[0] != nullptr;
  const int pairs = a.turned / 2;
  Plan p{};
  p.q = rows_for(Unit<T, N, IL>::count(a.head_dim, a.turned), a.num_heads, a.num_tokens);
  int64_t lds;
  bool wide = false;
  if (blocks) {
    p.runs.units = Unit<T, N, IL>::count(a.head_dim, a.turned);
    p.runs.lanes = std::min(64, power_of_two(p.runs.units));
    // As many tokens as a block has, so that one workgroup has all of a block's heads at hand; 32 where workgroups abound and
    // cosines are made for a block's tokens only once more: in us, with blocks of 8, 15 + 2 * 5 heads of 64, 8192 tokens 15.1
    // (14.3 with 32), 16,384 26.2 (22.9), 32,767 48.4 (39.4); 32 + 2 * 8 of 128 37.3 (36.9), 90.9 (87.9), 175 (161); blocks of 16,
    // 16 + 2 * 16 of 128 33.9 (35.0), 80.0 (80.0), 24,576 128 (133), 32,767 157 (157).  Eight with blocks of 32 take 1.5 times as
    // long, and 32 with single tokens in blocks of 16 of one head 1.7 times.
    p.runs.tokens = a.num_tokens >= 32768 ? 32 : std::min(std::max(1 << a.block_shift, 8), 32);
    const auto bytes = [&] { return kTops + ((int64_t)p.runs.tokens + (1 << a.block_shift) - 1) * pairs * 8; };
    while (p.runs.tokens > 1 && bytes() > kLdsBytes) p.runs.tokens /= 2;
    // Workgroups that share a chunk's heads: until there are 1024, but each with items for all waves, whose number depends on
    // whether the chunk is single tokens or whole blocks: enough for either with few tokens, for both with many.  In us, with
    // as many as either allows (and both): 15 + 2 * 5 heads of 64, blocks of 8, 64 tokens 5.9 (7.9), 1024 6.3 (8.3), 3000 8.3
    // (9.8); 32 + 2 * 8 of 128, blocks of 16, 1024 9.1 (9.9), 2048 12.4 (11.0), 3000 16.8 (15.7); of 32, 1024 11.7 (12.6), 2048
    // 17.8 (14.4), 3000 20.0 (15.9); single tokens, blocks of 32, 1024 8.6 (14.4), 2048 13.4 (15.8).  512, 1024, 2048
    // workgroups: 2049 tokens into blocks of 8 17.7, 13.6, 13.4; 4096 19.9, 21.0, 23.5; 8192 of 15 + 2 * 5 heads 14.3, 14.7, 17.4.
    const int singles = p.runs.tokens * 2 * a.num_kv_heads * p.runs.lanes / kThreads;
    const int whole = std::max(1, p.runs.tokens >> a.block_shift) * 2 * a.num_kv_heads / (kThreads / 64);
    const int most = std::max(1, a.num_tokens <= 2048 ? std::max(singles, whole) : std::min(singles, whole));
    p.runs.split = (int)std::min<int64_t>(most, std::max<int64_t>(1, 1024 * p.runs.tokens / a.num_tokens));
    lds = bytes();
    wide = lds > kLdsBytes;
    if (wide) lds = kTops;
    p.runs.chunks = (int)((a.num_tokens + p.runs.tokens - 1) / p.runs.tokens);
    const int64_t all = (int64_t)((p.runs.chunks + 7) / 8) * 8 * p.runs.split;
    if (all > 0xffffff) return fail_static(SCOOT_ERR_UNSUPPORTED, "kv append: too many tokens for one call");
    p.runs.groups = (int)all;
  } else {
    p.k = rows_for(Unit<T, N, IL>::count(a.head_dim, a.turned), a.num_kv_heads, a.num_tokens);
    p.v = rows_for(Unit<T, N, IL>::count(a.head_dim, 0), a.num_kv_heads, a.num_tokens);
    lds = (int64_t)p.k.tokens * pairs * 8;
  }
  lds = std::max(lds, (int64_t)p.q.tokens * pairs * 8);
  const int64_t groups = p.q.groups + p.k.groups + p.v.groups + p.runs.groups;
  if (groups * kThreads > 0xffffffffLL) return fail_static(SCOOT_ERR_UNSUPPORTED, "kv append: too many tokens for one call");
  const auto go = [&](auto kernel) {
    if (lds > 64 * 1024) {
      const int rc = allow_full_lds((const void*)kernel, "kv append");
      if (rc != SCOOT_OK) return rc;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(kThreads), (size_t)lds, s, a, p);
    return launched("kv append launch");
  };
  if (blocks) return wide ? go(append_kernel<T, N, IL, kScalesWide>) : go(append_kernel<T, N, IL, kScales>);
  return f8 ? go(append_kernel<T, N, IL, kOneScale>) : go(append_kernel<T, N, IL, kAsIs>);
}

template <typename T>
int append_typed(const KvAppendArgs& a, bool f8, hipStream_t s) {
  // Pieces of eight elements: every row starts on 16 bytes, and a piece's pairs are in one or two pieces.
  bool eight = a.turned % (a.interleaved ? 8 : 16) == 0;
  if (a.num_heads)
    eight = eight && (((uintptr_t)a.q | (uintptr_t)a.out) & 15) == 0 &&
            ((a.q_token_stride | a.q_head_stride | a.out_token_stride | a.out_head_stride) & 7) == 0;
  if (a.num_kv_heads)
    for (int i = 0; i < 2; ++i)
      eight = eight && ((uintptr_t)a.src[i] & 15) == 0 && ((a.token_stride[i] | a.head_stride[i]) & 7) == 0;
  if (a.interleaved) return eight ? append_launch<T, 8, true>(a, f8, s) : append_launch<T, 1, true>(a, f8, s);
  return eight ? append_launch<T, 8, false>(a, f8, s) : append_launch<T, 1, false>(a, f8, s);
}

}  // namespace

int launch_kv_append(const KvAppendArgs& a, scoot_kv_type type, scoot_kv_type cache_type, void* stream) {
  const bool f8 = cache_type == SCOOT_KV_F8;
  return type == SCOOT_KV_F16 ? append_typed<_Float16>(a, f8, (hipStream_t)stream) : append_typed<__bf16>(a, f8, (hipStream_t)stream);
}

}  // namespace scoot
