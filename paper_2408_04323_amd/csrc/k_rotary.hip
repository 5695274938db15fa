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

// cos and sin of x in double: x less the nearest multiple n of pi / 2, which is taken away in two parts (exact but for
// 2^-53 of the rest, as fma rounds once), and the Taylor series up to pi / 4, whose next terms are below 2^-54.
__device__ __forceinline__ float2 turn_of(double x, double magnitude, bool reverse) {
  const double n = __builtin_rint(x * 0.63661977236758134308);
  double r = __builtin_fma(-n, 1.57079632679489655800, x);
  r = __builtin_fma(-n, 6.12323399573676603587e-17, r);
  const double z = r * r;
  double s = -1.0 / 1307674368000.0;  // 15!
  s = __builtin_fma(s, z, 1.0 / 6227020800.0);
  s = __builtin_fma(s, z, -1.0 / 39916800.0);
  s = __builtin_fma(s, z, 1.0 / 362880.0);
  s = __builtin_fma(s, z, -1.0 / 5040.0);
  s = __builtin_fma(s, z, 1.0 / 120.0);
  s = __builtin_fma(s, z, -1.0 / 6.0);
  s = __builtin_fma(s * z, r, r);
  double c = 1.0 / 20922789888000.0;  // 16!
  c = __builtin_fma(c, z, -1.0 / 87178291200.0);
  c = __builtin_fma(c, z, 1.0 / 479001600.0);
  c = __builtin_fma(c, z, -1.0 / 3628800.0);
  c = __builtin_fma(c, z, 1.0 / 40320.0);
  c = __builtin_fma(c, z, -1.0 / 720.0);
  c = __builtin_fma(c, z, 1.0 / 24.0);
  c = __builtin_fma(c, z, -0.5);
  c = __builtin_fma(c, z, 1.0);
  const int quarter = (int)(n - 4.0 * __builtin_floor(n * 0.25));
  double cx = quarter & 1 ? s : c, sx = quarter & 1 ? c : s;
  if (quarter == 1 || quarter == 2) cx = -cx;
  if ((quarter >= 2) != reverse) sx = -sx;
  return make_float2((float)(cx * magnitude), (float)(sx * magnitude));
}

// A thread's unit: two pieces of N elements of a vector (N = 8, or 1 where rows or pairs are not aligned to that), such
// that pairs lie within the unit: the pairs N u .. N u + N - 1 in either layout.
template <typename T, int N, bool IL>
struct Unit {
  typedef typename std::conditional<N == 8, typename Vec8<T>::type, T>::type Raw;
  int e0, e1;  // first elements; e1 < 0: no second piece
  bool t0, t1; // turned

  __device__ __forceinline__ Unit(int u, int dim, int turned) {
    if (IL) {
      e0 = 2 * N * u;
      e1 = e0 + N;
      t0 = e0 < turned;
      t1 = e1 < turned || (N == 1 && t0);
    } else {
      const int pairs = turned / (2 * N);
      t0 = t1 = u < pairs;
      e0 = t0 ? N * u : turned + 2 * N * (u - pairs);
      e1 = t0 ? e0 + turned / 2 : e0 + N;
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
  __device__ __forceinline__ void store_f8(uint8_t* row, const float (&y)[2][N], float scale) const {
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int e = p ? e1 : e0;
      if (e < 0) continue;
      float f[N];
#pragma unroll
      for (int i = 0; i < N; ++i) f[i] = limit_f8(y[p][i], scale);
      if constexpr (N == 8) *(int2*)(row + e) = to_f8(f);
      else row[e] = (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[0], 0, false);
    }
  }
};

// (c, s) of a unit's pairs; those past the last pair belong to pieces that stay.
template <int N>
__device__ __forceinline__ void pairs_of(const float2* cs, int u, int pairs, float2 (&r)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) r[i] = N * u + i < pairs ? cs[N * u + i] : make_float2(1.0f, 0.0f);
}

constexpr int kThreads = 256;

// How workgroups take vectors one by one: `units` units to a vector, of which `lanes` threads take one (or several) each;
// `tokens` tokens and, of each, `heads` heads at a time.
struct Rows {
  int units, lanes, tokens, heads;
  int64_t groups;
};

// -------------------------------------------------------- vectors one by one
//
// A thread keeps its token and its unit, and so the unit's cosines and sines,
// and goes over the heads: queries, then keys, then values.  The workgroup
// makes each cosine and sine of its tokens once.
template <typename T, int N, bool IL, bool F8>
__device__ __forceinline__ void rows_part(const KvAppendArgs& a, const Rows& w, int64_t group, int kv_heads, float2* cs) {
  const int tid = threadIdx.x, pairs = a.turned / 2;
  const int r = tid / w.lanes, tl = r / w.heads, h0 = r % w.heads, rows = a.num_heads + 2 * kv_heads;
  const int64_t first = group * w.tokens, t = first + tl;
  bool live = tl < w.tokens && t < a.num_tokens;
  if (live && pairs) live = a.positions[t] >= 0;
  int64_t slot = -1;
  if (live && kv_heads) {
    slot = a.slots[t];
    if (slot >= a.num_slots) slot = -1;
  }
  const int most = slot >= 0 ? rows : a.num_heads;  // without a slot only queries
  const int64_t block = slot >> a.block_shift, at = slot & ((1 << a.block_shift) - 1);
  const auto source = [&](int h) {
    if (h < a.num_heads) return (const T*)a.q + t * a.q_token_stride + h * a.q_head_stride;
    const int s = h >= a.num_heads + kv_heads, g = h - a.num_heads - (s ? kv_heads : 0);
    return (const T*)(s ? a.src[1] : a.src[0]) + t * (s ? a.token_stride[1] : a.token_stride[0]) +
           g * (s ? a.head_stride[1] : a.head_stride[0]);
  };
  for (int u0 = 0; u0 < w.units; u0 += w.lanes) {  // once, but for long vectors of single elements
    const int u = u0 + tid % w.lanes;
    const Unit<T, N, IL> unit(u, a.head_dim, a.turned);
    const bool mine = live && u < w.units;
    typename Unit<T, N, IL>::Two x = {}, next = {};
    int h = h0;
    if (mine && h < most) x = unit.load(source(h));  // on its way meanwhile
    if (u0 == 0) {
      for (int i = tid; i < w.tokens * pairs; i += kThreads) {
        const int64_t ti = first + i / pairs;
        if (ti < a.num_tokens) cs[i] = turn_of((double)a.positions[ti] * a.freqs[i % pairs], a.magnitude, a.reverse);
      }
      __syncthreads();
    }
    if (!mine) continue;
    float2 turn[N];
    pairs_of<N>(cs + tl * pairs, u, pairs, turn);
    for (; h < most; h += w.heads) {
      if (h + w.heads < most) next = unit.load(source(h + w.heads));
      float y[2][N];
      unit.floats(x, h < a.num_heads + kv_heads, turn, y);
      if (h < a.num_heads) {
        unit.store((T*)a.out + t * a.out_token_stride + h * a.out_head_stride, y);
      } else {
        const int s = h >= a.num_heads + kv_heads, g = h - a.num_heads - (s ? kv_heads : 0);
        const int64_t to = (((block * kv_heads + g) << a.block_shift) + at) * a.head_dim;
        if (F8) unit.store_f8((uint8_t*)(s ? a.cache[1] : a.cache[0]) + to, y, s ? a.scale[1] : a.scale[0]);
        else unit.store((T*)(s ? a.cache[1] : a.cache[0]) + to, y);
      }
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
// The tokens of one block are rows in a row: a run, at most a block's.  The
// workgroup that owns a run's first token takes all of it, a wave one head of
// the keys or of the values (or several heads where the run is short): largest
// value, scale, then the values, which stay in registers in between if they are
// few.
struct Runs {
  int units, lanes;   // of a vector; lanes: a power of two, 64 at most
  int tokens, split;  // tokens of a workgroup, workgroups that share their heads
  int in_lds;         // rows whose cosines and sines fit the LDS: all of a block's, or none
  int64_t groups;
};
constexpr int kHeld = 4;  // units of a lane that stay in registers

// The exponent of the smallest power of two E with x <= 448 E, 448 = 1.75 * 2^8, from -64 to 64.
__device__ __forceinline__ int exponent_for(float x) {
  const uint32_t b = __float_as_uint(x);
  const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffff) > 0x600000);
  return e < -64 ? -64 : e > 64 ? 64 : e;  // that of 0 and of the smallest floats, too
}

template <typename T, int N, bool IL>
__device__ __forceinline__ void run_part(const KvAppendArgs& a, const Runs& w, int part, int64_t t, int64_t slot, int n, float2* cs) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, pairs = a.turned / 2, bs = 1 << a.block_shift;
  const int64_t block = slot >> a.block_shift;
  const int begin = (int)(slot & (bs - 1));  // values before this one are in the block already
  __syncthreads();
  if (w.in_lds)
    for (int i = threadIdx.x; i < n * pairs; i += kThreads)
      cs[i] = turn_of((double)a.positions[t + i / pairs] * a.freqs[i % pairs], a.magnitude, false);
  __syncthreads();
  // Lanes: `lanes` for the units, then rows, then heads.
  const int slots = 64 / w.lanes;
  int rows = 1;
  while (rows < slots && rows < n) rows *= 2;
  const int heads = slots / rows, span = w.lanes * rows;
  const int u0 = lane & (w.lanes - 1), r0 = lane / w.lanes & (rows - 1), tasks = 2 * a.num_kv_heads;
  const bool held = w.units <= w.lanes && n <= kHeld * rows;
  for (int g = (part * (kThreads / 64) + wave) * heads; g < tasks; g += w.split * (kThreads / 64) * heads) {
    const int task = g + lane / span;
    const bool mine = task < tasks;
    const int s = task >= a.num_kv_heads, h = task - (s ? a.num_kv_heads : 0);
    const T* src = (const T*)(s ? a.src[1] : a.src[0]) + h * (s ? a.head_stride[1] : a.head_stride[0]);
    const int64_t step = s ? a.token_stride[1] : a.token_stride[0];
    uint8_t* to = (uint8_t*)(s ? a.cache[1] : a.cache[0]) + ((block * a.num_kv_heads + h) << a.block_shift) * a.head_dim;
    float* scale_at = (s ? a.scales[1] : a.scales[0]) + block * a.num_kv_heads + h;
    const float old = mine && begin ? *scale_at : 0.0f;
    const auto turned = [&](const Unit<T, N, IL>& unit, const typename Unit<T, N, IL>::Two& x, int r, int u, float (&y)[2][N]) {
      float2 turn[N];
      if (w.in_lds) {
        pairs_of<N>(cs + r * pairs, u, s ? 0 : pairs, turn);
      } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
          turn[i] = !s && N * u + i < pairs ? turn_of((double)a.positions[t + r] * a.freqs[N * u + i], a.magnitude, false) : make_float2(1.0f, 0.0f);
      }
      unit.floats(x, !s, turn, y);
    };
    float top = 0.0f;
    const auto largest = [&](const Unit<T, N, IL>& unit, const float (&y)[2][N]) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float p = __builtin_fabsf(y[0][i]), q = __builtin_fabsf(y[1][i]);
        top = p < INFINITY ? fmaxf(top, p) : top;  // infinities are limited when stored, NaN is kept
        top = unit.e1 >= 0 && q < INFINITY ? fmaxf(top, q) : top;
      }
    };
    typename Unit<T, N, IL>::Two x[kHeld] = {};
    const Unit<T, N, IL> one(u0, a.head_dim, a.turned);
    if (held) {
      const bool in = mine && u0 < w.units;
#pragma unroll
      for (int i = 0; i < kHeld; ++i)
        if (in && r0 + i * rows < n) x[i] = one.load(src + (t + r0 + i * rows) * step);
#pragma unroll
      for (int i = 0; i < kHeld; ++i) {
        if (!(in && r0 + i * rows < n)) continue;
        float y[2][N];
        turned(one, x[i], r0 + i * rows, u0, y);
        largest(one, y);
      }
    } else if (mine) {
      for (int r = r0; r < n; r += rows)
        for (int u = u0; u < w.units; u += w.lanes) {
          const Unit<T, N, IL> unit(u, a.head_dim, a.turned);
          float y[2][N];
          turned(unit, unit.load(src + (t + r) * step), r, u, y);
          largest(unit, y);
        }
    }
    for (int o = 1; o < span; o *= 2) top = fmaxf(top, __shfl_xor(top, o));
    float scale = __uint_as_float((uint32_t)(exponent_for(top) + 127) << 23);
    const bool before = old > 0.0f && old < INFINITY, grows = before && scale > old;
    if (before && !grows) scale = old;
    if (mine && lane % span == 0) *scale_at = scale;
    if (mine && grows) {
      const float by = old / scale;
      for (int64_t i = (int64_t)(lane % span) * 8; i < (int64_t)begin * a.head_dim; i += span * 8) {
        const int2 v = *(const int2*)(to + i);
        float f[8];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int p = j ? v.y : v.x;
          f[4 * j] = __builtin_amdgcn_cvt_f32_fp8(p, 0);
          f[4 * j + 1] = __builtin_amdgcn_cvt_f32_fp8(p, 1);
          f[4 * j + 2] = __builtin_amdgcn_cvt_f32_fp8(p, 2);
          f[4 * j + 3] = __builtin_amdgcn_cvt_f32_fp8(p, 3);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] *= by;
        *(int2*)(to + i) = to_f8(f);
      }
    }
    if (held) {
      const bool in = mine && u0 < w.units;
#pragma unroll
      for (int i = 0; i < kHeld; ++i) {
        const int r = r0 + i * rows;
        if (!(in && r < n)) continue;
        float y[2][N];
        turned(one, x[i], r, u0, y);
        one.store_f8(to + (a.slots[t + r] & (bs - 1)) * a.head_dim, y, scale);
      }
    } else if (mine) {
      for (int r = r0; r < n; r += rows)
        for (int u = u0; u < w.units; u += w.lanes) {
          const Unit<T, N, IL> unit(u, a.head_dim, a.turned);
          float y[2][N];
          turned(unit, unit.load(src + (t + r) * step), r, u, y);
          unit.store_f8(to + (a.slots[t + r] & (bs - 1)) * a.head_dim, y, scale);
        }
    }
  }
}

template <typename T, int N, bool IL>
__device__ __forceinline__ void runs_part(const KvAppendArgs& a, const Runs& w, int64_t group, float2* cs) {
  const int part = (int)(group % w.split), bs = 1 << a.block_shift, lane = threadIdx.x & 63;
  const int64_t first = group / w.split * w.tokens;
  const auto block_of = [&](int64_t t) -> int64_t {  // -1: not stored
    if (t < 0 || t >= a.num_tokens || (a.turned && a.positions[t] < 0)) return -1;
    const int64_t slot = a.slots[t];
    return slot < 0 || slot >= a.num_slots ? -1 : slot >> a.block_shift;
  };
  for (int64_t t = first; t < first + w.tokens && t < a.num_tokens; ++t) {
    const int64_t block = block_of(t);
    if (block < 0 || block_of(t - 1) == block) continue;
    int n = 0;  // rows of the run
    for (int r = 0; r < bs && n == r; r += 64) {
      const uint64_t out = __builtin_amdgcn_ballot_w64(r + lane >= bs || block_of(t + r + lane) != block);
      n = r + (out ? __builtin_ctzll(out) : 64);
    }
    run_part<T, N, IL>(a, w, part, t, a.slots[t], n, cs);
  }
}

template <typename T, int N, bool IL, bool F8, bool BLOCKS>
__global__ __launch_bounds__(kThreads) void append_kernel(KvAppendArgs a, Rows rows, Runs runs) {
  extern __shared__ float2 cs[];
  int64_t group = blockIdx.x;
  if constexpr (BLOCKS) {
    if (group < runs.groups) {
      runs_part<T, N, IL>(a, runs, group, cs);
      return;
    }
    group -= runs.groups;
  }
  rows_part<T, N, IL, F8>(a, rows, group, BLOCKS ? 0 : a.num_kv_heads, cs);
}

int power_of_two(int x) {
  int p = 1;
  while (p < x) p *= 2;
  return p;
}

constexpr int kLdsBytes = 160 * 1024;

template <typename T, int N, bool IL>
int append_launch(const KvAppendArgs& a, bool f8, hipStream_t s) {
  const bool blocks = a.scales[0] != nullptr;
  const int pairs = a.turned / 2;
  const int units = IL ? (a.head_dim + 2 * N - 1) / (2 * N) : a.turned / (2 * N) + (a.head_dim - a.turned + 2 * N - 1) / (2 * N);
  Rows rows{};
  rows.units = units;
  rows.lanes = std::min(units, kThreads);
  const int vectors = a.num_heads + (blocks ? 0 : 2 * a.num_kv_heads), per = kThreads / rows.lanes;
  rows.tokens = std::min(16, std::max(1, per / std::max(1, vectors)));
  while (rows.tokens * 2 <= std::min(per, 16) && a.num_tokens / (rows.tokens * 2) >= 1024) rows.tokens *= 2;
  rows.heads = per / rows.tokens;
  rows.groups = vectors ? (a.num_tokens + rows.tokens - 1) / rows.tokens : 0;
  Runs runs{};
  int lds = rows.tokens * pairs * 8;
  if (blocks) {
    runs.units = units;
    runs.lanes = std::min(64, power_of_two(units));
    runs.tokens = a.num_tokens <= 2048 ? 1 : 4;
    runs.split = 1;
    const int64_t all = ((int64_t)pairs << a.block_shift) * 8;
    runs.in_lds = all <= kLdsBytes;
    if (runs.in_lds) lds = std::max(lds, (int)all);
    runs.groups = (a.num_tokens + runs.tokens - 1) / runs.tokens * runs.split;
  }
  const int64_t groups = rows.groups + runs.groups;
  if (groups * kThreads > 0xffffffffLL) return fail_static(SCOOT_ERR_UNSUPPORTED, "kv append: too many tokens for one call");
  const auto go = [&](auto kernel) {
    if (lds > 64 * 1024) {
      const int rc = allow_full_lds((const void*)kernel, "kv append");
      if (rc != SCOOT_OK) return rc;
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)groups), dim3(kThreads), lds, s, a, rows, runs);
    return launched("kv append launch");
  };
  if (blocks) return go(append_kernel<T, N, IL, true, true>);
  return f8 ? go(append_kernel<T, N, IL, true, false>) : go(append_kernel<T, N, IL, false, false>);
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
