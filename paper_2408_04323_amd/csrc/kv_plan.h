// How an attention call over the block cache is split, and which form of the
// kernel it takes.  Host code only.
#pragma once

#include <algorithm>
#include <cstdint>

namespace scoot {
namespace kvattn {

constexpr int kWaves = 4;                // of a workgroup (one of few rows may have eight)
constexpr int kFew = 16;                 // rows of a request that one workgroup's waves handle together
constexpr int kRows = 32;                // rows of a wave otherwise
constexpr int kTile = kRows * kWaves;    // rows of a tile
constexpr int kStripKeys = 64;           // keys per strip of a shared tile
constexpr int kWideRow = 256;            // bytes of a cache row up to which eight waves' strips fit the LDS

struct Plan {
  int64_t items;    // tiles or requests
  int splits;
  int part;         // keys per part, a multiple of 128
  int tile_rows;    // rows of a tile; 0: the items are requests, of few rows each
  int waves;        // of a workgroup
};

// Bytes of a strip of K and V.
constexpr int strip_bytes(int row_bytes) { return 2 * kStripKeys * row_bytes; }
// Waves per SIMD that the registers are to suffice for; no buffers: few rows.
constexpr int waves_per_simd(int head_dim, int buffers) {
  return buffers == 0 ? 2 : head_dim == 64 ? 3 : head_dim == 128 ? 2 : 1;
}
// Buffers of tiles.  Four gain something where the registers leave a compute unit one workgroup and the buffers take
// less than 128 KiB: 8-bit heads of 192, 500 tokens over 30,000 323 -> 317 us.  8-bit heads of 256 193 -> 194; heads of 64
// and 128 with a compute unit for every workgroup: one prompt of 300 tokens 9.7 -> 10.0 and 12.8 -> 13.1, 500 tokens over
// 30,000 152 and 251 with either.
constexpr int buffers(int head_dim, int row_bytes) {
  return waves_per_simd(head_dim, 2) == 1 && 4 * strip_bytes(row_bytes) < 128 * 1024 ? 4 : 2;
}

constexpr int64_t kUnits = 256;   // compute units
constexpr int kPartOf = 128;      // parts are multiples of this many keys: a strip of 32 for each of four waves
constexpr int kMinPart = 256;     // of few rows
constexpr int kMinTilePart = 256; // of tiles: four strips (940 keys, heads of 128: 16.0 us, 19.6 with 512; with 128 540 keys
                                  // 17.1 -> 16.5, but 2040 keys, heads of 64, 14.0 -> 15.2)
constexpr double kJoinLaunch = 5e-6;  // seconds, bytes per second
constexpr double kJoinRate = 4e12;
constexpr int kAlone8 = 1024;     // keys that eight waves of one workgroup do not share with another,
constexpr int kAlone4 = 768;      // and four waves

// Parts of the keys of tiles: the number with the shortest time.  A strip of 64
// keys takes a workgroup as long as strip_time() says with one, two or three of
// them on its compute unit (heads of 128: 1.15 and 1.81 us); what does not fit at
// once follows.  Parts cost a launch and their way through memory, once out and
// once in.  Against as many parts as fill the chip: chunks of 331 tokens over 547
// 37 -> 27 us (one part, not two), of 160 over 10,087 50 -> 40 (ten, not twenty), of
// 270 over 24,258 347 -> 257 (more than fit at once, not two).
inline double strip_time(int head_dim, int beside) {
  if (head_dim <= 64) return (beside == 0 ? 0.77e-6 : beside == 1 ? 1.1e-6 : 1.63e-6);
  if (head_dim <= 128) return beside == 0 ? 1.15e-6 : 1.81e-6;
  return head_dim * 7.4e-9;  // 192: 1.4 us, 256: 1.9 us
}

inline int64_t parts_of_tiles(int64_t groups, int64_t keys, int64_t rows, int head_dim) {
  const int fit = head_dim <= 64 ? 3 : head_dim <= 128 ? 2 : 1;  // workgroups that a compute unit holds
  const int64_t most = (keys + kMinTilePart - 1) / kMinTilePart;
  int64_t best = 1;
  double least = 0;
  for (int i = 1; i <= 8 + fit; ++i) {  // few parts, and as many as give every unit one, two, three workgroups
    const int64_t n = i <= 8 ? i : (i - 8) * kUnits / groups;
    if (n > most || (i > 8 && n <= 8)) continue;
    const int64_t beside = std::min<int64_t>((groups * n - 1) / kUnits, fit - 1);
    double t = (double)keys / (64 * n) * strip_time(head_dim, (int)beside) * std::max(1.0, (double)(groups * n) / (fit * kUnits));
    if (n > 1) t += kJoinLaunch + (double)(2 * n * rows * head_dim * 4) / kJoinRate;
    if (i == 1 || t < least) least = t, best = n;
  }
  return best;
}

// Parts of the keys of few rows.  A part costs its share of a second launch and of
// memory; what it gives is more workgroups, as long as they do not already draw
// what the memory gives.  Measured with caches in memory (not in L2), in us:
// * One request, heads of 128 (eight waves): 800 keys 9.8 in one part, 11.1 in
//   four; 1000 11.1, 11.3; 1500 13.7, 11.6; 2000 17.4, 12.8; 4000 39.8 in one, 15.1 in
//   eight, 14.1 in sixteen.  Heads of 192 (four waves): 600 12.3 in one part, 13.1
//   in two; 800 13.7, 13.3 in three; 1000 15.4, 13.5.  So kAlone8 and kAlone4, and then
//   parts of 256 keys and more: 9000 keys, heads of 256: 25 in 8 parts, 21 in 16, 19 in 32.
// * Parts until every unit has one workgroup, not several: 100 requests of up to
//   16,000, heads of 256 278 with 256 workgroups, 283 with 512, 294 with 1024; 8 of up to
//   16,000, heads of 128 68, 77, 77; 4 of 16,000, 8 bits 32, 38, 48.
// * ... of ten keys for every workgroup at least: 16 of 4000, heads of 64 (256 workgroups)
//   49 in one part, 56 in two; 16 of 1000, heads of 256 26 in one, 19 in three.
// * More workgroups than units get parts for the units that have one more, and for unequal
//   lengths, of seven keys for every workgroup at least.  288 workgroups, all of 4095 keys,
//   131 in one part, 120 in two; 400 of up to 16,000, heads of 192 595 in one part, 587 in
//   four, 521 in five; 512 of up to 4095, heads of 256 258 in one, 275 in two.
// All of 182 such calls: 2.4% over the best of seven rules each, at most 16%.
inline int64_t parts_of_few(int64_t groups, int64_t keys, int waves) {
  if (keys <= (waves == 8 ? kAlone8 : kAlone4)) return 1;
  const bool more = groups > kUnits;
  return std::min((more ? 8 : 1) * kUnits / groups, keys / std::max<int64_t>(kMinPart, (more ? 7 : 10) * groups));
}

// Requests of at most 16 rows (new tokens x heads per key head) are items of
// their own; once some have more, tiles of 128 rows are.
inline Plan plan(int64_t num_tokens, int num_heads, int num_kv_heads, int head_dim, int element_bytes, int num_seqs, int64_t max_new_len,
          int64_t max_seq_len, int window) {
  Plan p{};
  const int64_t G = num_heads / num_kv_heads;
  const int64_t longest = std::min<int64_t>(max_new_len, num_tokens);
  const bool tiles = longest * G > kFew;
  p.tile_rows = tiles ? kTile : 0;
  p.items = tiles ? num_tokens * G / p.tile_rows + num_seqs : num_seqs;
  int64_t keys = max_seq_len;
  if (window > 0) keys = std::min<int64_t>(keys, (int64_t)window + (tiles ? p.tile_rows / G : longest) + 32);
  keys = std::max<int64_t>(keys, 1);
  // Tiles that have rows: as many as the numbers if all requests but one are single tokens, else fewer, at least one for
  // every request and for every 128 rows; so many if there is one request.
  const int64_t least = std::max<int64_t>(num_seqs, (num_tokens * G + kTile - 1) / kTile);
  const int64_t most = tiles && num_seqs == 1 ? least : p.items;
  const int64_t real = tiles ? (most + least) / 2 : p.items;
  const int64_t groups = std::max<int64_t>(1, real * num_kv_heads);
  int64_t want;
  p.waves = kWaves;
  if (tiles) {
    want = parts_of_tiles(groups, keys, num_tokens * num_heads, head_dim);
  } else {
    // Few items of few rows: eight waves each (one request of 1000 keys, heads of 128, in one part 11.6 -> 10.5 us; of 130
    // keys 7.5 -> 7.8).
    if (groups <= kUnits && head_dim * element_bytes <= kWideRow) p.waves = 8;
    want = parts_of_few(groups, keys, p.waves);
  }
  want = std::max<int64_t>(1, want);
  int64_t part = (keys + want - 1) / want;
  part = std::max<int64_t>(tiles ? kMinTilePart : kPartOf, (part + kPartOf - 1) / kPartOf * kPartOf);
  p.part = (int)std::min<int64_t>(part, (int64_t)1 << 30);
  // Of few rows, less than kPartOf keys go to the part before; a tile's parts are done by their time, and the longest
  // decides (40 tokens over 540 keys in parts of 256, 256 and 28: heads of 256 26.9 us, 29.8 with 256 and 284).
  p.splits = (int)std::max<int64_t>(1, (keys + p.part - (tiles ? 1 : kPartOf)) / p.part);
  return p;
}

}  // namespace kvattn
}  // namespace scoot
