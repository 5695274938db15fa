// What the waves of a workgroup tell each other through words of LDS, one for each wave.  A host build with threads as waves
// takes this header, too.
#pragma once

namespace scoot {
namespace kvattn {

// Calls each(x) for what every wave says, in their order.  `group`: sync(), the workgroup's barrier; wave(), the caller's
// number; leads(), true for one of a wave's lanes.  The first barrier is for the words' last use: without it a wave that is
// ahead would write its word while another one still reads what it said before.
template <int W, typename Group, typename Each>
__device__ __forceinline__ void exchange(const Group& group, int* words, int mine, Each each) {
  group.sync();
  if (group.leads()) words[group.wave()] = mine;
  group.sync();
#pragma unroll
  for (int w = 0; w < W; ++w) each(words[w]);
}

// Whether `x` holds in any wave.
template <int W, typename Group>
__device__ __forceinline__ int any_of_waves(const Group& group, int* words, bool x) {
  int any = 0;
  exchange<W>(group, words, x, [&](int said) { any |= said; });
  return any;
}

// The larger one of two numbers of 16 bits, in each half of a word.
__device__ __forceinline__ int most_of(int a, int b) {
  const int low = (a & 0xffff) > (b & 0xffff) ? a & 0xffff : b & 0xffff, high = a >> 16 > b >> 16 ? a >> 16 : b >> 16;
  return high << 16 | low;
}
// The largest of what the waves say, in each half; neither half is 2^15 or more.
template <int W, typename Group>
__device__ __forceinline__ int most_of_waves(const Group& group, int* words, int x) {
  int most = 0;
  exchange<W>(group, words, x, [&](int said) { most = most_of(most, said); });
  return most;
}

}  // namespace kvattn
}  // namespace scoot
