// The words through which an attention kernel's waves talk (csrc/kv_waves.h), with threads as waves, in the kernel's order: are
// entries missing, then, again and again, the largest exponent, then is a result spoilt, then exponents again.  Every answer is
// compared; built with -fsanitize=thread, an access that no barrier orders is reported, too.
#include <algorithm>
#include <atomic>
#include <condition_variable>
#include <cstdio>
#include <mutex>
#include <thread>
#include <vector>

#define __device__
#define __forceinline__ inline
#include "kv_waves.h"

using namespace scoot::kvattn;

namespace {
constexpr int W = 4;

class Barrier {
 public:
  void wait() {
    std::unique_lock<std::mutex> l(m_);
    const int turn = turn_;
    if (++in_ == W) {
      in_ = 0;
      ++turn_;
      cv_.notify_all();
    } else {
      cv_.wait(l, [&] { return turn_ != turn; });
    }
  }

 private:
  std::mutex m_;
  std::condition_variable cv_;
  int in_ = 0, turn_ = 0;
};

struct Threads {
  Barrier* barrier;
  int w;
  void sync() const { barrier->wait(); }
  bool leads() const { return true; }
  int wave() const { return w; }
};

int words[W];
std::atomic<int> wrong{0};
}  // namespace

int main() {
  Barrier barrier;
  std::vector<std::thread> waves;
  for (int w = 0; w < W; ++w)
    waves.emplace_back([&barrier, w] {
      const Threads g{&barrier, w};
      for (int i = 0; i < 2000; ++i) {
        wrong += (any_of_waves<W>(g, words, false) != 0);
        for (int n = 0; n < 2; ++n) wrong += most_of_waves<W>(g, words, 1 + (i + w * 7 + n) % 50) <= 0;
        wrong += (any_of_waves<W>(g, words, i % W == w) == 0);
        const auto low = [i](int v) { return 100 + (i * 3 + v * 11) % 60; };
        const auto high = [i](int v) { return (i * 5 + v * 17) % 256; };
        int most[2] = {0, 0};
        for (int v = 0; v < W; ++v) most[0] = std::max(most[0], low(v)), most[1] = std::max(most[1], high(v));
        wrong += (most_of_waves<W>(g, words, high(w) << 16 | low(w)) != (most[1] << 16 | most[0]));
      }
    });
  for (std::thread& t : waves) t.join();
  std::printf("%d wrong\n", wrong.load());
  return wrong != 0;
}
