// Which form of the attention kernel calls take: reads "tokens heads kv_heads head_dim element_bytes requests max_new_len
// max_seq_len window" line by line and prints "few" or "tiles", waves, LDS buffers (0: few rows), parts
// and keys per part.
#include <cstdio>

#include "kv_plan.h"

using namespace scoot::kvattn;

int main() {
  long long tokens, heads, kv_heads, dim, bytes, seqs, max_new, max_seq, window;
  while (std::scanf("%lld %lld %lld %lld %lld %lld %lld %lld %lld", &tokens, &heads, &kv_heads, &dim, &bytes, &seqs, &max_new, &max_seq,
                    &window) == 9) {
    const Plan p = plan(tokens, (int)heads, (int)kv_heads, (int)dim, (int)bytes, (int)seqs, max_new, max_seq, (int)window);
    std::printf("%s %d %d %d %d\n", p.tile_rows ? "tiles" : "few", p.waves,
                p.tile_rows ? buffers((int)dim, (int)(dim * bytes)) : 0, p.splits, p.part);
  }
  return 0;
}
