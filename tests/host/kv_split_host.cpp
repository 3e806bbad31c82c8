// Host driver for the splits of attention over the KV cache: reads lines "heads d hq seqs max_new max_cached tokens
// capacity seen" and prints "chunk nsplit splits", then the first key and the end of each split for a row that sees that many.
#include <cstdio>

#include "kv_plan.h"

using namespace lrqat;

int main() {
  KvSizes z;
  long long tokens, capacity;
  int seen;
  while (std::scanf("%d %d %d %d %d %d %lld %lld %d", &z.heads, &z.d, &z.hq, &z.seqs, &z.max_new, &z.max_cached, &tokens, &capacity, &seen) == 9) {
    z.tokens = tokens;
    z.capacity = capacity;
    const KvAttnPlan p = kv_attn_plan(z);
    const int count = kv_splits(int64_t(seen) - 1, p.chunk, p.nsplit);
    if (kv_split_up(int64_t(seen) - 1, p.chunk, p.nsplit) != (count > 1)) return 1;
    std::printf("%d %d %d", p.chunk, p.nsplit, count);
    for (int s = 0; s < p.nsplit; ++s) std::printf(" %d %d", s * p.chunk, kv_split_end(s, p.nsplit, p.chunk, seen));
    std::printf("\n");
  }
  return 0;
}
