// Prints what csrc/kv4_plan.h plans for calls read as lines of B H Hkv Nq d cache_len chunk_len window.
#include <cstdio>

#include "kv4_plan.h"

int main() {
  long long a[8];
  while (std::scanf("%lld %lld %lld %lld %lld %lld %lld %lld", a, a + 1, a + 2, a + 3, a + 4, a + 5, a + 6, a + 7) == 8) {
    const fastvr::Kv4Plan p = fastvr::kv4_plan(a[0], a[1], a[2], a[3], a[4], a[5], a[6], a[7]);
    std::printf("%d %s %s\n", p.q_tiles, p.n_split == 1 ? "none" : (p.whole > 0 ? "tail" : "split"),
                p.n_split == 1 ? "None" : (fastvr::kv4_join_waves(p) == 1 ? "wave" : "group"));
  }
  return 0;
}
