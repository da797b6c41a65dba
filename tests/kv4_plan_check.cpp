// Checks of the 4-bit attention's work plan and interval arithmetic (csrc/kv4_plan.h),
// built with sanitizers and run on the CPU by tests/test_kv4_plan.py.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "kv4_plan.h"

using namespace fastvr;

#define CHECK(x)                                                    \
  do {                                                              \
    if (!(x)) {                                                     \
      std::printf("line %d: %s\n", __LINE__, #x);                   \
      std::exit(1);                                                 \
    }                                                               \
  } while (0)

int main() {
  // intervals against the definition, key by key
  long cases = 0;
  for (int len = 0; len <= 14; ++len)
    for (int L = 1; L <= 15; ++L)
      for (int W = -1; W <= 5; ++W) {
        int last_lo = 0, last_hi = 0;
        for (int pos = -3; pos < len; ++pos) {
          int lo = -1, hi = -1;
          kv4_interval(pos, len, L, W, &lo, &hi);
          for (int key = 0; key < len; ++key) {
            const int diff = pos < 0 ? -1 : pos / L - key / L;
            const bool sees = pos >= 0 && diff >= 0 && (W < 0 || diff <= W);
            CHECK(sees == (key >= lo && key < hi));
          }
          CHECK(lo >= last_lo && hi >= last_hi && lo <= hi && hi <= len);
          CHECK(pos < 0 || (lo <= pos && pos < hi));
          last_lo = lo;
          last_hi = hi;
          ++cases;
        }
      }
  // the largest positions do not overflow
  {
    const int n = 16 * 1024 * 1024;
    int lo, hi;
    kv4_interval(n - 1, n, n, -1, &lo, &hi);
    CHECK(lo == 0 && hi == n);
    kv4_interval(n - 1, n, 1, n - 1, &lo, &hi);
    CHECK(lo == 0 && hi == n);
    kv4_interval(n - 1, n, n - 1, 0, &lo, &hi);
    CHECK(lo == n - 1 && hi == n);
  }
  // the order of a head's tiles: each of them once, the longest first, and every run of 32 with
  // tiles from all over the head
  for (int n = 1; n < 700; ++n) {
    const int runs = kv4_runs(n);
    std::vector<int> seen(n, 0), order(n);
    for (int i = 0; i < n; ++i) {
      order[i] = kv4_tile(i, n, runs);
      CHECK(order[i] >= 0 && order[i] < n);
      CHECK(seen[order[i]]++ == 0);
    }
    CHECK(order[0] == n - 1);
    if (runs > 1)
      for (int j = 0; j + n / runs <= n; ++j) {
        double sum = 0;
        for (int i = 0; i < n / runs; ++i) sum += order[j + i];
        const double mean = sum / (n / runs), all = (n - 1) / 2.0;
        CHECK(std::fabs(mean - all) <= 0.5 * runs + 0.5 * runs);
      }
    ++cases;
  }
  // plans: every step of every tile belongs to one workgroup, sizes and workspace agree
  long with_whole = 0;
  std::mt19937 rng(7);
  auto pick = [&](int64_t lo, int64_t hi) { return std::uniform_int_distribution<int64_t>(lo, hi)(rng); };
  auto log_pick = [&](double hi) { return (int64_t)std::exp2(std::uniform_real_distribution<double>(0, hi)(rng)); };
  for (int i = 0; i < 20000; ++i) {
    const int64_t B = log_pick(6), Hkv = log_pick(5), G = log_pick(4), nq = log_pick(15), n = log_pick(24) - (i % 50 == 0);
    const int64_t d = i % 2 ? 64 : 128, L = i % 3 ? log_pick(20) : 1, W = i % 2 ? -1 : pick(0, 300);
    const Kv4Plan p = kv4_plan(B, Hkv * G, Hkv, nq, d, n, L, W);
    CHECK(p.q_tiles == 1 || p.q_tiles == 2 || p.q_tiles == 4);
    CHECK(p.row_tiles * 16 * p.q_tiles >= nq * G && (p.row_tiles - 1) * 16 * p.q_tiles < nq * G);
    CHECK(p.n_split >= 1 && p.n_split <= kKv4MaxSplit && p.whole >= 0);
    const int64_t tiles = B * Hkv * p.row_tiles, rest = tiles - p.whole;
    CHECK(p.n_split > 1 ? rest > 0 : rest == 0);
    CHECK(p.units == p.whole + rest * p.n_split);
    CHECK(p.rows == rest * (p.row_tiles > 1 ? 16 * p.q_tiles : nq * G));
    CHECK(p.ws_bytes == p.rows * p.n_split * (d * 4 + 8) && p.ws_bytes <= kKv4MaxWorkspace);
    with_whole += p.n_split > 1 && p.whole > 0;
    const Kv4Plan again = kv4_plan(B, Hkv * G, Hkv, nq, d, n, L, W);
    CHECK(again.n_split == p.n_split && again.whole == p.whole && again.ws_bytes == p.ws_bytes);
    const int steps = (int)(n / kKv4StepKeys + 1);
    int at = 0;
    for (int s = 0; s < p.n_split; ++s) {
      CHECK(kv4_split_at(steps, s, p.n_split) == at);
      at = kv4_split_at(steps, s + 1, p.n_split);
    }
    CHECK(at == steps);
    ++cases;
  }
  CHECK(with_whole > 100);
  std::printf("%ld cases ok\n", cases);
  return 0;
}
