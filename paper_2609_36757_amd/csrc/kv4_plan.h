// Work plan of the attention over a 4-bit cache (host code, plain C++, no HIP
// calls): tile height, which tiles' keys are split, and over how many workgroups.
// It depends on the call's sizes only, so that the workspace can be asked for
// beforehand; lengths on the device only shorten what a workgroup does.
#pragma once

#include <stdint.h>

#include <initializer_list>

namespace fastvr {

struct Kv4Plan {
  int32_t q_tiles;    // 16-row tiles of a workgroup: 1, 2 or 4
  int64_t row_tiles;  // workgroups over the rows of one (batch, key head)
  int64_t whole;      // tiles, the first ones, whose keys one workgroup walks
  int32_t n_split;    // workgroups over the keys of each of the others
  int64_t units;      // workgroups
  int64_t rows;       // rows with partial results: those of the split tiles
  int64_t ws_bytes;
};

constexpr int kKv4StepKeys = 32;
constexpr int kKv4Waves = 4;
constexpr int kKv4MaxSplit = 64;
constexpr int64_t kKv4MaxWorkspace = int64_t(64) << 20;
// Keys [lo, hi) that the token at position pos of a sequence of len tokens sees; none
// for pos < 0.  Neither end falls as pos grows.  (Kernel code; constexpr compiles it for
// the host as well.)
constexpr void kv4_interval(int pos, int len, int chunk_len, int window, int* lo, int* hi) {
  *lo = *hi = 0;
  if (pos < 0) return;
  const int c = (int)((uint32_t)pos / (uint32_t)chunk_len), first = c * chunk_len;
  if (window >= 0 && c > window) *lo = first - window * chunk_len;
  *hi = len - first > chunk_len ? first + chunk_len : len;
}

// Order of a head's row tiles.  Later rows may see more keys, so they go first.  The units of a
// round of 256 are dealt to the 8 XCDs in runs of 32 (xcd_unit) that share an L2; so that every run has
// tiles from all over the head, run j of `runs` holds the tiles j, j + runs, ... from the end.  With 256 tiles
// and more a round is one head's, dealing its units one by one does the same (0 runs).  32 query heads on 8, 8192
// queries over 8192 keys that see the ones before them: 690 us in rising order, an XCD having the longest 32
// tiles of each round, 510 in this one.
constexpr int kv4_runs(int row_tiles) { return row_tiles >= 256 || row_tiles <= 1 ? 0 : (row_tiles + 31) / 32; }
constexpr int kv4_tile(int i, int row_tiles, int runs) {
  if (runs <= 1) return row_tiles - 1 - i;
  const int len = (int)((uint32_t)row_tiles / (uint32_t)runs), longer = row_tiles - len * runs;
  const int split = longer * (len + 1);  // the first `longer` runs hold one tile more
  const int of = i < split ? len + 1 : len, from = i < split ? i : i - split;
  const int run = (int)((uint32_t)from / (uint32_t)of), in = from - run * of;
  return row_tiles - 1 - (in * runs + run + (i < split ? 0 : longer));
}

// First of n steps that workgroup `split` of `n_split` takes (the next one's first ends them).
// (n * split <= 2^19 * 64; a division of 64 bits would take longer than a step's loads)
constexpr int kv4_split_at(int n, int split, int n_split) { return (int)((uint32_t)n * (uint32_t)split / (uint32_t)n_split); }

// Time of a call in ns with q row tiles a workgroup (of `tiles` such tiles) and s
// workgroups over the keys of each, from measurements on a chip with 256 CUs, of kernels that
// held the softmax weights as one bf16 number (the second one adds up to 10% with one and two row
// tiles, and a third to a call of four that writes fp32).  head_dim 64 is not modelled apart: of its kernels
// with one and two row tiles 5 and 4 workgroups fit on a CU, not 4 and 2, and its steps take other times;
// the factor 0.85 stands for all of that.
//  * what a workgroup needs besides its steps: 4.3, 5.5 and 8 us for 1, 2 and 4 row tiles;
//  * a wave's steps one after the other, 630, 650 and 1080 ns each while a CU has one
//    workgroup, 400, 600 and 830 ns a workgroup where its instructions are the limit
//    (head_dim 64: 0.85 of that), in as many rounds as do not fit at once (4, 2 and 2 on a CU);
//  * the cache at 5.5 TB/s once, and from L2 at four times that for every other row tile; of
//    this and the steps the shorter hides behind the longer by 70%;
//  * from two workgroups a tile on the second kernel, 3 us and 3 us more on the host, 25 ns a
//    workgroup, 0.25 ns a row, and the partial results written and read.
// Measured, 12 heads, head_dim 128: one query over 65280 keys 318 us with 1 workgroup a tile, 87 with
// 4, 27.9 with 16, 23.5 with 32; 64 queries over 1000 keys 9.3, 11.3 and 16.6 us with 1, 2 and 4 row
// tiles, 3120 over 18720 keys 410 and 369 us with 2 and 4 (all tiles split), 323 with 4 and 512 of the 588
// tiles whole; 6000 over 65280 keys 2286 us with all tiles whole, 1989 with 1024 of 1128.  4000 queries over 4000
// keys that see the ones before them: 79 us as if all tiles took the longest one's time, 76 now.
// With `whole` tiles ahead that are not split, these take as long as whole rounds, filled or not, since
// the others' workgroups take the places that are left; each workgroup of the others then adds half of
// what it needs besides its steps.
//  * tiles that see `even` of the longest one's keys on average take that share of the rounds, and half
//    a round at the end, but no less than the longest one alone.
inline double kv4_time(int64_t whole, int64_t tiles, int q, int64_t steps, double even, double bytes, int64_t rows,
                       int64_t d, int64_t s) {
  const int at = q == 1 ? 0 : (q == 2 ? 1 : 2);
  constexpr double kFixed[3] = {4300, 5500, 8000}, kWait[3] = {630, 650, 1080}, kBusy[3] = {400, 600, 830};
  const int64_t at_once = q == 1 ? 4 * 256 : 2 * 256;
  const double rounds_each = q == 1 ? 1.0 / (4 * 256) : 1.0 / (2 * 256);
  const int64_t units = tiles * s, all = whole + units, here = all < at_once ? all : at_once;
  const uint32_t own = ((uint32_t)(steps + s - 1) / (uint32_t)s + kKv4Waves - 1) / kKv4Waves;
  const double busy = kBusy[at] * (double)((here + 255) / 256);
  const double step = (kWait[at] > busy ? kWait[at] : busy) * (d == 128 ? 1.0 : 0.85);
  // (many rounds overlap, only their last one is not full)
  double rounds = (double)units * even * rounds_each + 0.5;
  if (even == 1.0 && units < 4 * at_once) rounds = (double)((uint32_t)(units + at_once - 1) / (uint32_t)at_once);
  rounds = rounds > 1.0 ? rounds : 1.0;
  const double ahead = even * (double)whole * rounds_each * step * (double)((steps + kKv4Waves - 1) / kKv4Waves);
  const double wait = (step * (double)own + (whole > 0 ? 0.5 * kFixed[at] : 0.0)) * rounds + ahead, read = bytes * (1.0 / 5500.0);
  return kFixed[at] + (wait > read ? wait + 0.3 * read : read + 0.3 * wait) +
         (s > 1 ? 6000.0 + 25.0 * (double)s + 0.25 * (double)rows + (double)(rows * s * (d * 4 + 8)) * (2.0 / 5000.0) : 0.0);
}

// B, H, Hkv, nq >= 1; 0 <= cache_len; 1 <= chunk_len; window >= -1; H a multiple of Hkv.
inline Kv4Plan kv4_plan(int64_t B, int64_t H, int64_t Hkv, int64_t nq, int64_t d, int64_t cache_len, int64_t chunk_len,
                        int64_t window) {
  Kv4Plan p{};
  const int64_t G = H / Hkv, R = nq * G;
  constexpr int64_t kAtOnce[5] = {0, 4 * 256, 2 * 256, 0, 2 * 256};
  // keys that a token sees on average, from 8 of them
  double seen = (double)cache_len;
  if (nq > 1 && chunk_len < cache_len) {
    constexpr int kSample = 8;
    const int W = (int)(window < cache_len ? window : -1);
    int64_t sum = 0;
    for (int i = 0; i < kSample; ++i) {
      int lo, hi;
      kv4_interval((int)(cache_len - nq + nq * (2 * i + 1) / (2 * kSample)), (int)cache_len, (int)chunk_len, W, &lo, &hi);
      sum += hi - lo + kKv4StepKeys;
    }
    seen = (double)sum / kSample;
  }
  double best = 0;
  for (int q : {4, 2, 1}) {
    if (q > 1 && R <= 8 * q) continue;  // half of the rows, and more, would be empty
    const int64_t tile = 16 * q, row_tiles = (R + tile - 1) / tile, tiles = B * Hkv * row_tiles;
    // keys that a tile's rows see at most: their own chunks and the window before them
    int64_t keys = cache_len;
    const int64_t tokens = (tile + G - 1) / G + 1;
    if (window >= 0 && chunk_len < cache_len && window < cache_len / chunk_len) {
      const int64_t span = (window + 2) * chunk_len + tokens;
      keys = span < keys ? span : keys;
    }
    const int64_t steps = (keys + kKv4StepKeys - 1) / kKv4StepKeys + 1;
    const double share = seen / (double)(keys + kKv4StepKeys), even = row_tiles > 1 && share < 0.9 ? share : 1.0;
    // (in double from the start: of sizes that the caller refuses afterwards the product passes 2^63)
    const double bytes = (double)(B * Hkv) * (double)(keys * (d / 2 + d / 32) * 2) * (1.0 + 0.25 * (double)(row_tiles - 1));
    // all tiles split alike, or only those that would fill a last round in part
    const int64_t full = tiles / kAtOnce[q] * kAtOnce[q];
    for (int tail = 0; tail < (full > 0 && full < tiles ? 2 : 1); ++tail) {
      const int64_t whole = tail ? full : 0, rest = tiles - whole, rows = rest * (row_tiles > 1 ? tile : R);
      // numbers of splits in general, and those that just fill one to four rounds
      constexpr int kGeneral = 12, kFull = 4;
      int64_t splits[kGeneral + kFull] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, kKv4MaxSplit};
      for (int k = 1; k <= kFull; ++k) {
        const int64_t s = rest > k * kAtOnce[q] ? 1 : (int64_t)((uint32_t)(k * kAtOnce[q]) / (uint32_t)rest);
        splits[kGeneral + k - 1] = s < kKv4MaxSplit ? s : kKv4MaxSplit;
      }
      double times[kGeneral + kFull], least = 0;
      int n = 0;
      for (int64_t s : splits) {
        if (s > 1 && (s > steps || rows * s * (d * 4 + 8) > kKv4MaxWorkspace)) continue;
        times[n] = kv4_time(whole, rest, q, steps, even, bytes, rows, d, s);
        least = n == 0 || times[n] < least ? times[n] : least;
        splits[n++] = s;
      }
      if (p.q_tiles != 0 && least >= best) continue;
      best = least;
      p.q_tiles = q;
      p.row_tiles = row_tiles;
      // of splits that take the same time the most: shorter sequences than the longest leave
      // some of their workgroups nothing to do
      p.n_split = 1;
      for (int i = 0; i < n; ++i)
        if (times[i] <= (tail ? 1.0 : 1.03) * least && splits[i] > p.n_split) p.n_split = (int32_t)splits[i];
      p.whole = p.n_split > 1 ? whole : tiles;
      p.rows = p.n_split > 1 ? rows : 0;
    }
  }
  p.units = p.whole + (B * Hkv * p.row_tiles - p.whole) * p.n_split;
  // partial results of each (row, split): O, then maximum and sum
  p.ws_bytes = p.rows * p.n_split * (d * 4 + 8);
  return p;
}

// Waves that join a row's shares: a workgroup of four for a row, or, where a wave a row fills the
// chip and holds all of a row's shares, one.
inline int kv4_join_waves(const Kv4Plan& p) { return p.n_split <= 16 && p.rows >= 2048 ? 1 : kKv4Waves; }

}  // namespace fastvr
