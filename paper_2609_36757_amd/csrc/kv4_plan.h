// Work plan of the attention over a 4-bit cache (host code, plain C++, no HIP
// calls): tile height, and over how many workgroups the keys of a tile are split.
// It depends on the call's sizes only, so that the workspace can be asked for
// beforehand; lengths on the device only shorten what a workgroup does.
#pragma once

#include <stdint.h>

#include <initializer_list>

namespace fastvr {

struct Kv4Plan {
  int32_t q_tiles;    // 16-row tiles of a workgroup: 1, 2 or 4
  int64_t row_tiles;  // workgroups over the rows of one (batch, key head)
  int32_t n_split;    // workgroups over the keys of one tile
  int64_t units;      // workgroups
  int64_t rows;       // rows of the call: B * H * Nq
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
  const int c = pos / chunk_len, first = c * chunk_len;
  if (window >= 0 && c > window) *lo = first - window * chunk_len;
  *hi = len - first > chunk_len ? first + chunk_len : len;
}

// First of n steps that workgroup `split` of `n_split` takes (the next one's first ends them).
constexpr int kv4_split_at(int n, int split, int n_split) { return (int)((int64_t)n * split / n_split); }

// Time of a call in ns, for s workgroups over the keys of a tile: a wave's steps one after
// the other, 630 ns each (four row tiles: 1300, and 1650 with two workgroups on a CU), in
// as many rounds as the workgroups need (four fit on a CU, two of those with more row
// tiles); the cache's bytes at 5.5 TB/s, which hide the steps, or hide behind them, by 70%;
// from two workgroups a tile on the second kernel, which joins them (3 us, and 3 us more on
// the host), and the traffic of the partial results.  Measured for one query over 65280 keys of 12 heads: 1 workgroup a tile
// 318 us, 4 87, 16 27.9, 32 23.5, 64 23.6.
inline double kv4_time(int64_t tiles, int64_t q_tiles, int64_t steps, int64_t bytes, int64_t rows, int64_t d, int64_t s) {
  const int64_t units = tiles * s, at_once = q_tiles == 1 ? 1024 : 512;
  const int64_t own = ((steps + s - 1) / s + kKv4Waves - 1) / kKv4Waves;
  const double step = q_tiles <= 2 ? 630.0 : (units <= 256 ? 1300.0 : 1650.0);
  // (many rounds overlap, only their last one is not full)
  const double rounds = units < 4 * at_once ? (double)((units + at_once - 1) / at_once) : (double)units / (double)at_once + 0.5;
  const double wait = step * (double)own * rounds, read = (double)bytes / 5500.0;
  return (wait > read ? wait + 0.3 * read : read + 0.3 * wait) +
         (s > 1 ? 6000.0 + (double)(rows * s * (d * 4 + 8) * 2) / 5000.0 : 0.0);
}

// B, H, Hkv, nq >= 1; 0 <= cache_len; 1 <= chunk_len; window >= -1; H a multiple of Hkv.
inline Kv4Plan kv4_plan(int64_t B, int64_t H, int64_t Hkv, int64_t nq, int64_t d, int64_t cache_len, int64_t chunk_len,
                        int64_t window) {
  Kv4Plan p{};
  const int64_t G = H / Hkv, R = nq * G;
  p.q_tiles = R <= 16 ? 1 : (R <= 32 ? 2 : 4);
  const int64_t tile = 16 * p.q_tiles;
  p.row_tiles = (R + tile - 1) / tile;
  p.rows = B * H * nq;
  // keys that a tile's rows see at most: their own chunks and the window before them
  int64_t keys = cache_len;
  const int64_t tokens = (tile + G - 1) / G + 1;
  if (window >= 0 && chunk_len < cache_len && window < cache_len / chunk_len) {
    const int64_t span = (window + 2) * chunk_len + tokens;
    keys = span < keys ? span : keys;
  }
  const int64_t steps = (keys + kKv4StepKeys - 1) / kKv4StepKeys + 1;
  const int64_t tiles = B * Hkv * p.row_tiles;
  const int64_t bytes = tiles * keys * (d / 2 + d / 32) * 2;
  p.n_split = 1;
  double best = kv4_time(tiles, p.q_tiles, steps, bytes, p.rows, d, 1);
  for (int32_t s : {2, 3, 4, 6, 8, 12, 16, 24, 32, 48, kKv4MaxSplit}) {
    // (no more partial results than gain 2% a step, or than 64 MB)
    if (s > steps || p.rows * s * (d * 4 + 8) > kKv4MaxWorkspace) break;
    const double time = kv4_time(tiles, p.q_tiles, steps, bytes, p.rows, d, s);
    if (time < 0.98 * best) {
      best = time;
      p.n_split = s;
    }
  }
  p.units = tiles * p.n_split;
  // partial results of each (row, split): O, then maximum and sum
  p.ws_bytes = p.n_split > 1 ? p.rows * p.n_split * (d * 4 + 8) : 0;
  return p;
}

}  // namespace fastvr
