// Work plan of the attention over a 4-bit cache (host code, plain C++, no HIP
// calls): tile height, and over how many workgroups the keys of a tile are split.
// It depends on the call's sizes only, so that the workspace can be asked for
// beforehand; lengths on the device only shorten what a workgroup does.
#pragma once

#include <stdint.h>

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
constexpr int64_t kKv4TargetUnits = 1024;  // 4 workgroups on each of 256 CUs
constexpr int64_t kKv4MinSteps = 16;       // steps of a workgroup worth a split

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
  int64_t s = kKv4TargetUnits / tiles;
  if (s > steps / kKv4MinSteps) s = steps / kKv4MinSteps;
  p.n_split = (int32_t)(s < 1 ? 1 : (s > kKv4MaxSplit ? kKv4MaxSplit : s));
  p.units = tiles * p.n_split;
  // partial results of each (row, split): O, then maximum and sum
  p.ws_bytes = p.n_split > 1 ? p.rows * p.n_split * (d * 4 + 8) : 0;
  return p;
}

}  // namespace fastvr
