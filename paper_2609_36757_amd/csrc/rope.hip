// Rotary positions of query and key heads, and their gradient (the turn by the
// negative angle).
//
// Pair p of a token turns by theta = position * inv_freq[p].  The angle is taken in
// quarter turns in fp64, t = position * (inv_freq[p] * 2 / pi): its nearest integer
// gives the quadrant, the rest r in [-1/2, 1/2] goes to fp32, so far positions keep
// an absolute angle error below 1e-7 + position * 2e-16 radians.  sin and cos of
// r * pi / 2 are their Taylor sums (to r^9 and r^10: the first terms left out are
// below 2e-9 and 5e-10).
//
// The kernel is bound by HBM bandwidth: x is read and y written once.  A thread
// takes one unit of a token, 8 elements of a head (interleaved) or 8 + 8 (halves),
// for up to kHeads heads: its sines and cosines are taken once for all of them,
// while their loads are in flight.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gfx950_ops.h"
#include "launch.h"

namespace fastvr {
namespace {

using namespace dev;

constexpr int kThreads = 256;

struct RopeParams {
  const void* x;
  void* y;
  int64_t x_sb, x_st, y_sb, y_st;
  const int32_t* pos;
  const double* f;
  int64_t pos_sb;
  int32_t n_axes, split1, split2, n_pairs;
  uint32_t rows;  // tokens * head splits
  int32_t H, splits, units, rows_per_block;
  float amp, sin_amp;  // sin_amp: negative for the inverse turn
};

// amplitude * (cos, sin) of pair p of the token at `pos`
__device__ __forceinline__ void turn(const RopeParams& p, const int32_t* pos, int pair, float& c, float& s) {
  const int axis = pair < p.split1 ? 0 : (pair < p.split2 ? 1 : 2);
  const double t = (double)pos[axis] * (p.f[pair] * 0.63661977236758134308);  // quarter turns
  const double n = __builtin_rint(t);
  const float r = (float)(t - n);
  const int quad = (int)(n - 4.0 * __builtin_rint(n * 0.25)) & 3;
  const float z = r * r;
  // (pi/2)^k / k!
  float sn = __builtin_fmaf(z, 1.6044118e-4f, -4.6817541e-3f);
  sn = __builtin_fmaf(sn, z, 7.9692626e-2f);
  sn = __builtin_fmaf(sn, z, -6.4596410e-1f);
  sn = __builtin_fmaf(sn, z, 1.5707963f) * r;
  float cs = __builtin_fmaf(z, -2.5202042e-5f, 9.1926027e-4f);
  cs = __builtin_fmaf(cs, z, -2.0863481e-2f);
  cs = __builtin_fmaf(cs, z, 2.5366951e-1f);
  cs = __builtin_fmaf(cs, z, -1.2337006f);
  cs = __builtin_fmaf(cs, z, 1.0f);
  const float a = (quad & 1) ? sn : cs, b = (quad & 1) ? cs : sn;
  c = ((quad == 1 || quad == 2) ? -a : a) * p.amp;
  s = ((quad & 2) ? -b : b) * p.sin_amp;
}

template <bool F32>
struct Vec8;
template <>
struct Vec8<false> {
  u32x4 v;
  __device__ __forceinline__ void load(const void* base, int64_t e) {
    v = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(base) + e);
  }
  __device__ __forceinline__ void unpack(float (&f)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __builtin_bit_cast(float, v[i] << 16);
      f[2 * i + 1] = __builtin_bit_cast(float, v[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ void store(void* base, int64_t e, const float (&f)[8]) {
    bf16x8 b;
#pragma unroll
    for (int i = 0; i < 8; ++i) b[i] = (__bf16)f[i];
    *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(base) + e) = __builtin_bit_cast(u32x4, b);
  }
};
template <>
struct Vec8<true> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const void* base, int64_t e) {
    const f32x4* s = reinterpret_cast<const f32x4*>(static_cast<const float*>(base) + e);
    a = s[0];
    b = s[1];
  }
  __device__ __forceinline__ void unpack(float (&f)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[i] = a[i];
      f[4 + i] = b[i];
    }
  }
  static __device__ __forceinline__ void store(void* base, int64_t e, const float (&f)[8]) {
    f32x4* d = reinterpret_cast<f32x4*>(static_cast<float*>(base) + e);
    d[0] = f32x4{f[0], f[1], f[2], f[3]};
    d[1] = f32x4{f[4], f[5], f[6], f[7]};
  }
};

enum Layout { kInterleaved, kHalves };

// grid: x = blocks of rows (token, head split), y = batch.  Lanes run over the units
// of a row first, so neighbouring lanes read neighbouring bytes.
template <bool X32, bool Y32, int LAYOUT, int HEADS, int D>
__global__ __launch_bounds__(kThreads) void rope_kernel(const RopeParams p) {
  const int lrow = (int)threadIdx.x / p.units, u = (int)threadIdx.x - lrow * p.units;
  const uint32_t row = blockIdx.x * (uint32_t)p.rows_per_block + lrow;
  if (lrow >= p.rows_per_block || row >= p.rows) return;
  const uint32_t tok = row / (uint32_t)p.splits;
  const int hs = (int)(row - tok * (uint32_t)p.splits);
  const int64_t b = blockIdx.y;
  const int64_t xo = b * p.x_sb + (int64_t)tok * p.x_st, yo = b * p.y_sb + (int64_t)tok * p.y_st;
  const int32_t* pos = p.pos + b * p.pos_sb + (int64_t)tok * p.n_axes;
  // halves: units below n_pairs / 8 hold the pairs of elements e0 + i and e0 + n_pairs + i,
  // the others 8 elements behind the pairs, which pass
  const bool two = LAYOUT == kHalves && u < p.n_pairs / 8;
  const int e0 = LAYOUT == kHalves && !two ? p.n_pairs + u * 8 : u * 8;
  Vec8<X32> in[HEADS], in2[HEADS];
#pragma unroll
  for (int k = 0; k < HEADS; ++k) {
    const int h = hs + k * p.splits;
    if (h < p.H) {
      in[k].load(p.x, xo + h * D + e0);
      if (two) in2[k].load(p.x, xo + h * D + e0 + p.n_pairs);
    }
  }
  constexpr int kPairs = LAYOUT == kHalves ? 8 : 4;
  const int pair0 = LAYOUT == kHalves ? u * 8 : u * 4;
  float c[kPairs], s[kPairs];
#pragma unroll
  for (int i = 0; i < kPairs; ++i)
    if (pair0 + i < p.n_pairs) turn(p, pos, pair0 + i, c[i], s[i]);
#pragma unroll
  for (int k = 0; k < HEADS; ++k) {
    const int h = hs + k * p.splits;
    if (h < p.H) {
      float f[8], g[8];
      in[k].unpack(f);
      if (LAYOUT == kInterleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (pair0 + i < p.n_pairs) {
            const float a0 = f[2 * i], b0 = f[2 * i + 1];
            f[2 * i] = a0 * c[i] - b0 * s[i];
            f[2 * i + 1] = a0 * s[i] + b0 * c[i];
          }
      } else if (two) {
        in2[k].unpack(g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float a0 = f[i], b0 = g[i];
          f[i] = a0 * c[i] - b0 * s[i];
          g[i] = a0 * s[i] + b0 * c[i];
        }
        Vec8<Y32>::store(p.y, yo + h * D + e0 + p.n_pairs, g);
      }
      Vec8<Y32>::store(p.y, yo + h * D + e0, f);
    }
  }
}

// Halves whose second one does not start on 8 elements (n_pairs not a multiple of
// 8): a unit is one pair, or one element behind the pairs.
template <bool X32, bool Y32, int D>
__global__ __launch_bounds__(kThreads) void rope_single_kernel(const RopeParams p) {
  const int lrow = (int)threadIdx.x / p.units, u = (int)threadIdx.x - lrow * p.units;
  const uint32_t row = blockIdx.x * (uint32_t)p.rows_per_block + lrow;
  if (lrow >= p.rows_per_block || row >= p.rows) return;
  const uint32_t tok = row / (uint32_t)p.splits;
  const int hs = (int)(row - tok * (uint32_t)p.splits);
  const int64_t b = blockIdx.y;
  const int64_t xo = b * p.x_sb + (int64_t)tok * p.x_st, yo = b * p.y_sb + (int64_t)tok * p.y_st;
  auto get = [&](int64_t e) {
    return X32 ? static_cast<const float*>(p.x)[e] : (float)static_cast<const __bf16*>(p.x)[e];
  };
  auto put = [&](int64_t e, float v) {
    if (Y32)
      static_cast<float*>(p.y)[e] = v;
    else
      static_cast<__bf16*>(p.y)[e] = (__bf16)v;
  };
  float c = 1.f, s = 0.f;
  if (u < p.n_pairs) turn(p, p.pos + b * p.pos_sb + (int64_t)tok * p.n_axes, u, c, s);
  for (int h = hs; h < p.H; h += p.splits) {
    if (u < p.n_pairs) {
      const float a0 = get(xo + h * D + u), b0 = get(xo + h * D + u + p.n_pairs);
      put(yo + h * D + u, a0 * c - b0 * s);
      put(yo + h * D + u + p.n_pairs, a0 * s + b0 * c);
    } else {
      put(yo + h * D + p.n_pairs + u, get(xo + h * D + p.n_pairs + u));
    }
  }
}

template <bool X32, bool Y32, int D>
void launch_t(const RopeParams& p, int layout, int heads, dim3 grid, hipStream_t stream) {
  const dim3 block(kThreads);
  auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, p); };
  if (layout < 0)
    run(rope_single_kernel<X32, Y32, D>);
  else if (layout == kInterleaved)
    heads == 1 ? run(rope_kernel<X32, Y32, kInterleaved, 1, D>) : run(rope_kernel<X32, Y32, kInterleaved, 4, D>);
  else
    heads == 1 ? run(rope_kernel<X32, Y32, kHalves, 1, D>) : run(rope_kernel<X32, Y32, kHalves, 4, D>);
}

}  // namespace

hipError_t launch_rope(const RopeArgs& a, hipStream_t stream) {
  RopeParams p;
  p.x = a.x; p.y = a.y;
  p.x_sb = a.x_sb; p.x_st = a.x_st; p.y_sb = a.y_sb; p.y_st = a.y_st;
  p.pos = a.positions;
  p.pos_sb = a.pos_sb;
  p.f = a.inv_freq;
  p.n_axes = (int32_t)a.n_axes;
  p.split1 = (int32_t)a.split1;
  p.split2 = (int32_t)a.split2;
  p.n_pairs = (int32_t)a.n_pairs;
  p.H = (int32_t)a.H;
  p.amp = a.amplitude;
  p.sin_amp = a.inverse ? -a.amplitude : a.amplitude;
  const int d = (int)a.d;
  const bool single = !a.interleaved && a.n_pairs % 8 != 0;
  // units of a head: 8 elements each; halves: 8 pairs, then 8 elements behind them
  p.units = single ? d - p.n_pairs : (a.interleaved ? d / 8 : (d - p.n_pairs) / 8);
  p.rows_per_block = kThreads / p.units;
  // one head a thread while that does not fill the chip, four from there
  const int heads = a.B * a.N * a.H * p.units <= 256 * 2048 ? 1 : 4;
  p.splits = (int32_t)((a.H + heads - 1) / heads);
  p.rows = (uint32_t)(a.N * p.splits);
  const dim3 grid((unsigned)((p.rows + p.rows_per_block - 1) / p.rows_per_block), (unsigned)a.B);
  const int layout = single ? -1 : (a.interleaved ? kInterleaved : kHalves);
#define FASTVR_ROPE_T(X, Y) \
  (d == 128 ? launch_t<X, Y, 128>(p, layout, heads, grid, stream) : launch_t<X, Y, 64>(p, layout, heads, grid, stream))
  if (a.x_fp32)
    a.y_fp32 ? FASTVR_ROPE_T(true, true) : FASTVR_ROPE_T(true, false);
  else
    a.y_fp32 ? FASTVR_ROPE_T(false, true) : FASTVR_ROPE_T(false, false);
#undef FASTVR_ROPE_T
  return hipGetLastError();
}

}  // namespace fastvr
