// Rotary positions of query and key heads, and their gradient (the turn by the
// negative angle).
//
// Pair p of a token turns by theta = position * inv_freq[p].  The angle is taken in
// quarter turns in fp64, t = position * (inv_freq[p] * 2 / pi): its nearest integer
// gives the quadrant, the rest r in [-1/2, 1/2] goes to fp32, so far positions keep an
// absolute angle error below 1e-7 + 3.4e-16 * |position * inv_freq[p]| radians (three
// roundings in fp64, of 2^-53 each).  sin and cos of
// r * pi / 2 are their Taylor sums (to r^9 and r^10: the first terms left out are
// below 2e-9 and 5e-10).
//
// The kernel is bound by HBM bandwidth: x is read and y written once.  A thread
// takes one unit of a token, 8 (fp32: 4) elements of a head (interleaved) or twice as
// many (halves), for one head or four: its sines and cosines are taken once for all of
// them, while their loads are in flight.  65280 tokens of 12 heads in bf16 (402 MB):
// 73 us, 5.5 TB/s, as a copy of that size; 18720 tokens in fp32 (230 MB) 45 us, 5.1
// TB/s.  (Non-temporal stores gain 4 to 14% alone, and lose it in what reads y next.)
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

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
  uint32_t N;
  int32_t H, splits;  // a thread takes heads hs, hs + splits, ...
  float amp, sin_amp;  // sin_amp: negative for the inverse turn
};

// amplitude * (cos, sin) of pair p, of frequency f, of a token at positions pos
__device__ __forceinline__ void turn(const RopeParams& p, const double (&pos)[3], double f, int pair, float& c, float& s) {
  const double at = pair < p.split1 ? pos[0] : (pair < p.split2 ? pos[1] : pos[2]);
  const double t = at * (f * 0.63661977236758134308);  // quarter turns
  // adding 1.5 * 2^52 rounds to an integer, whose low bits are the sum's
  const double sum = t + 6755399441055744.0;
  const uint32_t quad = (uint32_t)__builtin_bit_cast(uint64_t, sum);
  const float r = (float)(t - (sum - 6755399441055744.0));
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
  c = (((quad + 1) & 2) ? -a : a) * p.amp;
  s = ((quad & 2) ? -b : b) * p.sin_amp;
}

__device__ __forceinline__ void positions(const RopeParams& p, int64_t b, int64_t tok, double (&pos)[3]) {
  const int32_t* src = p.pos + b * p.pos_sb + tok * p.n_axes;
  pos[0] = src[0];
  pos[1] = pos[2] = 0.0;
  if (p.n_axes > 1) pos[1] = src[1];
  if (p.n_axes > 2) pos[2] = src[2];
}

// E elements of a head: 8 where x and y are bf16, else 4, so that the wider side takes
// 16 bytes a lane and a wave's instruction one kilobyte in a row.
template <bool F32, int E>
struct Vec {
  typedef uint32_t Raw __attribute__((ext_vector_type(E / 2)));
  Raw v;
  __device__ __forceinline__ void load(const void* base, int64_t e) {
    v = *reinterpret_cast<const Raw*>(static_cast<const uint16_t*>(base) + e);
  }
  __device__ __forceinline__ void unpack(float (&f)[E]) const {
#pragma unroll
    for (int i = 0; i < E / 2; ++i) {
      f[2 * i] = __builtin_bit_cast(float, v[i] << 16);
      f[2 * i + 1] = __builtin_bit_cast(float, v[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ void store(void* base, int64_t e, const float (&f)[E]) {
    typedef __bf16 Out __attribute__((ext_vector_type(E)));
    Out b;
#pragma unroll
    for (int i = 0; i < E; ++i) b[i] = (__bf16)f[i];
    *reinterpret_cast<Raw*>(static_cast<uint16_t*>(base) + e) = __builtin_bit_cast(Raw, b);
  }
};
template <>
struct Vec<true, 4> {
  f32x4 v;
  __device__ __forceinline__ void load(const void* base, int64_t e) {
    v = *reinterpret_cast<const f32x4*>(static_cast<const float*>(base) + e);
  }
  __device__ __forceinline__ void unpack(float (&f)[4]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = v[i];
  }
  static __device__ __forceinline__ void store(void* base, int64_t e, const float (&f)[4]) {
    *reinterpret_cast<f32x4*>(static_cast<float*>(base) + e) = f32x4{f[0], f[1], f[2], f[3]};
  }
};

enum Layout { kInterleaved, kHalves };
template <bool X32, bool Y32>
constexpr int kUnit = X32 || Y32 ? 4 : 8;

// Block: x = unit of a head, y = head split, z = token; grid: x = token blocks, y = blocks
// of head splits, z = batch.  Neighbouring lanes read neighbouring bytes.
template <bool X32, bool Y32, int LAYOUT, int HEADS, int D>
__global__ __launch_bounds__(kThreads) void rope_kernel(const RopeParams p) {
  const int u = threadIdx.x, hs = (int)(blockIdx.y * blockDim.y + threadIdx.y);
  const uint32_t tok = blockIdx.x * blockDim.z + threadIdx.z;
  if (tok >= p.N || hs >= p.splits) return;
  const int64_t b = blockIdx.z;
  const int64_t xo = b * p.x_sb + (int64_t)tok * p.x_st, yo = b * p.y_sb + (int64_t)tok * p.y_st;
  constexpr int E = kUnit<X32, Y32>;
  // halves: units below n_pairs / E hold the pairs of elements e0 + i and e0 + n_pairs + i,
  // the others E elements behind the pairs, which pass
  const bool two = LAYOUT == kHalves && u < p.n_pairs / E;
  const int e0 = LAYOUT == kHalves && !two ? p.n_pairs + u * E : u * E;
  Vec<X32, E> in[HEADS], in2[HEADS];
#pragma unroll
  for (int k = 0; k < HEADS; ++k) {
    const int h = hs + k * p.splits;
    if (h < p.H) {
      in[k].load(p.x, xo + h * D + e0);
      if (two) in2[k].load(p.x, xo + h * D + e0 + p.n_pairs);
    }
  }
  constexpr int kPairs = LAYOUT == kHalves ? E : E / 2;
  const int pair0 = u * kPairs;
  float c[kPairs], s[kPairs];
  if (pair0 < p.n_pairs) {
    double pos[3], f[kPairs];
    positions(p, b, tok, pos);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) f[i] = p.f[pair0 + i < p.n_pairs ? pair0 + i : pair0];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) turn(p, pos, f[i], pair0 + i, c[i], s[i]);
  }
#pragma unroll
  for (int k = 0; k < HEADS; ++k) {
    const int h = hs + k * p.splits;
    if (h < p.H) {
      float f[E], g[E];
      in[k].unpack(f);
      if (LAYOUT == kInterleaved) {
#pragma unroll
        for (int i = 0; i < E / 2; ++i)
          if (pair0 + i < p.n_pairs) {
            const float a0 = f[2 * i], b0 = f[2 * i + 1];
            f[2 * i] = a0 * c[i] - b0 * s[i];
            f[2 * i + 1] = a0 * s[i] + b0 * c[i];
          }
      } else if (two) {
        in2[k].unpack(g);
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const float a0 = f[i], b0 = g[i];
          f[i] = a0 * c[i] - b0 * s[i];
          g[i] = a0 * s[i] + b0 * c[i];
        }
        Vec<Y32, E>::store(p.y, yo + h * D + e0 + p.n_pairs, g);
      }
      Vec<Y32, E>::store(p.y, yo + h * D + e0, f);
    }
  }
}

// Halves whose second one does not start on a unit (n_pairs not a multiple of its
// elements): a thread turns the E elements of its own unit, and takes their partners, at any
// place of the row, from LDS.  A block's rows are whole heads, and all of them are read
// before the first is written, so y may be x here too.  90 of 128 elements turned, 65280 tokens of
// 12 heads (401 MB): 82 to 92 us, 4.4 to 4.9 TB/s, with vector instructions issuing in 86% of
// the cycles: each sine is taken twice (205 us with one pair a thread).
template <bool X32, bool Y32, int HEADS, int D>
__global__ __launch_bounds__(kThreads) void rope_ragged_kernel(const RopeParams p) {
  constexpr int E = kUnit<X32, Y32>, kUnits = D / E;
  typedef typename std::conditional<X32, float, __bf16>::type X;
  __shared__ __attribute__((aligned(16))) X sm[HEADS][kThreads / kUnits][D];
  const int u = threadIdx.x, hs = (int)(blockIdx.y * blockDim.y + threadIdx.y);
  const int row = (int)(threadIdx.z * blockDim.y + threadIdx.y);
  const uint32_t tok = blockIdx.x * blockDim.z + threadIdx.z;
  const bool live = tok < p.N && hs < p.splits;
  const int64_t b = blockIdx.z;
  const int64_t xo = b * p.x_sb + (int64_t)tok * p.x_st, yo = b * p.y_sb + (int64_t)tok * p.y_st;
  const int e0 = u * E;
  Vec<X32, E> in[HEADS];
#pragma unroll
  for (int k = 0; k < HEADS; ++k) {
    const int h = hs + k * p.splits;
    if (live && h < p.H) in[k].load(p.x, xo + h * D + e0);
  }
  float c[E], s[E];
  if (live && e0 < 2 * p.n_pairs) {
    double pos[3], f[E];
    positions(p, b, tok, pos);
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int e = e0 + i, pair = e < p.n_pairs ? e : (e < 2 * p.n_pairs ? e - p.n_pairs : 0);
      f[i] = p.f[pair];
    }
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const int e = e0 + i;
      turn(p, pos, f[i], e < p.n_pairs ? e : e - p.n_pairs, c[i], s[i]);
      s[i] = e < p.n_pairs ? -s[i] : s[i];
    }
  }
#pragma unroll
  for (int k = 0; k < HEADS; ++k) {
    const int h = hs + k * p.splits;
    if (live && h < p.H) *reinterpret_cast<decltype(in[k].v)*>(&sm[k][row][e0]) = in[k].v;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < HEADS; ++k) {
    const int h = hs + k * p.splits;
    if (live && h < p.H) {
      float f[E];
      in[k].unpack(f);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const int e = e0 + i;
        if (e < 2 * p.n_pairs) f[i] = f[i] * c[i] + (float)sm[k][row][e < p.n_pairs ? e + p.n_pairs : e - p.n_pairs] * s[i];
      }
      Vec<Y32, E>::store(p.y, yo + h * D + e0, f);
    }
  }
}

template <bool X32, bool Y32, int D>
void launch_t(const RopeParams& p, int layout, int heads, dim3 grid, dim3 block, hipStream_t stream) {
  auto run = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, block, 0, stream, p); };
  if (layout < 0)
    heads == 1 ? run(rope_ragged_kernel<X32, Y32, 1, D>) : run(rope_ragged_kernel<X32, Y32, 4, D>);
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
  const int E = a.x_fp32 || a.y_fp32 ? 4 : 8;
  const bool ragged = !a.interleaved && a.n_pairs % E != 0;
  // units of a head: E elements each; halves on unit borders: E pairs, then E elements behind them
  const int units = a.interleaved || ragged ? d / E : (d - p.n_pairs) / E;
  // four heads a thread, for one taking of its sines, where that leaves a wave for every SIMD
  const int heads = a.B * a.N * a.H * units >= 4 * 65536 ? 4 : 1;
  p.splits = (int32_t)((a.H + heads - 1) / heads);
  p.N = (uint32_t)a.N;
  const int ny = p.splits < kThreads / units ? p.splits : kThreads / units, nz = kThreads / (units * ny);
  const dim3 block(units, ny, nz);
  const dim3 grid((unsigned)((a.N + nz - 1) / nz), (unsigned)((p.splits + ny - 1) / ny), (unsigned)a.B);
  const int layout = ragged ? -1 : (a.interleaved ? kInterleaved : kHalves);
#define FASTVR_ROPE_T(X, Y) \
  (d == 128 ? launch_t<X, Y, 128>(p, layout, heads, grid, block, stream) : launch_t<X, Y, 64>(p, layout, heads, grid, block, stream))
  if (a.x_fp32)
    a.y_fp32 ? FASTVR_ROPE_T(true, true) : FASTVR_ROPE_T(true, false);
  else
    a.y_fp32 ? FASTVR_ROPE_T(false, true) : FASTVR_ROPE_T(false, false);
#undef FASTVR_ROPE_T
  return hipGetLastError();
}

}  // namespace fastvr
