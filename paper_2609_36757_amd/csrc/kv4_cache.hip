// Append to and read back a KV cache in 4 bits (format: fastvr.h).
//
// Append: per block of 32 elements the largest magnitude a (an integer maximum over
// the bf16 bits without sign: it orders infinities and NaN above all numbers); its
// exponent E and the leading mantissa bits give the scale byte, E - 2, one more from
// a mantissa of 1.75 on, at least 2 and at most 252 (so that all values are normal
// bf16 numbers); the elements go through the converting instruction, which divides by
// the power of two and rounds to nearest even (its results equal the format's rounding
// for every bf16 number, subnormal quotients and saturation among them).
//
// Both kernels are bound by HBM bandwidth: 2 bytes an element on the bf16 side, 0.53
// on the cache's; 16320 tokens of 12 heads (127 MB) are appended in 23.8 us (5.3 TB/s)
// and read back in 20.0 us (6.3 TB/s), one token of 16 sequences in 3.3 and 2.4 us, a
// launch.  A lane takes 8 elements, 16 (8) lanes a token row of head_dim 128 (64),
// four lanes a block; lanes run over the tokens of one head, whose codes are
// contiguous in the cache.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gfx950_ops.h"
#include "kv4.h"
#include "launch.h"

namespace fastvr {
namespace {

using namespace dev;

constexpr int kThreads = 256;
constexpr int kUnroll = 4;

struct CopyParams {
  uint8_t* codes[2];   // K, V
  uint8_t* scales[2];
  uint16_t* rows[2];   // bf16 rows
  int64_t sb[2], st[2];
  const int32_t* starts;
  int32_t H, capacity, first, n;
};

// maximum over the four lanes of a block
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  uint32_t o = (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xf, 0xf, true);  // lanes 1 0 3 2
  x = o > x ? o : x;
  o = (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xf, 0xf, true);  // lanes 2 3 0 1
  return o > x ? o : x;
}

// grid: x = groups of kUnroll * kThreads / (D / 8) tokens, y = head, z = 2 * batch + (0: K, 1: V)
template <int D>
__global__ __launch_bounds__(kThreads) void kv4_append_kernel(const CopyParams p) {
  constexpr int kLanes = D / 8, kTok = kThreads / kLanes;
  const int kv = blockIdx.z & 1, h = blockIdx.y;
  const int64_t b = blockIdx.z >> 1;
  const int u = threadIdx.x % kLanes;
  const int t0 = (int)(blockIdx.x * (kTok * kUnroll) + threadIdx.x / kLanes);
  const int64_t first = p.starts != nullptr ? p.starts[b] : p.first;
  const uint16_t* src = p.rows[kv] + b * p.sb[kv] + (int64_t)h * D + u * 8;
  const int64_t slab = (b * p.H + h) * p.capacity;
  u32x4 x[kUnroll];
#pragma unroll
  for (int k = 0; k < kUnroll; ++k) {
    const int t = t0 + k * kTok;
    x[k] = u32x4{};
    if (t < p.n) x[k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src + (int64_t)t * p.st[kv]));
  }
#pragma unroll
  for (int k = 0; k < kUnroll; ++k) {
    const int t = t0 + k * kTok;
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = x[k][i] & 0x7fffu, hi = (x[k][i] >> 16) & 0x7fffu;
      a = a > lo ? a : lo;
      a = a > hi ? a : hi;
    }
    a = quad_max(a);
    const bool bad = a >= 0x7f80u;
    int e = (int)(a >> 7) - 2 + ((a & 127u) >= 96u ? 1 : 0);
    e = e < 2 ? 2 : (e > 252 ? 252 : e);
    const float scale = kv4_scale((uint32_t)e);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (uint32_t)x[k][0]), scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (uint32_t)x[k][1]), scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (uint32_t)x[k][2]), scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (uint32_t)x[k][3]), scale, 3);
    const int64_t row = first + t;
    if (t < p.n && row >= 0 && row < p.capacity) {
      *reinterpret_cast<uint32_t*>(p.codes[kv] + (slab + row) * (D / 2) + u * 4) = bad ? 0u : c;
      if ((u & 3) == 0) p.scales[kv][(slab + row) * (D / 32) + (u >> 2)] = bad ? 255 : (uint8_t)e;
    }
  }
}

template <int D>
__global__ __launch_bounds__(kThreads) void kv4_read_kernel(const CopyParams p) {
  constexpr int kLanes = D / 8, kTok = kThreads / kLanes;
  const int kv = blockIdx.z & 1, h = blockIdx.y;
  const int64_t b = blockIdx.z >> 1;
  const int u = threadIdx.x % kLanes;
  const int t0 = (int)(blockIdx.x * (kTok * kUnroll) + threadIdx.x / kLanes);
  const int64_t first = p.starts != nullptr ? p.starts[b] : p.first;
  uint16_t* dst = p.rows[kv] + b * p.sb[kv] + (int64_t)h * D + u * 8;
  const int64_t slab = (b * p.H + h) * p.capacity;
  uint32_t c[kUnroll], s[kUnroll];
#pragma unroll
  for (int k = 0; k < kUnroll; ++k) {
    const int t = t0 + k * kTok;
    const int64_t row = first + t;
    c[k] = 0;
    s[k] = 127;
    if (t < p.n && row >= 0 && row < p.capacity) {
      c[k] = *reinterpret_cast<const uint32_t*>(p.codes[kv] + (slab + row) * (D / 2) + u * 4);
      s[k] = p.scales[kv][(slab + row) * (D / 32) + (u >> 2)];
    }
  }
#pragma unroll
  for (int k = 0; k < kUnroll; ++k) {
    const int t = t0 + k * kTok;
    if (t < p.n) *reinterpret_cast<u32x4*>(dst + (int64_t)t * p.st[kv]) = kv4_values(c[k], kv4_scale(s[k]));
  }
}

void fill(const Kv4CopyArgs& a, CopyParams& p, dim3& grid) {
  p.codes[0] = static_cast<uint8_t*>(a.cache.k_codes);
  p.codes[1] = static_cast<uint8_t*>(a.cache.v_codes);
  p.scales[0] = static_cast<uint8_t*>(a.cache.k_scales);
  p.scales[1] = static_cast<uint8_t*>(a.cache.v_scales);
  p.rows[0] = static_cast<uint16_t*>(a.k);
  p.rows[1] = static_cast<uint16_t*>(a.v);
  p.sb[0] = a.k_sb; p.sb[1] = a.v_sb;
  p.st[0] = a.k_st; p.st[1] = a.v_st;
  p.starts = a.starts;
  p.H = (int32_t)a.H;
  p.capacity = (int32_t)a.capacity;
  p.first = (int32_t)a.first;
  p.n = (int32_t)a.n;
  const int64_t group = kUnroll * kThreads / (a.d / 8);
  grid = dim3((unsigned)((a.n + group - 1) / group), (unsigned)a.H, (unsigned)(2 * a.B));
}

}  // namespace

hipError_t launch_kv4_append(const Kv4CopyArgs& a, hipStream_t stream) {
  CopyParams p;
  dim3 grid;
  fill(a, p, grid);
  if (a.d == 128)
    hipLaunchKernelGGL(kv4_append_kernel<128>, grid, dim3(kThreads), 0, stream, p);
  else
    hipLaunchKernelGGL(kv4_append_kernel<64>, grid, dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

hipError_t launch_kv4_read(const Kv4CopyArgs& a, hipStream_t stream) {
  CopyParams p;
  dim3 grid;
  fill(a, p, grid);
  if (a.d == 128)
    hipLaunchKernelGGL(kv4_read_kernel<128>, grid, dim3(kThreads), 0, stream, p);
  else
    hipLaunchKernelGGL(kv4_read_kernel<64>, grid, dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

}  // namespace fastvr
