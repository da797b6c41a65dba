// Attention over a KV cache in 4 bits: from one token of each sequence to whole
// chunks, with grouped heads and a length per sequence.
//
//   O_i = sum_j exp(scale q_i . k_j - LSE_i) v_j,  LSE_i = ln sum_j exp(scale q_i . k_j)
//
// over the keys that row i sees, a contiguous interval [lo_i, hi_i).  The rows of one
// key head are (token, head of the group) pairs in that order, so lo and hi do not
// fall from row to row.  A workgroup takes 16, 32 or 64 rows (QT row tiles) of one
// (batch, key head) and a share of the keys that they see; its four waves take steps
// of 32 keys in turn, each with its own running maximum, sum and O, and join them
// through LDS.  Where these workgroups are few, the keys are split over several of
// them and a second kernel joins their partial results (kv4_plan.h).
//
// A step, one wave: S^T = K Q^T and O^T += V^T P^T with v_mfma_f32_16x16x32_bf16.
//  * K comes from the cache straight into registers: a lane holds a quarter of a key
//    row, which four (two) converting instructions per dword turn into the A operand
//    in place (the order of head_dim along the reduction is free, Q is loaded in the
//    same one).
//  * S^T puts one row of the tile on a lane and 8 of the 32 keys on each of the four
//    lanes of that row; rounded to bf16 these 8 are the B operand of O^T as they are,
//    when V's operand holds the same 8 keys: two runs of 4.
//  * V: a lane converts the same 8 (4) elements of those 8 keys and swaps halves
//    between neighbouring keys (v_perm) to get, per element, 8 keys in a row.
//  * The maximum a row is measured against is raised only when a score exceeds it by
//    8 (in log2 units: P <= 2^8 then), so that most steps need no exchange between
//    lanes and no rescale of O.
// What is rounded: P enters the products as a sum of two bf16 numbers, the second one
// the rest of the first one's rounding, so a weight is off by 2^-16 of itself; with four
// row tiles and O in bf16 as one, off by half a step, 2^-8, the rounding that the caller
// asks of O.  (The second part takes half as many matrix instructions again and 20 vector
// instructions a row tile: 16320 queries over 65280 keys of 12 heads 5.1 ms with one part,
// 6.9 with two.  Where rows are few it costs little: one query over 65280 keys 22.9 and
// 23.2 us; one row tile a workgroup with all CUs full, 1024 tokens that see the ones before
// them, 14.7 and 16.1; two, 32 queries over 65280 keys, 26.2 and 28.8.)  The sums l and all of
// S, LSE and O are fp32, and O is rounded where bf16 is asked for.  K and V are exact in
// bf16, so their products with Q and P are exact.  (The matrix instruction that takes
// 4-bit operands and block scales itself would save K's conversion, with Q in two 8-bit
// parts; its sums were off by 4e-5 of the largest, too much for LSE.)
//
// What bounds it.  One row tile (a token of each sequence): the cache's bytes; a step's
// 4.3 KB take longer than its 220 vector instructions and 384 cycles of matrix core.  One
// query over 65280 keys of 12 heads: 20.2 us for 107 MB (5.3 TB/s, a copy's rate), and 4
// us for the join.  Four row tiles: the issue of vector instructions (conversion, exp2,
// sums: 265 a step of 64 rows, beside 64 matrix instructions of 16 cycles).  Over 16320
// queries and 65280 keys of 12 heads vector and matrix instructions issue in 80% of the
// cycles and the matrix cores are busy in 57% (under the profiler, where a call takes 10%
// longer); 81% and 38% with head_dim 64.  That call takes 5.0 to 5.7 ms by card and scores, 1140 to
// 1310 TFLOP/s (a large bf16 GEMM reaches 1500, the bf16 forward on an expanded cache 1300).  What it took: Q in
// LDS and V's scales loaded late, for two waves on a SIMD without a spilled register (15.9 ms
// with one wave on a SIMD; 5.6 with two); products at a higher wave priority (5.4); V
// converted and paired between the products (5.1).
//
// Keys a row does not see: their P is zero, and in the steps where that can happen
// V blocks that are not finite (rows behind a sequence may hold anything) are taken
// as zero, and the O of the rows that do see them becomes NaN at the end.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "class_plan.h"
#include "gfx950_ops.h"
#include "kv4.h"
#include "kv4_plan.h"
#include "launch.h"

namespace fastvr {
namespace {

using namespace dev;

constexpr int kThreads = 64 * kKv4Waves;
constexpr float kInf = __builtin_inff();
constexpr float kSlack = 8.f;  // log2 units a score may exceed the running reference by
// Reference of a row that has seen no key: below all scores, and finite, so that no
// difference of two references is NaN; such a row's sum is 0.
constexpr float kNone = -3e38f;

struct Kv4Params {
  const uint16_t* q;
  int64_t q_sb;
  int32_t q_st;
  const uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
  void* o;
  int64_t o_sb;
  int32_t o_st;
  int32_t o_bf16;
  float* lse;
  // of the split tiles' rows: [row][split][D] unnormalised O, then [row][split] (maximum, sum)
  float* part;
  const int32_t* lens;
  int32_t B, H, Hkv, G, nq, R, capacity, cache_len, chunk_len, window;
  int32_t row_tiles, runs, whole, rest, n_split, units;  // rest: split tiles
  int32_t tile_rows;                               // rows with partial results in each of them
  int64_t rows;                                    // in all of them
  float c;  // |scale| * log2(e)
  uint32_t sign;  // flips q for a negative scale
};

__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                 0);
}

// x of the lanes l and l ^ 16, in both of them
__device__ __forceinline__ float swap_rows(float x, float* other) {
  const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x),
                                                  false, false);
  *other = __builtin_bit_cast(float, (uint32_t)r[1]);
  return __builtin_bit_cast(float, (uint32_t)r[0]);
}
// maximum and sum over the four lanes of a row
__device__ __forceinline__ float row_max4(float x) {
  float o;
  x = swap_rows(x, &o);
  x = __builtin_fmaxf(x, o);
  x = swap_halves(x, &o);
  return __builtin_fmaxf(x, o);
}
__device__ __forceinline__ float row_sum4(float x) {
  float o;
  x = swap_rows(x, &o);
  x += o;
  x = swap_halves(x, &o);
  return x + o;
}

// maximum and sum over a wave's lanes
template <int CTRL>
__device__ __forceinline__ float row_move(float x) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
constexpr int kQuad1032 = 0xB1, kQuad2301 = 0x4E, kRowRor4 = 0x124, kRowRor8 = 0x128;
__device__ __forceinline__ float wave_max(float x) {
  x = __builtin_fmaxf(x, row_move<kQuad1032>(x));
  x = __builtin_fmaxf(x, row_move<kQuad2301>(x));
  x = __builtin_fmaxf(x, row_move<kRowRor4>(x));
  x = __builtin_fmaxf(x, row_move<kRowRor8>(x));
  return row_max4(x);
}
__device__ __forceinline__ float wave_sum(float x) {
  x += row_move<kQuad1032>(x);
  x += row_move<kQuad2301>(x);
  x += row_move<kRowRor4>(x);
  x += row_move<kRowRor8>(x);
  x = row_sum4(x);  // (lanes add in different orders: one of them for all)
  return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x)));
}

template <int D>
struct Step {  // what a lane loads for 32 keys
  static constexpr int kK = D / 32;   // dwords of K a lane holds per key
  uint32_t k[2][kK];
  uint32_t ks[2];
  uint32_t v[8];
  uint32_t vs[8];  // scale bytes of a key: all four (head_dim 128), or this lane's
};

template <int D, int QT>
__global__ __launch_bounds__(kThreads, QT == 1 ? 4 : 2) void kv4_attn_kernel(const Kv4Params p) {
  constexpr int kE = D / 16;    // elements of V a lane holds per key; O^T tiles
  constexpr int kKK = D / 32;   // reduction steps of S
  constexpr int kPitch = D + 4;
  constexpr int kRows = 16 * QT;
  __shared__ __attribute__((aligned(16))) float sm_o[kKv4Waves * 16 * kPitch];
  __shared__ float sm_m[kKv4Waves * kRows], sm_l[kKv4Waves * kRows];
  __shared__ int sm_lo[kRows], sm_n[kRows];  // first key and number of keys that a row sees
  // four tiles: Q's operands stay in LDS, in the order the lanes read them
  constexpr bool kQLds = QT > 2;
  __shared__ u32x4 sm_q[kQLds ? QT * kKK * 64 : 1];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, g = lane >> 4;
  // workgroup -> tile of all (batch, key head)s' row tiles, and split: first the whole tiles,
  // then the others, row_tiles of them at a time with all their splits.  Row tiles of one key range
  // run next to each other on one XCD and share its L2.
  const bool alone = (int)blockIdx.x < p.whole;
  const int blk = alone ? (int)blockIdx.x : (int)blockIdx.x - p.whole;
  int at = p.runs > 0 ? xcd_unit(blk, alone ? p.whole : p.units - p.whole) : blk, split = 0;
  if (!alone) {
    const int group = (int)((uint32_t)at / (uint32_t)(p.row_tiles * p.n_split)), first = group * p.row_tiles;
    const int n_here = p.rest - first < p.row_tiles ? p.rest - first : p.row_tiles;
    const int in = at - first * p.n_split;
    split = (int)((uint32_t)in / (uint32_t)n_here);
    at = p.whole + first + in - split * n_here;
  }
  const int n_split = alone ? 1 : p.n_split;
  const int bh = (int)((uint32_t)at / (uint32_t)p.row_tiles), tile = kv4_tile(at - bh * p.row_tiles, p.row_tiles, p.runs);
  const int b = (int)((uint32_t)bh / (uint32_t)p.Hkv), hk = bh - b * p.Hkv;
  int len = p.cache_len;
  if (p.lens != nullptr) {
    const int l = p.lens[b];
    len = l < 0 ? 0 : (l < len ? l : len);
  }

  // rows of this lane
  const int row0 = tile * kRows;
  const int row_last = (row0 + kRows < p.R ? row0 + kRows : p.R) - 1;
  int lo_min, hi_min, lo_max, hi_max;
  kv4_interval(len - p.nq + (int)((uint32_t)row0 / (uint32_t)p.G), len, p.chunk_len, p.window, &lo_min, &hi_min);
  kv4_interval(len - p.nq + (int)((uint32_t)row_last / (uint32_t)p.G), len, p.chunk_len, p.window, &lo_max, &hi_max);

  f32x4 acc[QT][kE];
  // reference in log2 units, the score from which it is raised, sum of this lane's keys
  float mc[QT], bound[QT], l[QT];
  const float inv_c = 1.0f / p.c;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    mc[t] = kNone;
    bound[t] = -kInf;
    l[t] = 0.f;
#pragma unroll
    for (int j = 0; j < kE; ++j) acc[t][j] = f32x4{};
  }

  const int64_t slab = (int64_t)bh * p.capacity;
  const __amdgpu_buffer_rsrc_t rkc = make_rsrc(p.k_codes + slab * (D / 2), (int64_t)p.capacity * (D / 2));
  const uint8_t* k_scales = p.k_scales + slab * (D / 32);
  const __amdgpu_buffer_rsrc_t rks = make_rsrc(p.k_scales + slab * (D / 32), (int64_t)p.capacity * (D / 32));
  const __amdgpu_buffer_rsrc_t rvc = make_rsrc(p.v_codes + slab * (D / 2), (int64_t)p.capacity * (D / 2));
  const __amdgpu_buffer_rsrc_t rvs = make_rsrc(p.v_scales + slab * (D / 32), (int64_t)p.capacity * (D / 32));
  // a lane's codes; its scale bytes are at 1 / 16 of these offsets (16 bytes of codes a scale)
  const uint32_t kc_off = n * (D / 2) + g * (D / 8), vc_off = 4 * g * (D / 2) + n * (D / 32);

  // The step's place goes into the scalar offset (below the slab's size), the rest are
  // lane offsets and immediates; rows behind the cache's capacity read as zero.  (Made
  // opaque, a lane offset is not added to each immediate ahead of the loop, which
  // takes a register per load.)
  Step<D> s;
  auto opaque = [](uint32_t x) {
    asm volatile("" : "+v"(x));
    return x;
  };
  auto load_k = [&](int st) {
    const int k0 = __builtin_amdgcn_readfirstlane(st * kKv4StepKeys);
    const uint32_t kc = opaque(kc_off), ks = (kc >> 4) & ~3u;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const uint32_t off = kc + 16 * x * (D / 2);
      if (D == 128) {
        const u32x4 w = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rkc, off, k0 * (D / 2), 0));
#pragma unroll
        for (int i = 0; i < kKK; ++i) s.k[x][i] = w[i];
      } else {
        const auto w = __builtin_amdgcn_raw_buffer_load_b64(rkc, off, k0 * (D / 2), 0);
#pragma unroll
        for (int i = 0; i < kKK; ++i) s.k[x][i] = w[i];
      }
      // the key's four scale bytes (head_dim 128), or this lane's one.  (The latter as an
      // ordinary load: of a buffer load's byte the compiler sinks the widening to the end
      // of the step, which then waits for it.)
      if (D == 128) {
        s.ks[x] = __builtin_amdgcn_raw_buffer_load_b32(rks, ks + 16 * x * (D / 32), k0 * (D / 32), 0);
      } else {
        const int key = k0 + 16 * x + n;
        s.ks[x] = k_scales[(uint32_t)(key < p.capacity ? key : p.capacity - 1) * (D / 32) + (g >> 1)];
      }
    }
  };
  // four tiles of head_dim 128: V's scales are loaded within their step, for want of registers
  constexpr bool kLateScales = D == 128 && QT > 2;
  auto load_vs = [&](int st) {
    const int k0 = __builtin_amdgcn_readfirstlane(st * kKv4StepKeys);
    const uint32_t vs = (opaque(vc_off) >> 4) & ~15u;
#pragma unroll
    for (int x = 0; x < 2; ++x) {  // (4-byte aligned: a slab's scales start at 4 * its rows)
      const u32x4 w = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rvs, vs + 64 * x, k0 * (D / 32), 0));
#pragma unroll
      for (int i = 0; i < 4; ++i) s.vs[4 * x + i] = w[i];
    }
  };
  auto load_v = [&](int st) {
    const int k0 = __builtin_amdgcn_readfirstlane(st * kKv4StepKeys);
    const uint32_t vc = opaque(vc_off);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t key = (i & 3) + 16 * (i >> 2);
      if (D == 128) {
        s.v[i] = __builtin_amdgcn_raw_buffer_load_b32(rvc, vc + key * (D / 2), k0 * (D / 2), 0);
      } else {
        s.v[i] = __builtin_amdgcn_raw_buffer_load_b16(rvc, vc + key * (D / 2), k0 * (D / 2), 0);
        s.vs[i] = __builtin_amdgcn_raw_buffer_load_b8(rvs, (vc >> 4) + key * (D / 32), k0 * (D / 32), 0);
      }
    }
    if (D == 128 && !kLateScales) load_vs(st);
  };
  const uint32_t vs_shift = 8 * (n >> 2), ks_shift = 8 * g;
  auto k_byte = [&](int x) { return D == 128 ? __builtin_amdgcn_ubfe(s.ks[x], ks_shift, 8) : s.ks[x]; };
  auto v_byte = [&](int i) { return D == 128 ? __builtin_amdgcn_ubfe(s.vs[i], vs_shift, 8) : s.vs[i]; };

  // steps of this workgroup, [begin, end); in steps [in_lo, in_hi) all rows see all keys
  const int s0 = lo_min / kKv4StepKeys;
  const int n_steps = hi_max > lo_min ? (hi_max + kKv4StepKeys - 1) / kKv4StepKeys - s0 : 0;
  const int begin = s0 + kv4_split_at(n_steps, split, n_split);
  const int end = __builtin_amdgcn_readfirstlane(s0 + kv4_split_at(n_steps, split + 1, n_split));
  const int in_lo = (lo_max + kKv4StepKeys - 1) / kKv4StepKeys, in_hi = hi_min / kKv4StepKeys;
  int st = __builtin_amdgcn_readfirstlane(begin + wave);
  if (st < end) {
    load_k(st);
    load_v(st);
  }

  u32x4 q[kQLds ? 1 : QT][kKK];
  auto load_q = [&](int t, u32x4(&dst)[kKK]) {
    const int rt = row0 + t * 16 + n, r = rt <= row_last ? rt : row_last;
    const int i = (int)((uint32_t)r / (uint32_t)p.G), h = hk * p.G + r - i * p.G;
    const uint16_t* src = p.q + (int64_t)b * p.q_sb + (int64_t)i * p.q_st + h * D + g * (D / 4);
#pragma unroll
    for (int kk = 0; kk < kKK; ++kk) dst[kk] = *reinterpret_cast<const u32x4*>(src + kk * 8) ^ p.sign;
  };
  if (kQLds) {
    static_assert(!kQLds || QT == kKv4Waves, "a wave brings one tile of Q");
    u32x4 mine[kKK];
    load_q(wave, mine);
#pragma unroll
    for (int kk = 0; kk < kKK; ++kk) sm_q[(wave * kKK + kk) * 64 + lane] = mine[kk];
  } else {
#pragma unroll
    for (int t = 0; t < QT; ++t) load_q(t, q[t]);
  }
  if (tid < kRows) {
    const int r = row0 + tid <= row_last ? row0 + tid : row_last;
    int lo, hi;
    kv4_interval(len - p.nq + (int)((uint32_t)r / (uint32_t)p.G), len, p.chunk_len, p.window, &lo, &hi);
    sm_lo[tid] = lo;
    sm_n[tid] = hi - lo;
  }
  __syncthreads();

  // A step in which some row does not see some key: scores to -inf, V blocks that are
  // not finite to zero; the O of rows that see such a block becomes NaN at the end.
  uint32_t spoilt = 0;  // a bit per tile
  auto mask = [&](int st, f32x4(&sc)[QT][2]) {
    const int k0 = st * kKv4StepKeys, n0 = opaque(n);
    const uint32_t one = opaque(D == 128 ? 0x7f7f7f7fu : 127u), zero = opaque(0u);
    bool nan_block = false;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (v_byte(i) > 252u) {
        nan_block = true;
        s.vs[i] = one;
        s.v[i] = zero;
      }
    const bool any_nan = __builtin_amdgcn_ballot_w64(nan_block) != 0;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const int lo = sm_lo[t * 16 + n0], seen = sm_n[t * 16 + n0], at = k0 + 4 * g - lo;
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          sc[t][x][i] = (uint32_t)(at + 16 * x + i) < (uint32_t)seen ? sc[t][x][i] : -kInf;
      if (any_nan) {
        // this lane's O of a tile is one 32-element block of one row: block g (head_dim 128), g / 2 (64)
#pragma clang loop unroll(disable)
        for (int key = k0; key < k0 + kKv4StepKeys; ++key) {
          const uint32_t byte = __builtin_amdgcn_raw_buffer_load_b8(
              rvs, (uint32_t)key * (D / 32) + (D == 128 ? g : g >> 1), 0, 0);
          if (byte > 252u && (uint32_t)(key - lo) < (uint32_t)seen) spoilt |= 1u << t;
        }
      }
    }
  };

  // Step st; the loads of step nx take the place of what has been used.
  auto step = [&](int st, int nx, bool masked, auto parts) {
    constexpr bool kTwo = decltype(parts)::value == 2;  // P as a sum of two bf16 numbers
    __builtin_amdgcn_s_setprio(1);
    const uint32_t q_lane = opaque(lane);  // (Q in LDS is read anew in each step)
    f32x4 sc[QT][2];
    const float scale[2] = {kv4_scale(k_byte(0)), kv4_scale(k_byte(1))};
#pragma unroll
    for (int kk = 0; kk < kKK; ++kk) {
      const u32x4 a[2] = {kv4_values(s.k[0][kk], scale[0]), kv4_values(s.k[1][kk], scale[1])};
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        const u32x4 qf = kQLds ? sm_q[(t * kKK + kk) * 64 + q_lane] : q[kQLds ? 0 : t][kk];
#pragma unroll
        for (int x = 0; x < 2; ++x) sc[t][x] = mfma16(a[x], qf, kk == 0 ? f32x4{} : sc[t][x]);
      }
      // (no more of Q in registers than the next reduction step)
      if (kQLds && kk % 2 == 1) __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
    if (kLateScales) load_vs(st);
    load_k(nx);
    if (QT > 2) __builtin_amdgcn_sched_barrier(0);
    if (masked) mask(st, sc);
    float m[QT];
    bool raise = false;
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      m[t] = -kInf;
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r) m[t] = __builtin_fmaxf(m[t], sc[t][x][r]);
      raise |= m[t] > bound[t];
    }
    if (__builtin_amdgcn_ballot_w64(raise)) {
      // raise the reference of the rows that need it to their maximum so far, those alone: a
      // row's bits depend on the keys that it sees only (NaN scores raise nothing)
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        const float top = row_max4(m[t]), m_new = top > bound[t] ? top * p.c : mc[t];
        const float alpha = __builtin_amdgcn_exp2f(mc[t] - m_new);
        mc[t] = m_new;
        bound[t] = top > bound[t] ? (m_new + kSlack) * inv_c : bound[t];
        l[t] *= alpha;
#pragma unroll
        for (int j = 0; j < kE; ++j) acc[t][j] *= alpha;
      }
    }
    u32x4 pf[QT], rest[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      float e[8], sum = 0.f;
      bf16x8 pb;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][i >> 2][i & 3], p.c, -mc[t]));  // 0 where masked
        sum += e[i];
        pb[i] = (__bf16)e[i];
      }
      l[t] += sum;
      pf[t] = __builtin_bit_cast(u32x4, pb);
      if (kTwo) {
        // (from the packed pairs: of single elements the compiler converts each once more)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t pair = pf[t][i >> 1];
          pb[i] = (__bf16)(e[i] - __builtin_bit_cast(float, (i & 1) ? pair & 0xffff0000u : pair << 16));
        }
        rest[t] = __builtin_bit_cast(u32x4, pb);
      }
    }
    if (QT > 2) __builtin_amdgcn_sched_barrier(0);  // one phase's registers at a time
    // V: keys 4 g + (0..3) and 16 + 4 g + (0..3), elements n * kE ..; two elements of the 8
    // keys at a time are converted and paired while the last two's products run
    __builtin_amdgcn_s_setprio(1);
    uint32_t code[8];
    float v_scale[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      code[i] = s.v[i];
      v_scale[i] = kv4_scale(v_byte(i));
    }
    load_v(nx);
    auto two = [&](auto pair) {
      constexpr int P = decltype(pair)::value;
      uint32_t w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = kv4_pair<P>(code[i], v_scale[i]);
      u32x4 a[2];
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          a[j][i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], j ? 0x07060302u : 0x05040100u);
      // (one tile: an accumulator's two products are not neighbours)
      constexpr int kAtOnce = QT == 1 ? 2 : 1;
#pragma unroll
      for (int j0 = 0; j0 < 2; j0 += kAtOnce)
#pragma unroll
        for (int part = 0; part < (kTwo ? 2 : 1); ++part)
#pragma unroll
          for (int j = j0; j < j0 + kAtOnce; ++j)
#pragma unroll
            for (int t = 0; t < QT; ++t)
              acc[t][2 * P + j] = mfma16(a[j], part == 0 ? pf[t] : rest[t], acc[t][2 * P + j]);
    };
    two(std::integral_constant<int, 0>{});
    two(std::integral_constant<int, 1>{});
    if (D == 128) {
      two(std::integral_constant<int, kE / 2 - 2>{});
      two(std::integral_constant<int, kE / 2 - 1>{});
    }
    __builtin_amdgcn_sched_group_barrier(SCHED_VALU, 32, 0);
#pragma unroll
    for (int i = 0; i < QT * kE; ++i) {
      __builtin_amdgcn_sched_group_barrier(SCHED_MFMA, kTwo ? 2 : 1, 0);
      __builtin_amdgcn_sched_group_barrier(SCHED_VALU, 8 / QT, 0);
    }
  };

  // What the loop carries of V's bytes and halves (head_dim 64) must be dwords: the compiler
  // otherwise carries them narrow, and widens, so waits for, each load at the end of the
  // step that issues it.  One value in each that is no extended byte prevents that.
  if (D == 64 && st < end) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      s.v[i] = opaque(s.v[i]);
      s.vs[i] = opaque(s.vs[i]);
    }
  }
  // (two loops one behind the other, of which one runs: as the two sides of a branch they spill)
  const int one_end = __builtin_amdgcn_readfirstlane(QT == 4 && p.o_bf16 ? end : 0);
  // (the last step loads itself once more)
  if (QT == 4)
    for (; st < one_end; st += kKv4Waves)
      step(st, st + kKv4Waves < end ? st + kKv4Waves : st, st < in_lo || st >= in_hi, std::integral_constant<int, 1>{});
  for (; st < end; st += kKv4Waves)
    step(st, st + kKv4Waves < end ? st + kKv4Waves : st, st < in_lo || st >= in_hi, std::integral_constant<int, 2>{});

  // join the waves
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    l[t] = row_sum4(l[t]);
    if (g == 0) {
      sm_m[wave * kRows + t * 16 + n] = mc[t];
      sm_l[wave * kRows + t * 16 + n] = l[t];
    }
  }
  // (a loop, though tiles are picked by constants: each unrolled round's instructions would
  // be fetched for one use, 1.1 us a round)
#pragma clang loop unroll(disable)
  for (int t = 0; t < QT; ++t) {
    __syncthreads();
    {
      float m = kNone;
#pragma unroll
      for (int w = 0; w < kKv4Waves; ++w) m = __builtin_fmaxf(m, sm_m[w * kRows + t * 16 + n]);
      const float own = sm_m[wave * kRows + t * 16 + n];
      const float f = (spoilt >> t & 1) ? __builtin_nanf("") : __builtin_amdgcn_exp2f(own - m);
      float* dst = sm_o + (wave * 16 + n) * kPitch;
      // element n' * kE + j of O^T row n' = 4 g + r
#pragma unroll
      for (int x = 0; x < QT; ++x)
        if (x == t)
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < kE; j += 4)
              *reinterpret_cast<f32x4*>(dst + (4 * g + r) * kE + j) =
                  f32x4{acc[x][j][r] * f, acc[x][j + 1][r] * f, acc[x][j + 2][r] * f, acc[x][j + 3][r] * f};
    }
    __syncthreads();
    const int rr = tid >> 4, e0 = (tid & 15) * kE;
    const int r = row0 + t * 16 + rr;
    if (r < p.R) {
      float m = kNone, sum = 0.f;
#pragma unroll
      for (int w = 0; w < kKv4Waves; ++w) m = __builtin_fmaxf(m, sm_m[w * kRows + t * 16 + rr]);
#pragma unroll
      for (int w = 0; w < kKv4Waves; ++w)
        sum += sm_l[w * kRows + t * 16 + rr] * __builtin_amdgcn_exp2f(sm_m[w * kRows + t * 16 + rr] - m);
      float v[kE];
#pragma unroll
      for (int j = 0; j < kE; ++j) {
        v[j] = 0.f;
#pragma unroll
        for (int w = 0; w < kKv4Waves; ++w) v[j] += sm_o[(w * 16 + rr) * kPitch + e0 + j];
      }
      if (!alone) {
        const int64_t row = (int64_t)(at - p.whole) * p.tile_rows + t * 16 + rr;
        float* dst = p.part + (row * p.n_split + split) * D + e0;
#pragma unroll
        for (int j = 0; j < kE; j += 4) *reinterpret_cast<f32x4*>(dst + j) = f32x4{v[j], v[j + 1], v[j + 2], v[j + 3]};
        if (e0 == 0) {
          float* ml = p.part + p.rows * p.n_split * D + (row * p.n_split + split) * 2;
          ml[0] = m;
          ml[1] = sum;
        }
      } else {
        const int i = (int)((uint32_t)r / (uint32_t)p.G), h = hk * p.G + r - i * p.G;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        const int64_t e = (int64_t)b * p.o_sb + (int64_t)i * p.o_st + h * D + e0;
        if (p.o_bf16) {
          typedef __bf16 Row __attribute__((ext_vector_type(kE)));
          Row row;
#pragma unroll
          for (int j = 0; j < kE; ++j) row[j] = (__bf16)(v[j] * inv);
          *reinterpret_cast<Row*>(static_cast<__bf16*>(p.o) + e) = row;
        } else {
          float* dst = static_cast<float*>(p.o) + e;
#pragma unroll
          for (int j = 0; j < kE; j += 4)
            *reinterpret_cast<f32x4*>(dst + j) = f32x4{v[j] * inv, v[j + 1] * inv, v[j + 2] * inv, v[j + 3] * inv};
        }
        if (e0 == 0 && p.lse != nullptr)
          p.lse[((int64_t)b * p.H + h) * p.nq + i] = sum == 0.f ? -kInf : (m + __builtin_log2f(sum)) * kLn2;
      }
    }
  }
}

// Joins the partial results of a row's splits.  WAVES = 4: a workgroup a row, wave w taking
// the splits w, w + 4, ...; WAVES = 1, for up to 16 splits: a wave a row.  D / 64 elements a lane.
template <int D, int WAVES>
__global__ __launch_bounds__(kThreads) void kv4_join_kernel(const Kv4Params p) {
  constexpr int kE = D / 64, kMine = 16;
  static_assert(kMine * kKv4Waves == kKv4MaxSplit, "every split has a wave");
  __shared__ float sm[WAVES == 1 ? 1 : kKv4Waves][D];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // (32 bits: a launch has fewer than 2^24 workgroups)
  const uint32_t row32 = WAVES == 1 ? blockIdx.x * kKv4Waves + wave : blockIdx.x, row_tiles = p.row_tiles;
  const uint32_t j = row32 / (uint32_t)p.tile_rows, at = p.whole + j, bh = at / row_tiles;
  const int r = kv4_tile((int)(at - bh * row_tiles), p.row_tiles, p.runs) * p.tile_rows + (int)(row32 - j * p.tile_rows);
  const int64_t row = row32;
  // (whole waves, and with WAVES = 4 whole workgroups; the last tile of a head may have fewer rows)
  if (row >= p.rows || r >= p.R) return;
  const int first = WAVES == 1 ? 0 : wave;
  const float* src = p.part + row * p.n_split * D + lane * kE;
  float x[kMine][kE];
#pragma unroll
  for (int k = 0; k < kMine; ++k)
#pragma unroll
    for (int j = 0; j < kE; ++j) x[k][j] = k * WAVES + first < p.n_split ? src[(k * WAVES + first) * D + j] : 0.f;
  // lane s holds split s (n_split <= 64)
  const float* ml = p.part + p.rows * p.n_split * D + row * p.n_split * 2;
  const float m_s = lane < p.n_split ? ml[2 * lane] : kNone;
  const float l_s = lane < p.n_split ? ml[2 * lane + 1] : 0.f;
  const float m = wave_max(m_s);
  const float f = __builtin_amdgcn_exp2f(m_s - m);
  const float sum = wave_sum(l_s * f);
  float v[kE] = {};
#pragma unroll
  for (int k = 0; k < kMine; ++k) {
    const float w =
        __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), k * WAVES + first));
#pragma unroll
    for (int j = 0; j < kE; ++j) v[j] += w * x[k][j];
  }
  if (WAVES > 1) {
#pragma unroll
    for (int j = 0; j < kE; ++j) sm[wave][lane * kE + j] = v[j];
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int j = 0; j < kE; ++j)
      v[j] = (sm[0][lane * kE + j] + sm[1 % WAVES][lane * kE + j]) + (sm[2 % WAVES][lane * kE + j] + sm[3 % WAVES][lane * kE + j]);
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  const int b = (int)(bh / (uint32_t)p.Hkv), i = (int)((uint32_t)r / (uint32_t)p.G);
  const int h = ((int)bh - b * p.Hkv) * p.G + r - i * p.G;
  const int64_t e = (int64_t)b * p.o_sb + (int64_t)i * p.o_st + h * D + lane * kE;
#pragma unroll
  for (int j = 0; j < kE; ++j) {
    if (p.o_bf16)
      static_cast<__bf16*>(p.o)[e + j] = (__bf16)(v[j] * inv);
    else
      static_cast<float*>(p.o)[e + j] = v[j] * inv;
  }
  if (lane == 0 && p.lse != nullptr)
    p.lse[((int64_t)b * p.H + h) * p.nq + i] = sum == 0.f ? -kInf : (m + __builtin_log2f(sum)) * kLn2;
}

template <int D>
hipError_t launch_t(const Kv4Params& p, const Kv4Plan& plan, hipStream_t stream) {
  const dim3 grid((unsigned)plan.units), block(kThreads);
  if (plan.q_tiles == 4)
    hipLaunchKernelGGL((kv4_attn_kernel<D, 4>), grid, block, 0, stream, p);
  else if (plan.q_tiles == 2)
    hipLaunchKernelGGL((kv4_attn_kernel<D, 2>), grid, block, 0, stream, p);
  else
    hipLaunchKernelGGL((kv4_attn_kernel<D, 1>), grid, block, 0, stream, p);
  if (plan.n_split > 1) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (kv4_join_waves(plan) == 1)
      hipLaunchKernelGGL((kv4_join_kernel<D, 1>), dim3((unsigned)((plan.rows + kKv4Waves - 1) / kKv4Waves)), block, 0, stream,
                         p);
    else
      hipLaunchKernelGGL((kv4_join_kernel<D, 4>), dim3((unsigned)plan.rows), block, 0, stream, p);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv4_attn(const Kv4AttnArgs& a, hipStream_t stream) {
  const Kv4Plan& plan = a.plan;
  Kv4Params p;
  p.q = static_cast<const uint16_t*>(a.q);
  p.q_sb = a.q_sb;
  p.q_st = (int32_t)a.q_st;
  p.k_codes = static_cast<const uint8_t*>(a.cache.k_codes);
  p.k_scales = static_cast<const uint8_t*>(a.cache.k_scales);
  p.v_codes = static_cast<const uint8_t*>(a.cache.v_codes);
  p.v_scales = static_cast<const uint8_t*>(a.cache.v_scales);
  p.o = a.o;
  p.o_sb = a.o_sb;
  p.o_st = (int32_t)a.o_st;
  p.o_bf16 = a.o_bf16 ? 1 : 0;
  p.lse = a.lse;
  p.part = static_cast<float*>(a.workspace);
  p.lens = a.lens;
  p.B = (int32_t)a.B;
  p.H = (int32_t)a.H;
  p.Hkv = (int32_t)a.Hkv;
  p.G = (int32_t)(a.H / a.Hkv);
  p.nq = (int32_t)a.nq;
  p.R = (int32_t)(a.nq * p.G);
  p.capacity = (int32_t)a.capacity;
  p.cache_len = (int32_t)a.cache_len;
  // a chunk longer than the cache is a chunk of the whole cache, a window past the
  // first chunk unbounded
  const int64_t L = a.chunk_len > a.cache_len ? (a.cache_len > 0 ? a.cache_len : 1) : a.chunk_len;
  p.chunk_len = (int32_t)L;
  p.window = (int32_t)(a.window_chunks > a.cache_len / L ? -1 : a.window_chunks);
  p.row_tiles = (int32_t)plan.row_tiles;
  p.runs = kv4_runs(p.row_tiles);
  p.whole = (int32_t)plan.whole;
  p.rest = (int32_t)(a.B * a.Hkv * plan.row_tiles - plan.whole);
  p.n_split = plan.n_split;
  p.tile_rows = plan.row_tiles > 1 ? 16 * plan.q_tiles : p.R;
  p.units = (int32_t)plan.units;
  p.rows = plan.rows;
  // (not 0: masked scores, -inf * c, stay -inf; 2^-126 leaves P at 1 for all others)
  p.c = __builtin_fmaxf(__builtin_fabsf(a.scale) * 1.44269504088896340736f, 0x1p-126f);
  p.sign = a.scale < 0.f ? 0x80008000u : 0u;
  return a.d == 128 ? launch_t<128>(p, plan, stream) : launch_t<64>(p, plan, stream);
}

}  // namespace fastvr
