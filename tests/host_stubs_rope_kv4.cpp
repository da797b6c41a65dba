// Stand-ins for the launchers of the rotary and 4-bit cache kernels, linked with
// tests/host_stubs.cpp: they launch nothing and check what the kernels rely on.
#include <hip/hip_runtime_api.h>

#include <cstdlib>

#include "launch.h"

namespace fastvr {

static hipError_t holds(bool x) {
  if (!x) std::abort();
  return hipSuccess;
}

hipError_t launch_rope(const RopeArgs& a, hipStream_t) {
  return holds(a.x && a.y && a.positions && (a.n_pairs == 0 || a.inv_freq) && a.B > 0 && a.B <= 65535 && a.H > 0 &&
               a.H <= 65535 && a.N > 0 && a.N <= (1 << 24) && a.n_pairs <= a.d / 2 && 0 <= a.split1 && a.split1 <= a.split2 &&
               a.split2 <= a.n_pairs && a.n_axes >= 1 && a.n_axes <= 3 && a.x_st >= a.H * a.d && a.y_st >= a.H * a.d);
}

static bool copy_holds(const Kv4CopyArgs& a) {
  return a.cache.k_codes && a.cache.k_scales && a.cache.v_codes && a.cache.v_scales && a.k && a.v && a.B > 0 && a.B <= 32767 &&
         a.H > 0 && a.H <= 65535 && a.n > 0 && a.capacity <= FASTVR_KV4_MAX_CAPACITY && a.first >= 0 &&
         (a.starts || a.first + a.n <= a.capacity);
}
hipError_t launch_kv4_append(const Kv4CopyArgs& a, hipStream_t) { return holds(copy_holds(a)); }
hipError_t launch_kv4_read(const Kv4CopyArgs& a, hipStream_t) { return holds(copy_holds(a)); }

hipError_t launch_kv4_attn(const Kv4AttnArgs& a, hipStream_t) {
  const Kv4Plan p = kv4_plan(a.B, a.H, a.Hkv, a.nq, a.d, a.cache_len, a.chunk_len, a.window_chunks);
  return holds(a.q && a.o && a.B > 0 && a.nq > 0 && a.H % a.Hkv == 0 && a.cache_len <= a.capacity && a.chunk_len >= 1 &&
               p.units == a.plan.units && p.ws_bytes == a.plan.ws_bytes && p.units <= kMaxKv4Units &&
               (p.ws_bytes == 0 || a.workspace) && (a.capacity == 0 || a.cache.k_codes));
}

}  // namespace fastvr
