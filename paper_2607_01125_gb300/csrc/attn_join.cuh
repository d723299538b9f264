// Joining the parts of a row of work that was cut along its long axis: every part leaves its sums in a slot, and the last of
// them to finish (a ticket) adds them up in the order of the parts, so that results do not depend on which one it is.
#pragma once
#include "attn.h"

namespace zoact {
namespace attn {

__device__ __forceinline__ float* slot_sums(const Slots& s, int slot) { return s.sums + (size_t)slot * (2 * TILE * TC_DIM); }
__device__ __forceinline__ float2* slot_stat(const Slots& s, int slot) { return s.stat + (size_t)slot * (2 * TILE); }

// Whether this group of threads (SYNC: its barrier) brings the last of n parts; its writes before come first.
template <class Sync>
__device__ __forceinline__ bool last_part(unsigned* ticket, int n, bool first_thread, int* shared_flag, Sync sync) {
  __threadfence();
  sync();
  if (first_thread) {
    const unsigned t = atomicAdd(ticket, 1u);
    *shared_flag = t == (unsigned)(n - 1);
    if (t == (unsigned)(n - 1)) *ticket = 0;
  }
  sync();
  const bool last = *shared_flag != 0;
  if (last) __threadfence();
  return last;
}

// Forward: rows [r0, r0 + n) of the parts in slots [slot, slot + nparts), each a row of D sums beside its statistics, are joined
// by threads tid of nt.  out(r, d, value) and stat(r, lse) take the results; r counts from r0.
template <class Out, class Stat>
__device__ __forceinline__ void join_rows(const Slots& s, int slot, int nparts, int r0, int n, int D, int tid, int nt, Out out,
                                          Stat stat) {
  const float* sums = slot_sums(s, slot) + (size_t)r0 * D;
  const float2* st = slot_stat(s, slot) + r0;
  for (int e = tid; e < n * D; e += nt) {
    const int r = e / D, d = e - r * D;
    float m = -INFINITY;
    for (int p = 0; p < nparts; ++p) m = fmaxf(m, __ldcg(&st[(size_t)p * 2 * TILE + r]).x);
    const float from = m == -INFINITY ? 0.f : m;
    float l = 0.f, o = 0.f;
    for (int p = 0; p < nparts; ++p) {
      const float2 x = __ldcg(&st[(size_t)p * 2 * TILE + r]);
      const float w = exp2f(x.x - from);
      l += w * x.y;
      o += w * __ldcg(&sums[(size_t)p * (2 * TILE * TC_DIM) + e]);
    }
    out(r, d, l > 0.f ? o / l : l == 0.f ? 0.f : l);
    if (d == 0) stat(r, m, l);
  }
}

}  // namespace attn
}  // namespace zoact
