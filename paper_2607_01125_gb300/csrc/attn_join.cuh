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

// The same for 16-bit outputs of heads of a multiple of 8 columns, four columns and JOIN rows' loads at a time: one by one, each
// waiting for the last, 128 rows of 128 took 60 us.  out(r, d, values) takes four columns.
constexpr int JOIN = 4;
template <class Out, class Stat>
__device__ __forceinline__ void join_rows4(const Slots& s, int slot, int nparts, int r0, int n, int D, int tid, int nt, Out out,
                                           Stat stat) {
  const float* sums = slot_sums(s, slot) + (size_t)r0 * D;
  const float2* st = slot_stat(s, slot) + r0;
  const int per = D / 4, total = n * per;
  for (int e0 = tid; e0 < total; e0 += JOIN * nt) {
    int r[JOIN];
    float m[JOIN], l[JOIN];
    float4 o[JOIN];
#pragma unroll
    for (int b = 0; b < JOIN; ++b) {
      r[b] = min(e0 + b * nt, total - 1) / per;
      m[b] = -INFINITY;
      l[b] = 0.f;
      o[b] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
#pragma unroll 2
    for (int p = 0; p < nparts; ++p)
#pragma unroll
      for (int b = 0; b < JOIN; ++b) m[b] = fmaxf(m[b], __ldcg(&st[(size_t)p * 2 * TILE + r[b]]).x);
#pragma unroll
    for (int b = 0; b < JOIN; ++b) m[b] = m[b] == -INFINITY ? 0.f : m[b];
#pragma unroll 2
    for (int p = 0; p < nparts; ++p)
#pragma unroll
      for (int b = 0; b < JOIN; ++b) {
        const int e = min(e0 + b * nt, total - 1);
        const float2 x = __ldcg(&st[(size_t)p * 2 * TILE + r[b]]);
        const float4 v = __ldcg(reinterpret_cast<const float4*>(sums + (size_t)p * (2 * TILE * TC_DIM)) + e);
        const float w = exp2f(x.x - m[b]);
        l[b] += w * x.y;
        o[b].x += w * v.x; o[b].y += w * v.y; o[b].z += w * v.z; o[b].w += w * v.w;
      }
#pragma unroll
    for (int b = 0; b < JOIN; ++b) {
      const int e = e0 + b * nt;
      if (e >= total) break;
      const float f = l[b] > 0.f ? 1.f / l[b] : l[b];             // (0: a row that saw nothing; NaN stays)
      o[b].x *= f; o[b].y *= f; o[b].z *= f; o[b].w *= f;
      const int d = (e - r[b] * per) * 4;
      out(r[b], d, o[b]);
      if (d == 0) stat(r[b], m[b], l[b]);
    }
  }
}

// Sums of parts alone: rows of D / 4 vectors from `first` floats into the slots.
template <class Out>
__device__ __forceinline__ void join_sums4(const Slots& s, int slot, int nparts, size_t first, int total, int tid, int nt, Out out) {
  const float* sums = slot_sums(s, slot) + first;
  for (int e0 = tid; e0 < total; e0 += JOIN * nt) {
    float4 o[JOIN];
#pragma unroll
    for (int b = 0; b < JOIN; ++b) o[b] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
    for (int p = 0; p < nparts; ++p)
#pragma unroll
      for (int b = 0; b < JOIN; ++b) {
        const float4 v = __ldcg(reinterpret_cast<const float4*>(sums + (size_t)p * (2 * TILE * TC_DIM)) + min(e0 + b * nt, total - 1));
        o[b].x += v.x; o[b].y += v.y; o[b].z += v.z; o[b].w += v.w;
      }
#pragma unroll
    for (int b = 0; b < JOIN; ++b)
      if (e0 + b * nt < total) out(e0 + b * nt, o[b]);
  }
}

}  // namespace attn
}  // namespace zoact
