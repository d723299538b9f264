// Attention over packed sequences and its gradient on the CUDA cores, in fp32: for fp32 operands, and for the shapes and strides
// that the tensor-core kernels do not take (heads wider than 128 or of a width that is no multiple of 8, rows that do not start
// on 16 bytes).
//
// One pass over the keys with a running maximum and sum for each row: S = Q K^T, P = exp(S - max), O = O exp(old max - max) + P V.
// A block of 256 threads has a tile of M rows of (position, head of the group) pairs against M keys; a thread has M / 16 rows
// and columns, spread 16 apart, so that its 16-byte reads of shared memory fall on different banks.  The gradient recomputes
// P = exp(S - lse) in two passes, one over the keys for dq and one over the rows for dk and dv, so that no sum needs atomics.
// Bound by latencies: tiles of 128 columns leave room for one block of 8 warps on an SM, which issues in 45% of the cycles (37% of
// the FMA rate) and reads shared memory in 45%.  8192 tokens of 32 heads on 8 of 128 22 ms (25 TFLOP/s), twice 2048 tokens 2.9 ms
// (23.5), two sequences of 64 in 4 heads of 64 13 us.
#include <type_traits>

#include "attn.h"
#include "attn_join.cuh"

namespace zoact {
namespace attn {

namespace {

constexpr int THREADS = 256;

template <int DP> struct Cfg {
  static constexpr int M = DP > 128 ? 32 : 64;       // rows and keys of a tile
  static constexpr int R = M / 16;                   // of a thread
  static constexpr int LD = DP + 4, LP = M + 4;      // row strides in shared memory
  static constexpr int C = DP / 64;                  // groups of 4 columns of a thread
};

struct Dev {
  Work work;
  Slots slots;
  int* status;
  Divisor by_rep;
  int rep, kv_heads, heads, head_dim, causal;
  int vec;                              // rows of q, k, v (and dO) lie on four elements, and so do heads
  float scale, scale_log2;
  const void *q, *k, *v, *O, *dO;
  int64_t ld_q, ld_k, ld_v, ld_o, ld_do, ld_dq, ld_dk, ld_dv;
  void *out, *dq, *dk, *dv;
  float* lse;
  const float* lse_in;
  const float* delta;
};

// Four elements of a row from column d on, zero behind the head (vec: they lie together).
template <typename T>
__device__ __forceinline__ float4 load4(const T* row, int d, int head_dim, bool vec) {
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  if (vec) {
    struct alignas(4 * sizeof(T)) Four { T v[4]; };
    if (d < head_dim) {
      const Four f = *reinterpret_cast<const Four*>(row + d);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = to_f32<T>(f.v[k]);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (d + k < head_dim) v[k] = to_f32<T>(row[d + k]);
  }
  return make_float4(v[0], v[1], v[2], v[3]);
}

// Rows [r0, r0 + M) of (position, head) pairs, n of them in all, of a tensor; zero behind them and behind the head.
template <typename T, int DP>
__device__ __forceinline__ void load_rows(float* s, const void* base, int64_t ld, const Item& w, int kvh, const Divisor& rep,
                                          int head_dim, bool vec, int r0, int n) {
  constexpr int M = Cfg<DP>::M;
#pragma unroll 4
  for (int e = threadIdx.x; e < M * DP / 4; e += THREADS) {
    const int r = e / (DP / 4), d = e % (DP / 4) * 4;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (r0 + r < n) {
      int j;
      const int pos = rep.div(r0 + r, j);
      x = load4<T>(static_cast<const T*>(base) + (int64_t)(w.q0 + pos) * ld + (int64_t)(kvh * rep.d + j) * head_dim, d, head_dim, vec);
    }
    *reinterpret_cast<float4*>(s + r * Cfg<DP>::LD + d) = x;
  }
}
template <typename T, int DP>
__device__ __forceinline__ void load_keys(float* s, const void* base, int64_t ld, int k0, int kvh, int head_dim, bool vec, int n) {
  constexpr int M = Cfg<DP>::M;
#pragma unroll 4
  for (int e = threadIdx.x; e < M * DP / 4; e += THREADS) {
    const int r = e / (DP / 4), d = e % (DP / 4) * 4;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (r < n) x = load4<T>(static_cast<const T*>(base) + (int64_t)(k0 + r) * ld + (int64_t)kvh * head_dim, d, head_dim, vec);
    *reinterpret_cast<float4*>(s + r * Cfg<DP>::LD + d) = x;
  }
}

// a[i][j] = row (ty + 16 i) of A times row (tx + 16 j) of B.
template <int DP>
__device__ __forceinline__ void product(const float* A, const float* B, int ty, int tx, float (&a)[Cfg<DP>::R][Cfg<DP>::R]) {
  constexpr int R = Cfg<DP>::R, LD = Cfg<DP>::LD;
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int j = 0; j < R; ++j) a[i][j] = 0.f;
#pragma unroll 4
  for (int d = 0; d < DP; d += 4) {
    float4 x[R], y[R];
#pragma unroll
    for (int i = 0; i < R; ++i) x[i] = *reinterpret_cast<const float4*>(A + (ty + 16 * i) * LD + d);
#pragma unroll
    for (int j = 0; j < R; ++j) y[j] = *reinterpret_cast<const float4*>(B + (tx + 16 * j) * LD + d);
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int j = 0; j < R; ++j) a[i][j] += x[i].x * y[j].x + x[i].y * y[j].y + x[i].z * y[j].z + x[i].w * y[j].w;
  }
}

// o[i][c] += sum over m of P[ty + 16 i][m] times columns 4 tx + 64 c .. + 3 of row m of B.
template <int DP>
__device__ __forceinline__ void add_product(const float* P, const float* B, int ty, int tx, float4 (&o)[Cfg<DP>::R][Cfg<DP>::C]) {
  constexpr int R = Cfg<DP>::R, C = Cfg<DP>::C, M = Cfg<DP>::M, LD = Cfg<DP>::LD, LP = Cfg<DP>::LP;
#pragma unroll 2
  for (int m = 0; m < M; m += 4) {
    float4 p[R];
#pragma unroll
    for (int i = 0; i < R; ++i) p[i] = *reinterpret_cast<const float4*>(P + (ty + 16 * i) * LP + m);
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int c = 0; c < C; ++c) {
        const float4 b = *reinterpret_cast<const float4*>(B + (m + u) * LD + 4 * tx + 64 * c);
#pragma unroll
        for (int i = 0; i < R; ++i) {
          const float f = u == 0 ? p[i].x : u == 1 ? p[i].y : u == 2 ? p[i].z : p[i].w;
          o[i][c].x += f * b.x; o[i][c].y += f * b.y; o[i][c].z += f * b.z; o[i][c].w += f * b.w;
        }
      }
  }
}

__device__ __forceinline__ float half_warp_max(float x) {
  for (int o = 8; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}
__device__ __forceinline__ float half_warp_sum(float x) {
  for (int o = 8; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}
__device__ __forceinline__ float at(const float4& v, int u) { return u == 0 ? v.x : u == 1 ? v.y : u == 2 ? v.z : v.w; }

// Tiles of M rows that an item has room for: its rows are at most 2 TILE (forward) or TILE.
template <int DP> constexpr int tiles_of(int rows) { return rows / Cfg<DP>::M; }

template <typename T, int DP>
__global__ void __launch_bounds__(THREADS) fwd_kernel(const Dev p) {
  constexpr int R = Cfg<DP>::R, C = Cfg<DP>::C, M = Cfg<DP>::M, LD = Cfg<DP>::LD, LP = Cfg<DP>::LP, SUB = tiles_of<DP>(2 * TILE);
  extern __shared__ float sm[];
  float *sq = sm, *sk = sq + M * LD, *sv = sk + M * LD, *sp = sv + M * LD;
  __shared__ int flag;
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  const int64_t total = (int64_t)work_count(p.work, p.kv_heads, tid == 0 && blockIdx.x == 0 ? p.status : nullptr) * SUB;
  for (int64_t u = blockIdx.x; u < total; u += gridDim.x) {
    const int sub = (int)(u % SUB), h = (int)(u / SUB % p.kv_heads);
    const Item w = p.work.items[u / SUB / p.kv_heads];
    const int n = w.npos * p.rep, r0 = sub * M;
    if (r0 >= n) continue;
    __syncthreads();
    load_rows<T, DP>(sq, p.q, p.ld_q, w, h, p.by_rep, p.head_dim, p.vec, r0, n);
    float m[R], l[R];
    float4 o[R][C];
    int see[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      m[i] = -INFINITY; l[i] = 0.f;
      const int r = r0 + ty + 16 * i;
      see[i] = r < n ? visible(w, p.causal, r / p.rep) : 0;
#pragma unroll
      for (int c = 0; c < C; ++c) o[i][c] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    const int last = min(r0 + M, n) - 1, keys = visible(w, p.causal, last / p.rep);
    for (int j0 = 0; j0 < keys; j0 += M) {
      __syncthreads();
      load_keys<T, DP>(sk, p.k, p.ld_k, w.k0 + j0, h, p.head_dim, p.vec, keys - j0);
      load_keys<T, DP>(sv, p.v, p.ld_v, w.k0 + j0, h, p.head_dim, p.vec, keys - j0);
      __syncthreads();
      float s[R][R];
      product<DP>(sq, sk, ty, tx, s);
#pragma unroll
      for (int i = 0; i < R; ++i) {
        float top = -INFINITY;
#pragma unroll
        for (int j = 0; j < R; ++j) {
          s[i][j] = j0 + tx + 16 * j < see[i] ? s[i][j] * p.scale_log2 : -INFINITY;
          top = fmaxf(top, s[i][j]);
        }
        const float now = fmaxf(m[i], half_warp_max(top)), from = now == -INFINITY ? 0.f : now;
        const float old = exp2f(m[i] - from);
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < R; ++j) {
          s[i][j] = exp2f(s[i][j] - from);
          sum += s[i][j];
          sp[(ty + 16 * i) * LP + tx + 16 * j] = s[i][j];
        }
        l[i] = l[i] * old + sum;
        m[i] = now;
#pragma unroll
        for (int c = 0; c < C; ++c) { o[i][c].x *= old; o[i][c].y *= old; o[i][c].z *= old; o[i][c].w *= old; }
      }
      __syncthreads();
      add_product<DP>(sp, sv, ty, tx, o);
    }
    const auto put = [&](int r, int d, float x) {       // r: row of the item
      const int pos = r / p.rep;
      static_cast<T*>(p.out)[(int64_t)(w.q0 + pos) * p.ld_o + (int64_t)(h * p.rep + r - pos * p.rep) * p.head_dim + d] = from_f32<T>(x);
    };
    const auto put_stat = [&](int r, float top, float sum) {
      const int pos = r / p.rep;
      if (p.lse) p.lse[(int64_t)(w.q0 + pos) * p.heads + h * p.rep + r - pos * p.rep] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.69314718f;
    };
    const int slot = w.slot + h * w.nparts + w.part;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int r = r0 + ty + 16 * i;
      const float sum = half_warp_sum(l[i]);
      if (r >= n) continue;
      if (w.nparts > 1) {
        if (tx == 0) slot_stat(p.slots, slot)[r] = make_float2(m[i], sum);
      } else if (tx == 0) {
        put_stat(r, m[i], sum);
      }
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int d = 4 * tx + 64 * c + e;
          if (d >= p.head_dim) continue;
          if (w.nparts > 1) slot_sums(p.slots, slot)[(size_t)r * p.head_dim + d] = at(o[i][c], e);
          else put(r, d, at(o[i][c], e) * inv);
        }
    }
    if (w.nparts > 1) {
      const int first = w.slot + h * w.nparts;
      if (last_part(p.slots.tickets + 4 * first + sub, w.nparts, tid == 0, &flag, [] { __syncthreads(); }))
        join_rows(p.slots, first, w.nparts, r0, min(M, n - r0), p.head_dim, tid, THREADS,
                  [&](int r, int d, float x) { put(r0 + r, d, x); }, [&](int r, float top, float sum) { put_stat(r0 + r, top, sum); });
    }
  }
}

// delta = the row sum of dO O for each (row, head) of the sequences, by a group of lanes that has V elements each of a pass over the
// head; in fp16 also the largest finite |dO| and |v| of each sequence's group of heads (0 before).  It runs through the items of dq,
// whose rows are those of the sequences, and for v through those of dk and dv.  EACH pairs of a group at a time; 4096 rows of 32
// heads of 128 in bf16 20 to 22 us (3.4 TB/s).
constexpr int EACH = 4;

// The largest of a warp's values goes to *to (above 0: ordered as integers).
__device__ __forceinline__ void keep_largest(float x, float* to) {
  for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  if ((threadIdx.x & 31) == 0 && x > __ldcg(to)) atomicMax(reinterpret_cast<int*>(to), __float_as_int(x));
}

template <typename T, int V>
__global__ void __launch_bounds__(THREADS) delta_kernel(const Work work, int* status, const T* dO, int64_t ld_do, const T* O,
                                                        int64_t ld_o, int kv_heads, Divisor rep, int head_dim, int group,
                                                        float* delta, float2* largest, const Work keys, const T* v, int64_t ld_v) {
  pdl_wait();
  pdl_trigger();
  // (the sums lie in the plan, where it has room for them)
  const int total = work_count(work, kv_heads, threadIdx.x == 0 && blockIdx.x == 0 ? status : nullptr);
  struct alignas(sizeof(T) * V) Vec { T v[V]; };
  const int lane = threadIdx.x & 31, in_group = lane & (group - 1), groups = THREADS / group;
  const int heads = kv_heads * rep.d;
  for (int u = blockIdx.x; u < total; u += gridDim.x) {
    const Item w = work.items[u / kv_heads];
    if (w.part != 0) continue;
    const int h0 = u % kv_heads * rep.d, n = w.npos * rep.d;
    float top = 0.f;
    for (int e0 = threadIdx.x / group; __any_sync(0xffffffffu, e0 < n); e0 += groups * EACH) {
      float s[EACH];
      int64_t at[EACH];
#pragma unroll
      for (int e = 0; e < EACH; ++e) {
        int g;
        const int64_t r = w.q0 + rep.div(min(e0 + e * groups, n - 1), g);
        const T *a = dO + r * ld_do + (int64_t)(h0 + g) * head_dim, *b = O + r * ld_o + (int64_t)(h0 + g) * head_dim;
        at[e] = r * heads + h0 + g;
        s[e] = 0.f;
        for (int d = in_group * V; d < head_dim; d += group * V) {
          const Vec x = *reinterpret_cast<const Vec*>(a + d), y = *reinterpret_cast<const Vec*>(b + d);
#pragma unroll
          for (int k = 0; k < V; ++k) {
            const float f = to_f32<T>(x.v[k]);
            s[e] += f * to_f32<T>(y.v[k]);
            if (std::is_same<T, __half>::value && fabsf(f) < INFINITY) top = fmaxf(top, fabsf(f));
          }
        }
      }
#pragma unroll
      for (int e = 0; e < EACH; ++e) {
        for (int o = group / 2; o > 0; o >>= 1) s[e] += __shfl_xor_sync(0xffffffffu, s[e], o);
        if (in_group == 0 && e0 + e * groups < n) delta[at[e]] = s[e];
      }
    }
    if constexpr (std::is_same<T, __half>::value) keep_largest(top, &largest[(int64_t)w.seq * kv_heads + u % kv_heads].x);
  }
  if constexpr (std::is_same<T, __half>::value) {
    const int total_v = work_count(keys, kv_heads, nullptr);
    for (int u = gridDim.x - 1 - blockIdx.x; u < total_v; u += gridDim.x) {      // from the blocks that have least to do
      const Item w = keys.items[u / kv_heads];
      if (w.part != 0) continue;
      const T* const a = v + (int64_t)w.k0 * ld_v + (int64_t)(u % kv_heads) * head_dim;
      float top = 0.f;
#pragma unroll 4
      for (int e = threadIdx.x / group; e < w.nk; e += groups)
        for (int d = in_group * V; d < head_dim; d += group * V) {
          const Vec x = *reinterpret_cast<const Vec*>(a + e * ld_v + d);
#pragma unroll
          for (int k = 0; k < V; ++k) {
            const float f = fabsf(to_f32<T>(x.v[k]));
            if (f < INFINITY) top = fmaxf(top, f);
          }
        }
      keep_largest(top, &largest[(int64_t)w.seq * kv_heads + u % kv_heads].y);
    }
  }
}

// In fp16, the largest values of the call before give way.  (The last block of dk and dv could do this, without a launch: the ragged
// fp16 gradient 71.8 us for 69.9.)
__global__ void __launch_bounds__(THREADS) reset_kernel(const Work work, float2* largest, int64_t n) {
  pdl_wait();
  pdl_trigger();
  if (work_count(work, 1, nullptr) == 0) return;
  for (int64_t i = (int64_t)blockIdx.x * THREADS + threadIdx.x; i < n; i += (int64_t)gridDim.x * THREADS) largest[i] = make_float2(0.f, 0.f);
}

// P and dS = P (dP - delta) of a tile, from its scaled products z (times log2 e) and dP; 0 where a key is not seen.
__device__ __forceinline__ void share_of(float z, float dp, float base, float delta, bool seen, float& pr, float& ds) {
  pr = seen ? exp2f(z + base) : 0.f;
  ds = seen ? pr * (dp - delta) : 0.f;
}

template <typename T, int DP>
__global__ void __launch_bounds__(THREADS) dq_kernel(const Dev p) {
  constexpr int R = Cfg<DP>::R, C = Cfg<DP>::C, M = Cfg<DP>::M, LD = Cfg<DP>::LD, LP = Cfg<DP>::LP, SUB = tiles_of<DP>(TILE);
  extern __shared__ float sm[];
  float *sq = sm, *sg = sq + M * LD, *sk = sg + M * LD, *sv = sk + M * LD, *sp = sv + M * LD;
  __shared__ int flag;
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  const int64_t total = (int64_t)work_count(p.work, p.kv_heads, tid == 0 && blockIdx.x == 0 ? p.status : nullptr) * SUB;
  for (int64_t u = blockIdx.x; u < total; u += gridDim.x) {
    const int sub = (int)(u % SUB), h = (int)(u / SUB % p.kv_heads);
    const Item w = p.work.items[u / SUB / p.kv_heads];
    const int n = w.npos * p.rep, r0 = sub * M;
    if (r0 >= n) continue;
    __syncthreads();
    load_rows<T, DP>(sq, p.q, p.ld_q, w, h, p.by_rep, p.head_dim, p.vec, r0, n);
    load_rows<T, DP>(sg, p.dO, p.ld_do, w, h, p.by_rep, p.head_dim, p.vec, r0, n);
    float base[R], delta[R];
    float4 o[R][C];
    int see[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int r = r0 + ty + 16 * i, pos = r / p.rep;
      const int64_t e = (int64_t)(w.q0 + pos) * p.heads + h * p.rep + r - pos * p.rep;
      see[i] = r < n ? visible(w, p.causal, pos) : 0;
      base[i] = r < n ? share_base(p.lse_in[e]) : 0.f;
      delta[i] = r < n ? p.delta[e] : 0.f;
#pragma unroll
      for (int c = 0; c < C; ++c) o[i][c] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    const int last = min(r0 + M, n) - 1, keys = visible(w, p.causal, last / p.rep);
    for (int j0 = 0; j0 < keys; j0 += M) {
      __syncthreads();
      load_keys<T, DP>(sk, p.k, p.ld_k, w.k0 + j0, h, p.head_dim, p.vec, keys - j0);
      load_keys<T, DP>(sv, p.v, p.ld_v, w.k0 + j0, h, p.head_dim, p.vec, keys - j0);
      __syncthreads();
      float s[R][R], dp[R][R];
      product<DP>(sq, sk, ty, tx, s);
      product<DP>(sg, sv, ty, tx, dp);
#pragma unroll
      for (int i = 0; i < R; ++i)
#pragma unroll
        for (int j = 0; j < R; ++j) {
          float pr, ds;
          share_of(s[i][j] * p.scale_log2, dp[i][j], base[i], delta[i], j0 + tx + 16 * j < see[i], pr, ds);
          sp[(ty + 16 * i) * LP + tx + 16 * j] = ds;
        }
      __syncthreads();
      add_product<DP>(sp, sk, ty, tx, o);
    }
    const auto put = [&](int r, int d, float x) {
      const int pos = r / p.rep;
      static_cast<T*>(p.dq)[(int64_t)(w.q0 + pos) * p.ld_dq + (int64_t)(h * p.rep + r - pos * p.rep) * p.head_dim + d] = from_f32<T>(x * p.scale);
    };
    const int slot = w.slot + h * w.nparts;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int r = r0 + ty + 16 * i;
      if (r >= n) continue;
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int d = 4 * tx + 64 * c + e;
          if (d >= p.head_dim) continue;
          if (w.nparts > 1) slot_sums(p.slots, slot + w.part)[(size_t)r * p.head_dim + d] = at(o[i][c], e);
          else put(r, d, at(o[i][c], e));
        }
    }
    if (w.nparts > 1 && last_part(p.slots.tickets + 4 * slot + sub, w.nparts, tid == 0, &flag, [] { __syncthreads(); })) {
      for (int e = tid; e < min(M, n - r0) * p.head_dim; e += THREADS) {
        const int r = r0 + e / p.head_dim, d = e % p.head_dim;
        float x = 0.f;
        for (int k = 0; k < w.nparts; ++k) x += __ldcg(slot_sums(p.slots, slot + k) + (size_t)r * p.head_dim + d);
        put(r, d, x);
      }
    }
  }
}

// A row of work of dk and dv has up to 2^31 positions, with up to MAX_REP heads each: its rows are counted in 32 bits within runs of
// POSITIONS of them (whole tiles, so that the sums' order does not depend on it).
constexpr int POSITIONS = 4096;
static_assert((int64_t)POSITIONS * MAX_REP + TILE <= 0x7fffffff && POSITIONS % TILE == 0, "rows of a run");

template <typename T, int DP>
__global__ void __launch_bounds__(THREADS) dkv_kernel(const Dev p) {
  constexpr int R = Cfg<DP>::R, C = Cfg<DP>::C, M = Cfg<DP>::M, LD = Cfg<DP>::LD, LP = Cfg<DP>::LP, SUB = tiles_of<DP>(BK);
  extern __shared__ float sm[];
  float *sq = sm, *sg = sq + M * LD, *sk = sg + M * LD, *sv = sk + M * LD, *sp = sv + M * LD, *sd = sp + M * LP;
  __shared__ float base[M], delta[M];
  __shared__ int see[M], flag;
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  const int64_t total = (int64_t)work_count(p.work, p.kv_heads, tid == 0 && blockIdx.x == 0 ? p.status : nullptr) * SUB;
  for (int64_t u = blockIdx.x; u < total; u += gridDim.x) {
    const int sub = (int)(u % SUB), h = (int)(u / SUB % p.kv_heads);
    const Item w = p.work.items[u / SUB / p.kv_heads];
    const int key0 = sub * M;
    if (key0 >= w.nk) continue;
    const int nk = min(M, w.nk - key0);
    __syncthreads();
    load_keys<T, DP>(sk, p.k, p.ld_k, w.k0 + key0, h, p.head_dim, p.vec, nk);
    load_keys<T, DP>(sv, p.v, p.ld_v, w.k0 + key0, h, p.head_dim, p.vec, nk);
    float4 ok[R][C], ov[R][C];
#pragma unroll
    for (int i = 0; i < R; ++i)
#pragma unroll
      for (int c = 0; c < C; ++c) ok[i][c] = ov[i][c] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int first = 0; first < w.npos; first += POSITIONS) {
      Item run = w;
      run.q0 += first;
      run.npos = min(POSITIONS, w.npos - first);
      run.diag += p.causal ? first : 0;
      const int n = run.npos * p.rep;
      for (int r0 = 0; r0 < n; r0 += M) {
        __syncthreads();
        if (visible(run, p.causal, min(r0 + M, n) / p.rep) <= key0) continue;      // none of these rows sees the keys
        load_rows<T, DP>(sq, p.q, p.ld_q, run, h, p.by_rep, p.head_dim, p.vec, r0, n);
        load_rows<T, DP>(sg, p.dO, p.ld_do, run, h, p.by_rep, p.head_dim, p.vec, r0, n);
        if (tid < M) {
          const int r = r0 + tid, pos = r / p.rep;
          const int64_t e = (int64_t)(run.q0 + pos) * p.heads + h * p.rep + r - pos * p.rep;
          see[tid] = r < n ? visible(run, p.causal, pos) - key0 : 0;
          base[tid] = r < n ? share_base(p.lse_in[e]) : 0.f;
          delta[tid] = r < n ? p.delta[e] : 0.f;
        }
        __syncthreads();
        float s[R][R], dp[R][R];
        product<DP>(sk, sq, ty, tx, s);
        product<DP>(sv, sg, ty, tx, dp);
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
          for (int j = 0; j < R; ++j) {
            const int key = ty + 16 * i, r = tx + 16 * j;
            float pr, ds;
            share_of(s[i][j] * p.scale_log2, dp[i][j], base[r], delta[r], key < see[r], pr, ds);
            sp[key * LP + r] = pr;
            sd[key * LP + r] = ds;
          }
        __syncthreads();
        add_product<DP>(sp, sg, ty, tx, ov);
        add_product<DP>(sd, sq, ty, tx, ok);
      }
    }
    const auto put = [&](int key, int d, float k, float v) {
      const int64_t row = w.k0 + key, col = (int64_t)h * p.head_dim + d;
      static_cast<T*>(p.dk)[row * p.ld_dk + col] = from_f32<T>(k * p.scale);
      static_cast<T*>(p.dv)[row * p.ld_dv + col] = from_f32<T>(v);
    };
    const int slot = w.slot + h * w.nparts;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int key = key0 + ty + 16 * i;
      if (key >= w.nk) continue;
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int d = 4 * tx + 64 * c + e;
          if (d >= p.head_dim) continue;
          if (w.nparts > 1) {
            float* s = slot_sums(p.slots, slot + w.part) + (size_t)key * p.head_dim + d;
            s[0] = at(ok[i][c], e);
            s[(size_t)BK * p.head_dim] = at(ov[i][c], e);
          } else {
            put(key, d, at(ok[i][c], e), at(ov[i][c], e));
          }
        }
    }
    if (w.nparts > 1 && last_part(p.slots.tickets + 4 * slot + sub, w.nparts, tid == 0, &flag, [] { __syncthreads(); })) {
      for (int e = tid; e < nk * p.head_dim; e += THREADS) {
        const int key = key0 + e / p.head_dim, d = e % p.head_dim;
        float k = 0.f, v = 0.f;
        for (int i = 0; i < w.nparts; ++i) {
          const float* s = slot_sums(p.slots, slot + i) + (size_t)key * p.head_dim + d;
          k += __ldcg(s);
          v += __ldcg(s + (size_t)BK * p.head_dim);
        }
        put(key, d, k, v);
      }
    }
  }
}

int dev_args(Ctx* ctx, const Args& a, int list, Dev* d) {
  Slots s = {};
  const int st = slots(ctx, &s);
  if (st) return st;
  const auto lies = [&](const void* q, int64_t ld) { return (uintptr_t)q % (4 * dtype_size(a.dtype)) == 0 && ld % 4 == 0; };
  const bool vec = a.s.head_dim % 4 == 0 && lies(a.q, a.ld_q) && lies(a.k, a.ld_k) && lies(a.v, a.ld_v) && lies(a.dO, a.ld_do);
  *d = {work_of(a, list), s, ctx->d_status, Divisor(a.s.rep()), a.s.rep(), a.s.kv_heads, a.s.heads, a.s.head_dim, a.s.causal, vec, a.scale,
        a.scale * 1.44269504f, a.q, a.k, a.v, a.O, a.dO, a.ld_q, a.ld_k, a.ld_v, a.ld_o, a.ld_do, a.ld_dq, a.ld_dk, a.ld_dv,
        a.O, a.dq, a.dk, a.dv, a.lse, a.lse, a.delta};
  return ZOACT_OK;
}

template <int DP> constexpr int smem_bytes(int list) {
  using G = Cfg<DP>;
  return 4 * (list == LIST_FWD ? 3 * G::M * G::LD + G::M * G::LP : 4 * G::M * G::LD + (list == LIST_DQ ? 1 : 2) * G::M * G::LP);
}

template <typename T, int DP>
int run(Ctx* ctx, const Args& a, int list) {
  Dev d;
  const int st = dev_args(ctx, a, list, &d);
  if (st) return st;
  auto kern = list == LIST_FWD ? fwd_kernel<T, DP> : list == LIST_DQ ? dq_kernel<T, DP> : dkv_kernel<T, DP>;
  const int smem = smem_bytes<DP>(list), per_sm = 2 * (smem + 1024) <= 232448 ? 2 : 1;
  ZOACT_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  const int64_t most = a.at.most[list] * a.s.kv_heads * (2 * TILE / Cfg<DP>::M), grid = (int64_t)per_sm * ctx->sm_count;
  ZOACT_CUDA_TRY(launch_pdl(ctx, kern, dim3((unsigned)(most < grid ? most : grid)), dim3(THREADS), (size_t)smem, d));
  ++ctx->n_launch;
  return ZOACT_OK;
}
template <typename T>
int run(Ctx* ctx, const Args& a, int list) {
  if (a.s.head_dim <= 64) return run<T, 64>(ctx, a, list);
  return a.s.head_dim <= 128 ? run<T, 128>(ctx, a, list) : run<T, 256>(ctx, a, list);
}
int run(Ctx* ctx, const Args& a, int list) {
  switch (a.dtype) {
    case ZOACT_DT_FP32: return run<float>(ctx, a, list);
    case ZOACT_DT_BF16: return run<__nv_bfloat16>(ctx, a, list);
    default: return run<__half>(ctx, a, list);
  }
}

template <typename T>
int delta(Ctx* ctx, const Args& a) {
  if (a.dtype == ZOACT_DT_FP16) {
    const int64_t n = (int64_t)a.s.n_seq * a.s.kv_heads, blocks = n == 0 ? 1 : (n + THREADS - 1) / THREADS;
    ZOACT_CUDA_TRY(launch_pdl(ctx, reset_kernel, dim3((unsigned)(blocks < ctx->sm_count ? blocks : ctx->sm_count)), dim3(THREADS), 0,
                              work_of(a, LIST_DQ), a.largest, n));
    ++ctx->n_launch;
  }
  constexpr int V = 16 / (int)sizeof(T);
  const auto lies = [](const void* p, int64_t ld) { return (uintptr_t)p % 16 == 0 && ld % V == 0; };
  const bool vec = a.s.head_dim % V == 0 && lies(a.O, a.ld_o) && lies(a.dO, a.ld_do) &&
                   (a.dtype != ZOACT_DT_FP16 || lies(a.v, a.ld_v));
  int group = 1;                        // lanes of a head: a power of two
  while (group < 32 && group * (vec ? V : 1) < a.s.head_dim) group *= 2;
  const int64_t blocks = a.at.most[LIST_DQ] * a.s.kv_heads, most = (int64_t)ctx->sm_count * 8;
  auto kern = vec ? delta_kernel<T, V> : delta_kernel<T, 1>;
  ZOACT_CUDA_TRY(launch_pdl(ctx, kern, dim3((unsigned)(blocks < most ? blocks : most)), dim3(THREADS), 0, work_of(a, LIST_DQ),
                            ctx->d_status, (const T*)a.dO, a.ld_do, (const T*)a.O, a.ld_o, a.s.kv_heads, Divisor(a.s.rep()),
                            a.s.head_dim, group, a.delta, a.largest, work_of(a, LIST_DKV), (const T*)a.v, a.ld_v));
  ++ctx->n_launch;
  return ZOACT_OK;
}

}  // namespace

int launch_delta(Ctx* ctx, const Args& a) {
  if (a.s.rows_q == 0) return ZOACT_OK;
  switch (a.dtype) {
    case ZOACT_DT_FP32: return delta<float>(ctx, a);
    case ZOACT_DT_BF16: return delta<__nv_bfloat16>(ctx, a);
    default: return delta<__half>(ctx, a);
  }
}

int launch_fwd_simt(Ctx* ctx, const Args& a) { return run(ctx, a, LIST_FWD); }

int launch_grad_simt(Ctx* ctx, const Args& a) {
  int st = run(ctx, a, LIST_DQ);
  return st ? st : run(ctx, a, LIST_DKV);
}

}  // namespace attn
}  // namespace zoact
