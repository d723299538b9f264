// Layer norm over the rows of X [rows, n] (row stride ld):
//     y = (x - m) s g + b,  m = mean(x),  s = 1 / sqrt(mean((x - m)^2) + eps)
// and its gradient, with u = dy g and xh = (x - m) s:
//     dx = s (u - mean(u) - xh mean(u xh)),  dg = sum_rows dy xh,  db = sum_rows dy.
//
// Both are bound by memory: forward reads and writes a row once, the gradient reads two and writes one.  A row is held in
// registers between its statistics (mean first, then the centred squares: no cancellation) and its output.  The gradient
// by the parameters needs every row of a column: persistent blocks keep their columns' sums in registers over all their
// rows, which bulk copies bring into a ring of shared memory ahead of them, and one small kernel adds the blocks' sums in
// block order.  Rows that no 16-byte copy can start at, and rows too long for a block's registers, take a row kernel and
// a column kernel instead, which read X and dY once each.
#include "internal.h"
#include "tc_common.cuh"

namespace zoact {
namespace {

constexpr int LN_THREADS = 256;

// Pairs of fp32 in one instruction, each half rounded as by itself.
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(*reinterpret_cast<uint64_t*>(&a)), "l"(*reinterpret_cast<uint64_t*>(&b)));
  return *reinterpret_cast<float2*>(&r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(*reinterpret_cast<uint64_t*>(&a)), "l"(*reinterpret_cast<uint64_t*>(&b)));
  return *reinterpret_cast<float2*>(&r);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(r)
      : "l"(*reinterpret_cast<uint64_t*>(&a)), "l"(*reinterpret_cast<uint64_t*>(&b)), "l"(*reinterpret_cast<uint64_t*>(&c)));
  return *reinterpret_cast<float2*>(&r);
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// A 16-byte vector's elements in pairs, and back.
template <typename T>
__device__ __forceinline__ void unpack(const uint4& u, float2* f) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
  if constexpr (sizeof(T) == 4) {
    f[0] = make_float2(__uint_as_float(w[0]), __uint_as_float(w[1]));
    f[1] = make_float2(__uint_as_float(w[2]), __uint_as_float(w[3]));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const T* e = reinterpret_cast<const T*>(&w[i]);
      f[i] = make_float2(to_f32<T>(e[0]), to_f32<T>(e[1]));
    }
  }
}
template <typename T>
__device__ __forceinline__ uint4 pack(const float2* f) {
  if constexpr (sizeof(T) == 4) {
    return make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[1].x), __float_as_uint(f[1].y));
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      T o[2] = {from_f32<T>(f[i].x), from_f32<T>(f[i].y)};
      w[i] = *reinterpret_cast<const uint32_t*>(o);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
}

template <typename TP>
__device__ __forceinline__ float param_at(const TP* p, int64_t i, float none) { return p ? to_f32<TP>(p[i]) : none; }

// E consecutive elements as fp32: one 16-byte (or two, for fp32 parameters of 16-bit rows) load, or one element.
template <typename T, int E>
__device__ __forceinline__ void load_e(const T* p, float* v) {
  if constexpr (E == 1) {
    v[0] = to_f32<T>(*p);
  } else {
    constexpr int N = 16 / (int)sizeof(T);
#pragma unroll
    for (int q = 0; q < E / N; ++q) {
      const uint4 u = *reinterpret_cast<const uint4*>(p + q * N);
      const T* e = reinterpret_cast<const T*>(&u);
#pragma unroll
      for (int i = 0; i < N; ++i) v[q * N + i] = to_f32<T>(e[i]);
    }
  }
}
template <typename T, int E>
__device__ __forceinline__ void load_stream(const T* p, float* v) {     // read once: kept out of the parameters' way in L1
  if constexpr (E == 1) {
    v[0] = to_f32<T>(*p);
  } else {
    static_assert(E * sizeof(T) == 16, "one vector");
    const uint4 u = __ldcs(reinterpret_cast<const uint4*>(p));
    const T* e = reinterpret_cast<const T*>(&u);
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = to_f32<T>(e[i]);
  }
}
template <typename T, int E>
__device__ __forceinline__ void store_e(T* p, const float* v) {
  if constexpr (E == 1) {
    *p = from_f32<T>(v[0]);
  } else {
    static_assert(E * sizeof(T) == 16, "one vector");
    uint4 u;
    T* e = reinterpret_cast<T*>(&u);
#pragma unroll
    for (int i = 0; i < E; ++i) e[i] = from_f32<T>(v[i]);
    *reinterpret_cast<uint4*>(p) = u;
  }
}
template <typename TP, int E>
__device__ __forceinline__ void load_param(const TP* p, int64_t i, float none, float* v) {
  if (p) {
    load_e<TP, E>(p + i, v);
  } else {
#pragma unroll
    for (int k = 0; k < E; ++k) v[k] = none;
  }
}

// The sum over a row's threads: a warp (blockDim.x = 32), or the block.  `red` holds two values a warp; calls alternate
// between two of them.
__device__ __forceinline__ float2 row_sum(float2 v, float2* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
    v.y += __shfl_xor_sync(0xffffffffu, v.y, o);
  }
  const int warps = blockDim.x >> 5;
  if (warps == 1) return v;
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  v = make_float2(0.f, 0.f);
  for (int w = 0; w < warps; ++w) { v.x += red[w].x; v.y += red[w].y; }
  return v;
}

// A row by blockDim.x threads, VPT vectors of E elements each in registers; blockDim.y rows a block (of one warp each).
// Threads of a row at most: what its registers (VPT vectors, up to 64 of them a thread at 1024) leave room for.
constexpr int most_threads(int e, bool grad) { return e == 1 ? 512 : grad ? 640 : 1024; }

template <typename T, typename TP, int E, int VPT>
__global__ void __launch_bounds__(most_threads(E, false))
ln_rows_kernel(const T* __restrict__ X, int64_t ld, int64_t rows, int n, const TP* __restrict__ g,
                               const TP* __restrict__ b, float eps, T* __restrict__ Y, float* __restrict__ mean,
                               float* __restrict__ rstd) {
  pdl_wait();                              // the input rows written by the previous kernel
  pdl_trigger();
  __shared__ float2 red[2][32];
  const int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  if (row >= rows) return;                 // whole warps; rows of several warps have a block each
  const T* x = X + row * ld;
  const int nv = n / E;
  float v[VPT][E];
  float2 s = make_float2(0.f, 0.f);
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int i = threadIdx.x + j * blockDim.x;
    if (i < nv) {
      load_stream<T, E>(x + (int64_t)i * E, v[j]);
#pragma unroll
      for (int k = 0; k < E; ++k) s.x += v[j][k];
    }
  }
  const float m = row_sum(s, red[0]).x / (float)n;
  s.x = 0.f;
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    if (threadIdx.x + j * blockDim.x < nv) {
#pragma unroll
      for (int k = 0; k < E; ++k) {
        v[j][k] -= m;
        s.x = fmaf(v[j][k], v[j][k], s.x);
      }
    }
  }
  const float r = 1.f / sqrtf(row_sum(s, red[1]).x / (float)n + eps);
  T* y = Y + row * n;
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int i = threadIdx.x + j * blockDim.x;
    if (i < nv) {
      float gg[E], bb[E];
      load_param<TP, E>(g, (int64_t)i * E, 1.f, gg);
      load_param<TP, E>(b, (int64_t)i * E, 0.f, bb);
#pragma unroll
      for (int k = 0; k < E; ++k) v[j][k] = fmaf(v[j][k] * r, gg[k], bb[k]);
      store_e<T, E>(y + (int64_t)i * E, v[j]);
    }
  }
  if (threadIdx.x == 0) {
    if (mean) mean[row] = m;
    if (rstd) rstd[row] = r;
  }
}

// A warp a row, the row's vectors packed in registers: no barrier, and with four rows a block ten times the bytes in flight
// of a block a row (8192 x 5120 fp16: 49 us with ln_rows_kernel, 160 threads a row).  For many rows; few rows take
// ln_rows_kernel, whose threads share a row's work.
template <typename T, typename TP, int VPT>
__global__ void __launch_bounds__(128)
ln_warp_kernel(const T* __restrict__ X, int64_t ld, int64_t rows, int n, const TP* __restrict__ g, const TP* __restrict__ b,
               float eps, T* __restrict__ Y, float* __restrict__ mean, float* __restrict__ rstd) {
  constexpr int E = 16 / (int)sizeof(T), P = E / 2;
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (row >= rows) return;
  const uint4* x = reinterpret_cast<const uint4*>(X + row * ld);
  const int nv = n / E;
  uint4 q[VPT];
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    q[j] = make_uint4(0u, 0u, 0u, 0u);
    if (lane + 32 * j < nv) q[j] = __ldcs(x + lane + 32 * j);
  }
  float2 s = make_float2(0.f, 0.f);
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    float2 f[P];
    unpack<T>(q[j], f);
#pragma unroll
    for (int i = 0; i < P; ++i) s = add2(s, f[i]);
  }
  float t = s.x + s.y;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
  const float m = t / (float)n;
  s = make_float2(0.f, 0.f);
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    float2 f[P];
    unpack<T>(q[j], f);
    if (lane + 32 * j < nv) {
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const float2 c = add2(f[i], both(-m));
        s = fma2(c, c, s);
      }
    }
  }
  t = s.x + s.y;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
  const float r = 1.f / sqrtf(t / (float)n + eps);
  uint4* y = reinterpret_cast<uint4*>(Y + row * n);
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int v = lane + 32 * j;
    if (v < nv) {
      float2 f[P];
      float gg[E], bb[E];
      unpack<T>(q[j], f);
      load_param<TP, E>(g, (int64_t)v * E, 1.f, gg);
      load_param<TP, E>(b, (int64_t)v * E, 0.f, bb);
#pragma unroll
      for (int i = 0; i < P; ++i)
        f[i] = fma2(mul2(add2(f[i], both(-m)), both(r)), make_float2(gg[2 * i], gg[2 * i + 1]),
                    make_float2(bb[2 * i], bb[2 * i + 1]));
      y[v] = pack<T>(f);
    }
  }
  if (lane == 0) {
    if (mean) mean[row] = m;
    if (rstd) rstd[row] = r;
  }
}

// dX alone, as ln_rows_kernel.
template <typename T, typename TP, int E, int VPT>
__global__ void __launch_bounds__(most_threads(E, true))
ln_grad_rows_kernel(const T* __restrict__ dY, int64_t ld_dy, const T* __restrict__ X, int64_t ld,
                                    int64_t rows, int n, const TP* __restrict__ g, const float* __restrict__ mean,
                                    const float* __restrict__ rstd, T* __restrict__ dX) {
  pdl_wait();
  pdl_trigger();
  __shared__ float2 red[32];
  const int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  if (row >= rows) return;
  const T* x = X + row * ld;
  const T* dy = dY + row * ld_dy;
  const float m = mean[row], r = rstd[row];
  const int nv = n / E;
  float u[VPT][E], xh[VPT][E];
  float2 s = make_float2(0.f, 0.f);
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int i = threadIdx.x + j * blockDim.x;
    if (i < nv) {
      load_stream<T, E>(dy + (int64_t)i * E, u[j]);
      load_stream<T, E>(x + (int64_t)i * E, xh[j]);
      float gg[E];
      load_param<TP, E>(g, (int64_t)i * E, 1.f, gg);
#pragma unroll
      for (int k = 0; k < E; ++k) {
        u[j][k] *= gg[k];
        xh[j][k] = (xh[j][k] - m) * r;
        s.x += u[j][k];
        s.y = fmaf(u[j][k], xh[j][k], s.y);
      }
    }
  }
  s = row_sum(s, red);
  s.x /= (float)n;
  s.y /= (float)n;
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int i = threadIdx.x + j * blockDim.x;
    if (i < nv) {
#pragma unroll
      for (int k = 0; k < E; ++k) u[j][k] = (u[j][k] - s.x - xh[j][k] * s.y) * r;
      store_e<T, E>(dX + row * n + (int64_t)i * E, u[j]);
    }
  }
}

// Rows longer than a block's registers: as the two kernels above, the row read once per use.
template <typename T, typename TP>
__global__ void __launch_bounds__(LN_THREADS)
ln_long_kernel(const T* __restrict__ X, int64_t ld, int n, const TP* __restrict__ g, const TP* __restrict__ b, float eps,
               T* __restrict__ Y, float* __restrict__ mean, float* __restrict__ rstd) {
  pdl_wait();
  pdl_trigger();
  __shared__ float2 red[2][32];
  const int64_t row = blockIdx.x;
  const T* x = X + row * ld;
  float2 s = make_float2(0.f, 0.f);
  for (int i = threadIdx.x; i < n; i += LN_THREADS) s.x += to_f32<T>(x[i]);
  const float m = row_sum(s, red[0]).x / (float)n;
  s.x = 0.f;
  for (int i = threadIdx.x; i < n; i += LN_THREADS) {
    const float c = to_f32<T>(x[i]) - m;
    s.x = fmaf(c, c, s.x);
  }
  const float r = 1.f / sqrtf(row_sum(s, red[1]).x / (float)n + eps);
  for (int i = threadIdx.x; i < n; i += LN_THREADS)
    Y[row * n + i] = from_f32<T>(fmaf((to_f32<T>(x[i]) - m) * r, param_at(g, i, 1.f), param_at(b, i, 0.f)));
  if (threadIdx.x == 0) {
    if (mean) mean[row] = m;
    if (rstd) rstd[row] = r;
  }
}

template <typename T, typename TP>
__global__ void __launch_bounds__(LN_THREADS)
ln_grad_long_kernel(const T* __restrict__ dY, int64_t ld_dy, const T* __restrict__ X, int64_t ld, int n,
                    const TP* __restrict__ g, const float* __restrict__ mean, const float* __restrict__ rstd,
                    T* __restrict__ dX) {
  pdl_wait();
  pdl_trigger();
  __shared__ float2 red[32];
  const int64_t row = blockIdx.x;
  const T* x = X + row * ld;
  const T* dy = dY + row * ld_dy;
  const float m = mean[row], r = rstd[row];
  float2 s = make_float2(0.f, 0.f);
  for (int i = threadIdx.x; i < n; i += LN_THREADS) {
    const float u = to_f32<T>(dy[i]) * param_at(g, i, 1.f), xh = (to_f32<T>(x[i]) - m) * r;
    s.x += u;
    s.y = fmaf(u, xh, s.y);
  }
  s = row_sum(s, red);
  s.x /= (float)n;
  s.y /= (float)n;
  for (int i = threadIdx.x; i < n; i += LN_THREADS) {
    const float u = to_f32<T>(dy[i]) * param_at(g, i, 1.f), xh = (to_f32<T>(x[i]) - m) * r;
    dX[row * n + i] = from_f32<T>((u - s.x - xh * s.y) * r);
  }
}

// Column sums of rows [y per, (y + 1) per) into part [gridDim.y][2][n], one thread a column.
template <typename T>
__global__ void __launch_bounds__(LN_THREADS)
ln_grad_cols_kernel(const T* __restrict__ dY, int64_t ld_dy, const T* __restrict__ X, int64_t ld, int64_t rows, int n,
                    const float* __restrict__ mean, const float* __restrict__ rstd, int64_t per, float* __restrict__ part) {
  pdl_wait();
  pdl_trigger();
  const int i = blockIdx.x * LN_THREADS + threadIdx.x;
  if (i >= n) return;
  const int64_t r0 = blockIdx.y * per, r1 = r0 + per < rows ? r0 + per : rows;
  float sg = 0.f, sb = 0.f;
#pragma unroll 8
  for (int64_t row = r0; row < r1; ++row) {
    const float dy = to_f32<T>(dY[row * ld_dy + i]);
    sg = fmaf(dy, (to_f32<T>(X[row * ld + i]) - mean[row]) * rstd[row], sg);
    sb += dy;
  }
  part[((int64_t)blockIdx.y * 2) * n + i] = sg;
  part[((int64_t)blockIdx.y * 2 + 1) * n + i] = sb;
}

// dg and db from part [parts][2][n], in part order within each of 32 groups.
__global__ void __launch_bounds__(1024)
ln_join_kernel(const float* __restrict__ part, int parts, int n, float* __restrict__ dg, float* __restrict__ db) {
  pdl_wait();
  pdl_trigger();
  __shared__ float red[32][33];
  const int c = threadIdx.x & 31, group = threadIdx.x >> 5;
  const int64_t col = (int64_t)blockIdx.x * 32 + c;
  float s = 0.f;
  if (col < 2 * (int64_t)n) {
#pragma unroll 8
    for (int p = group; p < parts; p += 32) s += __ldcg(part + (int64_t)p * 2 * n + col);
  }
  red[group][c] = s;
  __syncthreads();
  // warp w adds the groups of column w, pairwise by its lanes
  s = red[c][group];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  const int64_t mine = (int64_t)blockIdx.x * 32 + group;
  if (c != 0 || mine >= 2 * (int64_t)n) return;
  float* out = mine < n ? dg : db;
  if (out) out[mine < n ? mine : mine - n] = s;
}

// The whole gradient in one pass: block b takes rows b, b + gridDim.x, ...; thread t columns of vectors t, t + blockDim.x, ...
// for all of them.  `stages` rows of X and dY are in flight by bulk copies.  A row costs one block reduction; the barrier in
// it also says that its stage has been read.
constexpr int LN_MAX_STAGES = 8;
// A thread's columns take five registers each (their sums, gain, and the row's two values), 16 columns at most: rows up to
// 8192.
constexpr int RING_THREADS = 512;
template <typename T> constexpr int RING_VPTS = sizeof(T) == 4 ? 3 : 2;

template <typename T, typename TP, int VPT>
__global__ void __launch_bounds__(RING_THREADS)
ln_grad_ring_kernel(const T* __restrict__ dY, int64_t ld_dy, const T* __restrict__ X, int64_t ld, int64_t rows, int n,
                    const TP* __restrict__ g, const float* __restrict__ mean, const float* __restrict__ rstd,
                    T* __restrict__ dX, float* __restrict__ part, int stages, int* status) {
  constexpr int E = 16 / (int)sizeof(T);
  extern __shared__ __align__(128) uint8_t ring[];
  __shared__ uint64_t bars[LN_MAX_STAGES];
  __shared__ float2 red[2][16];
  __shared__ int abort_flag;
  const uint32_t row_bytes = (uint32_t)n * (uint32_t)sizeof(T);
  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) tc::mbar_init(tc::smem_u32(&bars[s]), 1);
    abort_flag = 0;
    tc::fence_mbar_init();
  }
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  const int nv = n / E;
  const int64_t mine = (rows - blockIdx.x + gridDim.x - 1) / gridDim.x;
  auto fetch = [&](int64_t i) {            // row i of this block into its stage
    const int64_t row = blockIdx.x + i * gridDim.x;
    const int s = (int)(i % stages);
    const uint32_t bar = tc::smem_u32(&bars[s]), dst = tc::smem_u32(ring) + (uint32_t)s * 2u * row_bytes;
    tc::mbar_arrive_expect_tx(bar, 2u * row_bytes);
    tc::bulk_load(dst, X + row * ld, row_bytes, bar);
    tc::bulk_load(dst + row_bytes, dY + row * ld_dy, row_bytes, bar);
  };
  if (threadIdx.x == 0)
    for (int64_t i = 0; i < mine && i < stages; ++i) fetch(i);
  constexpr int P = E / 2;
  float2 gg[VPT][P], sg[VPT][P], sb[VPT][P];
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int v = threadIdx.x + j * blockDim.x;
    float one[E];
    if (v < nv) load_param<TP, E>(g, (int64_t)v * E, 1.f, one);
#pragma unroll
    for (int k = 0; k < P; ++k) {
      gg[j][k] = make_float2(one[2 * k], one[2 * k + 1]);
      sg[j][k] = sb[j][k] = make_float2(0.f, 0.f);
    }
  }
  float m = mean[blockIdx.x], r = rstd[blockIdx.x];
  bool failed = false;
  for (int64_t i = 0; i < mine; ++i) {
    const int64_t row = blockIdx.x + i * gridDim.x;
    float m1 = 0.f, r1 = 0.f;              // the next row's statistics, ahead of their use
    if (i + 1 < mine) { m1 = mean[row + gridDim.x]; r1 = rstd[row + gridDim.x]; }
    const int s = (int)(i % stages);
    const bool ok = tc::mbar_wait(tc::smem_u32(&bars[s]), (uint32_t)(i / stages) & 1u, &abort_flag, status);
    const uint4* xs = reinterpret_cast<const uint4*>(ring + (size_t)s * 2 * row_bytes);
    const uint4* ys = xs + nv;
    float2 u[VPT][P], xh[VPT][P];
    float2 ta = make_float2(0.f, 0.f), tb = make_float2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int v = threadIdx.x + j * blockDim.x;
      if (v < nv) {
        unpack<T>(xs[v], xh[j]);
        unpack<T>(ys[v], u[j]);
#pragma unroll
        for (int k = 0; k < P; ++k) {
          xh[j][k] = mul2(add2(xh[j][k], both(-m)), both(r));
          sg[j][k] = fma2(u[j][k], xh[j][k], sg[j][k]);
          sb[j][k] = add2(sb[j][k], u[j][k]);
          u[j][k] = mul2(u[j][k], gg[j][k]);
          ta = add2(ta, u[j][k]);
          tb = fma2(u[j][k], xh[j][k], tb);
        }
      }
    }
    float2 t = make_float2(ta.x + ta.y, tb.x + tb.y);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      t.x += __shfl_xor_sync(0xffffffffu, t.x, o);
      t.y += __shfl_xor_sync(0xffffffffu, t.y, o);
    }
    float2* rd = red[i & 1];
    if ((threadIdx.x & 31) == 0) rd[threadIdx.x >> 5] = t;
    if (__syncthreads_or(!ok)) {           // the same answer for all threads
      failed = true;
      break;
    }
    if (threadIdx.x == 0 && i + stages < mine) fetch(i + stages);
    t = make_float2(0.f, 0.f);
    for (int w = 0; w < (int)(blockDim.x >> 5); ++w) { t.x += rd[w].x; t.y += rd[w].y; }
    if (dX) {
      const float2 c1 = both(-t.x / (float)n), c2 = both(-t.y / (float)n);
      uint4* out = reinterpret_cast<uint4*>(dX + row * n);
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int v = threadIdx.x + j * blockDim.x;
        if (v < nv) {
#pragma unroll
          for (int k = 0; k < P; ++k) u[j][k] = mul2(fma2(xh[j][k], c2, add2(u[j][k], c1)), both(r));
          out[v] = pack<T>(u[j]);
        }
      }
    }
    m = m1;
    r = r1;
  }
  if (failed) {                            // copies still in flight: time to land before the block's memory goes
    if (threadIdx.x == 0) {
      const uint64_t t0 = tc::global_timer_ns();
      while (tc::global_timer_ns() - t0 < 2000000ull) {
      }
    }
    __syncthreads();
    return;
  }
  if (!part) return;
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int v = threadIdx.x + j * blockDim.x;
    if (v < nv) {
      float* p = part + (int64_t)blockIdx.x * 2 * n + (int64_t)v * E;
#pragma unroll
      for (int k = 0; k < P; k += 2) {
        *reinterpret_cast<float4*>(p + 2 * k) = make_float4(sg[j][k].x, sg[j][k].y, sg[j][k + 1].x, sg[j][k + 1].y);
        *reinterpret_cast<float4*>(p + n + 2 * k) = make_float4(sb[j][k].x, sb[j][k].y, sb[j][k + 1].x, sb[j][k + 1].y);
      }
    }
  }
}

// The same for rows that no 16-byte copy can start at: elements t, t + blockDim.x, ... of a thread, the next row's loaded
// before this one's reduction.
constexpr int ONE_THREADS = 512;

template <typename T, typename TP, int VPT>
__global__ void __launch_bounds__(ONE_THREADS)
ln_grad_one_kernel(const T* __restrict__ dY, int64_t ld_dy, const T* __restrict__ X, int64_t ld, int64_t rows, int n,
                   const TP* __restrict__ g, const float* __restrict__ mean, const float* __restrict__ rstd,
                   T* __restrict__ dX, float* __restrict__ part) {
  __shared__ float2 red[2][16];
  pdl_wait();
  pdl_trigger();
  float gg[VPT], sg[VPT], sb[VPT], x1[VPT], y1[VPT];
  float m1 = 0.f, r1 = 0.f;
  auto fetch = [&](int64_t row) {
    m1 = mean[row];
    r1 = rstd[row];
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int i = threadIdx.x + j * blockDim.x;
      x1[j] = i < n ? to_f32<T>(X[row * ld + i]) : 0.f;
      y1[j] = i < n ? to_f32<T>(dY[row * ld_dy + i]) : 0.f;
    }
  };
  fetch(blockIdx.x);
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int i = threadIdx.x + j * blockDim.x;
    gg[j] = i < n ? param_at(g, i, 1.f) : 0.f;
    sg[j] = sb[j] = 0.f;
  }
  int turn = 0;
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x, turn ^= 1) {
    const float r = r1;
    float u[VPT], xh[VPT];
    float2 t = make_float2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < VPT; ++j) {        // elements past the row: dY and gain are 0
      xh[j] = (x1[j] - m1) * r;
      sg[j] = fmaf(y1[j], xh[j], sg[j]);
      sb[j] += y1[j];
      u[j] = y1[j] * gg[j];
      t.x += u[j];
      t.y = fmaf(u[j], xh[j], t.y);
    }
    if (row + gridDim.x < rows) fetch(row + gridDim.x);
    t = row_sum(t, red[turn]);
    if (dX) {
      t.x /= (float)n;
      t.y /= (float)n;
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int i = threadIdx.x + j * blockDim.x;
        if (i < n) dX[row * n + i] = from_f32<T>((u[j] - t.x - xh[j] * t.y) * r);
      }
    }
  }
  if (!part) return;
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int i = threadIdx.x + j * blockDim.x;
    if (i < n) {
      part[(int64_t)blockIdx.x * 2 * n + i] = sg[j];
      part[((int64_t)blockIdx.x * 2 + 1) * n + i] = sb[j];
    }
  }
}

bool vec16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

// The shape of a row's block: threads in x (rows in y for rows of one warp); vectors a thread: the fewest of `vpts` that need
// no more than 256 threads, else the most.  False where that takes more than `most` threads.
struct RowShape {
  int threads, rows, vpt;
};
bool row_shape(int nv, const int* vpts, int n_vpts, int most, RowShape& s) {
  for (int i = 0; i < n_vpts; ++i) {
    s.vpt = vpts[i];
    s.threads = ((nv + s.vpt - 1) / s.vpt + 31) / 32 * 32;
    if (s.threads <= 256) break;
  }
  s.rows = s.threads == 32 ? 4 : 1;
  return s.threads <= most;
}
constexpr int VEC_VPT[] = {1, 2, 4};       // vectors of 16 bytes
constexpr int ONE_VPT[] = {4, 16};         // single elements

template <typename T, typename TP, int E, int VPT>
int go_rows(Ctx* ctx, const RowShape& s, const void* X, int64_t rows, int n, int64_t ld, const void* g, const void* b,
            float eps, void* Y, float* mean, float* rstd) {
  ZOACT_CUDA_TRY(launch_pdl(ctx, ln_rows_kernel<T, TP, E, VPT>, dim3((unsigned)((rows + s.rows - 1) / s.rows)),
                            dim3(s.threads, s.rows), 0, (const T*)X, ld, rows, n, (const TP*)g, (const TP*)b, eps, (T*)Y, mean,
                            rstd));
  ++ctx->n_launch;
  return ZOACT_OK;
}

template <typename T, typename TP, int VPT>
int go_warp(Ctx* ctx, const void* X, int64_t rows, int n, int64_t ld, const void* g, const void* b, float eps, void* Y,
            float* mean, float* rstd) {
  ZOACT_CUDA_TRY(launch_pdl(ctx, ln_warp_kernel<T, TP, VPT>, dim3((unsigned)((rows + 3) / 4)), dim3(128), 0, (const T*)X, ld, rows,
                            n, (const TP*)g, (const TP*)b, eps, (T*)Y, mean, rstd));
  ++ctx->n_launch;
  return ZOACT_OK;
}

template <typename T, typename TP, int E, int VPT>
int go_grad_rows(Ctx* ctx, const RowShape& s, const void* dY, int64_t ld_dy, const void* X, int64_t rows, int n, int64_t ld,
                 const void* g, const float* mean, const float* rstd, void* dX) {
  ZOACT_CUDA_TRY(launch_pdl(ctx, ln_grad_rows_kernel<T, TP, E, VPT>, dim3((unsigned)((rows + s.rows - 1) / s.rows)),
                            dim3(s.threads, s.rows), 0, (const T*)dY, ld_dy, (const T*)X, ld, rows, n, (const TP*)g, mean, rstd,
                            (T*)dX));
  ++ctx->n_launch;
  return ZOACT_OK;
}

template <typename T, typename TP>
int run_ln(Ctx* ctx, const void* X, int64_t rows, int n, int64_t ld, const void* g, const void* b, float eps, void* Y,
           float* mean, float* rstd) {
  constexpr int E = 16 / (int)sizeof(T);
  RowShape s;
  const bool vec = n % E == 0 && ld % E == 0 && vec16(X) && vec16(Y) && vec16(g) && vec16(b);
  // a warp a row where there are enough rows for that and a row fits in a warp's registers
  if (vec && n / E <= 32 * 20 && rows >= 4 * (int64_t)ctx->sm_count) {
    const int vpt = (n / E + 31) / 32;
    if (vpt <= 4) return go_warp<T, TP, 4>(ctx, X, rows, n, ld, g, b, eps, Y, mean, rstd);
    if (vpt <= 8) return go_warp<T, TP, 8>(ctx, X, rows, n, ld, g, b, eps, Y, mean, rstd);
    if (vpt <= 16) return go_warp<T, TP, 16>(ctx, X, rows, n, ld, g, b, eps, Y, mean, rstd);
    return go_warp<T, TP, 20>(ctx, X, rows, n, ld, g, b, eps, Y, mean, rstd);
  }
  if (vec && row_shape(n / E, VEC_VPT, 3, most_threads(E, false), s)) {
    switch (s.vpt) {
      case 1: return go_rows<T, TP, E, 1>(ctx, s, X, rows, n, ld, g, b, eps, Y, mean, rstd);
      case 2: return go_rows<T, TP, E, 2>(ctx, s, X, rows, n, ld, g, b, eps, Y, mean, rstd);
      default: return go_rows<T, TP, E, 4>(ctx, s, X, rows, n, ld, g, b, eps, Y, mean, rstd);
    }
  }
  if (row_shape(n, ONE_VPT, 2, most_threads(1, false), s))
    return s.vpt == 4 ? go_rows<T, TP, 1, 4>(ctx, s, X, rows, n, ld, g, b, eps, Y, mean, rstd)
                      : go_rows<T, TP, 1, 16>(ctx, s, X, rows, n, ld, g, b, eps, Y, mean, rstd);
  ZOACT_CUDA_TRY(launch_pdl(ctx, ln_long_kernel<T, TP>, dim3((unsigned)rows), dim3(LN_THREADS), 0, (const T*)X, ld, n,
                            (const TP*)g, (const TP*)b, eps, (T*)Y, mean, rstd));
  ++ctx->n_launch;
  return ZOACT_OK;
}

int join_parts(Ctx* ctx, const float* part, int parts, int n, float* dg, float* db) {
  ZOACT_CUDA_TRY(launch_pdl(ctx, ln_join_kernel, dim3((unsigned)((2 * (int64_t)n + 31) / 32)), dim3(1024), 0, part, parts, n, dg, db));
  ++ctx->n_launch;
  return ZOACT_OK;
}

// Blocks an SM runs at once (their registers: up to 112 a thread), and stages of a block's ring: as many as 200 KB hold.
template <typename T, typename TP, int VPT>
int go_ring(Ctx* ctx, int threads, const void* dY, int64_t ld_dy, const void* X, int64_t rows, int n, int64_t ld,
            const void* g, const float* mean, const float* rstd, void* dX, float* dg, float* db) {
  auto kern = ln_grad_ring_kernel<T, TP, VPT>;
  const int per_sm = threads <= 128 ? 4 : threads <= 288 ? 2 : 1;
  const int64_t stage = 2 * (int64_t)n * (int)sizeof(T);
  int stages = (int)(200 * 1024 / per_sm / stage);
  stages = stages > LN_MAX_STAGES ? LN_MAX_STAGES : stages;
  const int smem = (int)(stages * stage);
  ZOACT_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  const int64_t most = (int64_t)ctx->sm_count * per_sm;
  const int blocks = (int)(rows < most ? rows : most);
  float* part = nullptr;
  if (dg || db) {
    part = (float*)scratch(ctx, SLOT_LN, (size_t)blocks * 2 * n * 4);
    if (!part) return ZOACT_ERR_NOMEM;
  }
  ZOACT_CUDA_TRY(launch_pdl(ctx, kern, dim3((unsigned)blocks), dim3(threads), smem, (const T*)dY, ld_dy, (const T*)X, ld, rows, n,
                            (const TP*)g, mean, rstd, (T*)dX, part, stages, ctx->d_status));
  ++ctx->n_launch;
  return part ? join_parts(ctx, part, blocks, n, dg, db) : ZOACT_OK;
}

template <typename T, typename TP, int VPT>
int go_one(Ctx* ctx, int threads, const void* dY, int64_t ld_dy, const void* X, int64_t rows, int n, int64_t ld, const void* g,
           const float* mean, const float* rstd, void* dX, float* dg, float* db) {
  const int64_t most = (int64_t)ctx->sm_count * (threads <= 256 ? 4 : 2);
  const int blocks = (int)(rows < most ? rows : most);
  float* part = nullptr;
  if (dg || db) {
    part = (float*)scratch(ctx, SLOT_LN, (size_t)blocks * 2 * n * 4);
    if (!part) return ZOACT_ERR_NOMEM;
  }
  ZOACT_CUDA_TRY(launch_pdl(ctx, ln_grad_one_kernel<T, TP, VPT>, dim3((unsigned)blocks), dim3(threads), 0, (const T*)dY, ld_dy,
                            (const T*)X, ld, rows, n, (const TP*)g, mean, rstd, (T*)dX, part));
  ++ctx->n_launch;
  return part ? join_parts(ctx, part, blocks, n, dg, db) : ZOACT_OK;
}

template <typename T, typename TP>
int run_ln_grad(Ctx* ctx, const void* dY, int64_t ld_dy, const void* X, int64_t rows, int n, int64_t ld, const void* g,
                const float* mean, const float* rstd, void* dX, float* dg, float* db) {
  constexpr int E = 16 / (int)sizeof(T);
  RowShape s;
  const bool vec = n % E == 0 && ld % E == 0 && ld_dy % E == 0 && vec16(X) && vec16(dY) && vec16(dX) && vec16(g);
  if (rows > 0 && vec && row_shape(n / E, VEC_VPT, RING_VPTS<T>, RING_THREADS, s)) {
    switch (s.vpt) {
      case 1: return go_ring<T, TP, 1>(ctx, s.threads, dY, ld_dy, X, rows, n, ld, g, mean, rstd, dX, dg, db);
      case 2: return go_ring<T, TP, 2>(ctx, s.threads, dY, ld_dy, X, rows, n, ld, g, mean, rstd, dX, dg, db);
      default:
        if constexpr (RING_VPTS<T> == 3)
          return go_ring<T, TP, 4>(ctx, s.threads, dY, ld_dy, X, rows, n, ld, g, mean, rstd, dX, dg, db);
    }
  }
  if (rows > 0 && !vec && row_shape(n, ONE_VPT, 2, ONE_THREADS, s))
    return s.vpt == 4 ? go_one<T, TP, 4>(ctx, s.threads, dY, ld_dy, X, rows, n, ld, g, mean, rstd, dX, dg, db)
                      : go_one<T, TP, 16>(ctx, s.threads, dY, ld_dy, X, rows, n, ld, g, mean, rstd, dX, dg, db);
  int st = ZOACT_OK;
  if (dX && rows > 0) {
    if (vec && row_shape(n / E, VEC_VPT, 3, most_threads(E, true), s)) {       // longer than the ring kernel's rows
      st = go_grad_rows<T, TP, E, 4>(ctx, s, dY, ld_dy, X, rows, n, ld, g, mean, rstd, dX);
    } else {
      ZOACT_CUDA_TRY(launch_pdl(ctx, ln_grad_long_kernel<T, TP>, dim3((unsigned)rows), dim3(LN_THREADS), 0, (const T*)dY, ld_dy,
                                (const T*)X, ld, n, (const TP*)g, mean, rstd, (T*)dX));
      ++ctx->n_launch;
    }
  }
  if (st || (!dg && !db)) return st;
  // ranges of at least 16 rows, as many as give an SM four blocks
  const int cols = (n + LN_THREADS - 1) / LN_THREADS;
  int64_t ranges = (4 * (int64_t)ctx->sm_count + cols - 1) / cols;
  const int64_t by_rows = (rows + 15) / 16;
  ranges = ranges < by_rows ? ranges : by_rows;
  if (ranges < 1) ranges = 1;
  const int64_t per = (rows + ranges - 1) / ranges;
  float* part = (float*)scratch(ctx, SLOT_LN, (size_t)ranges * 2 * n * 4);
  if (!part) return ZOACT_ERR_NOMEM;
  ZOACT_CUDA_TRY(launch_pdl(ctx, ln_grad_cols_kernel<T>, dim3((unsigned)cols, (unsigned)ranges), dim3(LN_THREADS), 0, (const T*)dY,
                            ld_dy, (const T*)X, ld, rows, n, mean, rstd, per, part));
  ++ctx->n_launch;
  return join_parts(ctx, part, (int)ranges, n, dg, db);
}

}  // namespace

int launch_layer_norm(Ctx* ctx, const void* X, int dtype, int64_t rows, int n, int64_t ld, const void* g, const void* b,
                      int pdtype, float eps, void* Y, float* mean, float* rstd) {
  if (rows == 0) return ZOACT_OK;
  const bool pf = pdtype == ZOACT_DT_FP32;
  switch (dtype) {
    case ZOACT_DT_FP32: return run_ln<float, float>(ctx, X, rows, n, ld, g, b, eps, Y, mean, rstd);
    case ZOACT_DT_BF16:
      return pf ? run_ln<__nv_bfloat16, float>(ctx, X, rows, n, ld, g, b, eps, Y, mean, rstd)
                : run_ln<__nv_bfloat16, __nv_bfloat16>(ctx, X, rows, n, ld, g, b, eps, Y, mean, rstd);
    default:
      return pf ? run_ln<__half, float>(ctx, X, rows, n, ld, g, b, eps, Y, mean, rstd)
                : run_ln<__half, __half>(ctx, X, rows, n, ld, g, b, eps, Y, mean, rstd);
  }
}

int launch_layer_norm_grad(Ctx* ctx, const void* dY, int64_t ld_dy, const void* X, int dtype, int64_t rows, int n,
                           int64_t ld, const void* g, int pdtype, const float* mean, const float* rstd, void* dX,
                           float* dg, float* db) {
  const bool pf = pdtype == ZOACT_DT_FP32;
  switch (dtype) {
    case ZOACT_DT_FP32: return run_ln_grad<float, float>(ctx, dY, ld_dy, X, rows, n, ld, g, mean, rstd, dX, dg, db);
    case ZOACT_DT_BF16:
      return pf ? run_ln_grad<__nv_bfloat16, float>(ctx, dY, ld_dy, X, rows, n, ld, g, mean, rstd, dX, dg, db)
                : run_ln_grad<__nv_bfloat16, __nv_bfloat16>(ctx, dY, ld_dy, X, rows, n, ld, g, mean, rstd, dX, dg, db);
    default:
      return pf ? run_ln_grad<__half, float>(ctx, dY, ld_dy, X, rows, n, ld, g, mean, rstd, dX, dg, db)
                : run_ln_grad<__half, __half>(ctx, dY, ld_dy, X, rows, n, ld, g, mean, rstd, dX, dg, db);
  }
}

}  // namespace zoact
