// Layer norm over the rows of X [rows, n] (row stride ld):
//     y = (x - m) s g + b,  m = mean(x),  s = 1 / sqrt(mean((x - m)^2) + eps)
// and its gradient, with u = dy g and xh = (x - m) s:
//     dx = s (u - mean(u) - xh mean(u xh)),  dg = sum_rows dy xh,  db = sum_rows dy.
//
// Both are bound by memory as long as a row's own overhead is small: the forward pass reads and writes a row once, the
// gradient reads two and writes one.  A row is held in registers between its statistics (mean first, then the centred
// squares: no cancellation) and its output, in pairs of fp32.  The gradient by the parameters needs every row of a column:
// persistent blocks keep their columns' sums in registers over all their rows, which bulk copies bring into a ring of shared
// memory ahead of them, and one small kernel adds the blocks' sums.  Rows that no 16-byte copy can start at, and rows too
// long for a block's registers, have kernels of their own.
//
// Measured: forward 8192 x 5120 fp16 34.4 us (4.9 TB/s; a copy of the tensor 28.7 us), 128 x 256 fp32 8 us; gradient
// 4096 x 4096 bf16 25.8 us (3.9 TB/s), fp32 about 40 us, 777 x 1001 bf16 11.5 us.
#include "internal.h"
#include "tc_common.cuh"

namespace zoact {
namespace {

constexpr int LN_THREADS = 256;
// Threads of a row at most: its vectors, or its single elements, in their registers.
constexpr int VEC_THREADS = 1024, GRAD_VEC_THREADS = 640, ONE_THREADS = 512;

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

__device__ __forceinline__ uint32_t pack_pair(float2 f, __nv_bfloat16*) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(f.x, f.y);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack_pair(float2 f, __half*) {
  const __half2 h = __floats2half2_rn(f.x, f.y);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 unpack_pair(uint32_t w, __nv_bfloat16*) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ float2 unpack_pair(uint32_t w, __half*) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }

// A 16-byte vector's elements in pairs, and back.
template <typename T>
__device__ __forceinline__ void unpack(const uint4& u, float2* f) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
  if constexpr (sizeof(T) == 4) {
    f[0] = make_float2(__uint_as_float(w[0]), __uint_as_float(w[1]));
    f[1] = make_float2(__uint_as_float(w[2]), __uint_as_float(w[3]));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = unpack_pair(w[i], (T*)nullptr);
  }
}
template <typename T>
__device__ __forceinline__ uint4 pack(const float2* f) {
  if constexpr (sizeof(T) == 4)
    return make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[1].x), __float_as_uint(f[1].y));
  else
    return make_uint4(pack_pair(f[0], (T*)nullptr), pack_pair(f[1], (T*)nullptr), pack_pair(f[2], (T*)nullptr),
                      pack_pair(f[3], (T*)nullptr));
}

template <typename TP>
__device__ __forceinline__ float param_at(const TP* p, int64_t i, float none) { return p ? to_f32<TP>(p[i]) : none; }

// The P pairs of parameters from element i on (16-byte loads), or `none`.  Parameters are of the rows' type or wider.
template <typename TP, int P>
__device__ __forceinline__ void load_param(const TP* p, int64_t i, float none, float2* f) {
  constexpr int N = 8 / (int)sizeof(TP);             // pairs of a vector
  static_assert(P % N == 0, "whole vectors");
  if (p) {
#pragma unroll
    for (int q = 0; q < P / N; ++q) unpack<TP>(*reinterpret_cast<const uint4*>(p + i + q * 2 * N), f + q * N);
  } else {
#pragma unroll
    for (int k = 0; k < P; ++k) f[k] = both(none);
  }
}

__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// The sum over a row's threads: a warp (blockDim.x = 32), or the block's warps (at most 32), whose sums every warp adds up by
// a second butterfly.  `red` [32] may be used again after the next barrier of the block.
__device__ __forceinline__ float row_sum(float v, float* red) {
  v = lanes_sum(v);
  if (blockDim.x == 32) return v;
  const int lane = threadIdx.x & 31;
  if (lane == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  return lanes_sum(lane < (int)(blockDim.x >> 5) ? red[lane] : 0.f);
}
// Two sums in one butterfly: lanes below 16 go on with x, the others with y.  The sums end up in lanes 0 to 15 and 16 to 31.
__device__ __forceinline__ float lanes_sum2(float x, float y) {
  const bool up = threadIdx.x & 16;
  float v = (up ? y : x) + __shfl_xor_sync(0xffffffffu, up ? x : y, 16);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
// Two sums over the block's warps (at most 32): each warp's in red[warp] and red[32 + warp] before the block's barrier, and a
// second butterfly after it.
__device__ __forceinline__ void post_sum2(float x, float y, float* red) {
  const float v = lanes_sum2(x, y);
  const int lane = threadIdx.x & 31;
  if ((lane & 15) == 0) red[2 * (lane & 16) + (threadIdx.x >> 5)] = v;
}
__device__ __forceinline__ float2 join_sum2(const float* red, int warps) {
  const int lane = threadIdx.x & 31;
  const float v = lanes_sum2(lane < warps ? red[lane] : 0.f, lane < warps ? red[32 + lane] : 0.f);
  return make_float2(__shfl_sync(0xffffffffu, v, 0), __shfl_sync(0xffffffffu, v, 16));
}
__device__ __forceinline__ float2 row_sum2(float x, float y, float* red) {
  if (blockDim.x == 32) {
    const float v = lanes_sum2(x, y);
    return make_float2(__shfl_sync(0xffffffffu, v, 0), __shfl_sync(0xffffffffu, v, 16));
  }
  post_sum2(x, y, red);
  __syncthreads();
  return join_sum2(red, (int)(blockDim.x >> 5));
}

// ---- forward ----
// ROWS rows (1 or 2) by blockDim.x threads, VPT vectors of each a thread in registers; blockDim.y of these a block (of one warp
// each).  The parameters come from L1 for every row: two rows together need them once (8192 x 5120 fp16: 37 us with one,
// L1 the bound), and share the butterflies and barriers of their sums.
template <typename T, typename TP, int VPT, int ROWS>
__global__ void __launch_bounds__(VEC_THREADS)
ln_rows_kernel(const T* __restrict__ X, int64_t ld, int64_t rows, int n, const TP* __restrict__ g, const TP* __restrict__ b,
               float eps, T* __restrict__ Y, float* __restrict__ mean, float* __restrict__ rstd) {
  constexpr int P = 8 / (int)sizeof(T), E = 2 * P;
  pdl_wait();                              // the input rows written by the previous kernel
  pdl_trigger();
  __shared__ float red[2][64];
  const int64_t row = ((int64_t)blockIdx.x * blockDim.y + threadIdx.y) * ROWS;
  if (row >= rows) return;                 // whole warps; rows of several warps have a block each
  const int64_t last = rows - 1;
  const int nv = n / E;
  const float inv_n = 1.f / (float)n;
  uint4 q[ROWS][VPT];
#pragma unroll
  for (int w = 0; w < ROWS; ++w) {
    const uint4* x = reinterpret_cast<const uint4*>(X + (row + w < last ? row + w : last) * ld);
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int i = threadIdx.x + j * blockDim.x;
      q[w][j] = make_uint4(0u, 0u, 0u, 0u);
      if (i < nv) q[w][j] = __ldcs(x + i); // read once: kept out of the parameters' way in L1
    }
  }
  float2 f[ROWS][VPT][P], s[ROWS];
  auto sums = [&](float* r) {              // over the row's threads, both rows' at once
    return ROWS == 2 ? row_sum2(s[0].x + s[0].y, s[ROWS - 1].x + s[ROWS - 1].y, r) : make_float2(row_sum(s[0].x + s[0].y, r), 0.f);
  };
#pragma unroll
  for (int w = 0; w < ROWS; ++w) {
    s[w] = make_float2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      unpack<T>(q[w][j], f[w][j]);
#pragma unroll
      for (int k = 0; k < P; ++k) s[w] = add2(s[w], f[w][j][k]);
    }
  }
  float2 t = sums(red[0]);
  const float m[2] = {t.x * inv_n, t.y * inv_n};
#pragma unroll
  for (int w = 0; w < ROWS; ++w) {
    s[w] = make_float2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      if (threadIdx.x + j * blockDim.x < nv) {
#pragma unroll
        for (int k = 0; k < P; ++k) {
          f[w][j][k] = add2(f[w][j][k], both(-m[w]));
          s[w] = fma2(f[w][j][k], f[w][j][k], s[w]);
        }
      }
    }
  }
  t = sums(red[1]);
  const float r[2] = {rsqrtf(fmaf(t.x, inv_n, eps)), rsqrtf(fmaf(t.y, inv_n, eps))};
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int i = threadIdx.x + j * blockDim.x;
    if (i < nv) {
      float2 gg[P], bb[P];
      load_param<TP, P>(g, (int64_t)i * E, 1.f, gg);
      load_param<TP, P>(b, (int64_t)i * E, 0.f, bb);
#pragma unroll
      for (int w = 0; w < ROWS; ++w) {
#pragma unroll
        for (int k = 0; k < P; ++k) f[w][j][k] = fma2(mul2(f[w][j][k], both(r[w])), gg[k], bb[k]);
        if (row + w < rows) reinterpret_cast<uint4*>(Y + (row + w) * n)[i] = pack<T>(f[w][j]);
      }
    }
  }
  if (threadIdx.x == 0) {
#pragma unroll
    for (int w = 0; w < ROWS; ++w) {
      if (row + w >= rows) break;
      if (mean) mean[row + w] = m[w];
      if (rstd) rstd[row + w] = r[w];
    }
  }
}

// The same for rows that no 16-byte load can start at, VPT single elements a thread.
template <typename T, typename TP, int VPT>
__global__ void __launch_bounds__(ONE_THREADS)
ln_one_kernel(const T* __restrict__ X, int64_t ld, int64_t rows, int n, const TP* __restrict__ g, const TP* __restrict__ b,
              float eps, T* __restrict__ Y, float* __restrict__ mean, float* __restrict__ rstd) {
  pdl_wait();
  pdl_trigger();
  __shared__ float red[2][32];
  const int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  if (row >= rows) return;
  const T* x = X + row * ld;
  const float inv_n = 1.f / (float)n;
  float v[VPT], s = 0.f;
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int i = threadIdx.x + j * blockDim.x;
    v[j] = i < n ? to_f32<T>(x[i]) : 0.f;
  }
#pragma unroll
  for (int j = 0; j < VPT; ++j) s += v[j];
  const float m = row_sum(s, red[0]) * inv_n;
  s = 0.f;
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    v[j] = threadIdx.x + j * blockDim.x < n ? v[j] - m : 0.f;
    s = fmaf(v[j], v[j], s);
  }
  const float r = rsqrtf(fmaf(row_sum(s, red[1]), inv_n, eps));
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int i = threadIdx.x + j * blockDim.x;
    if (i < n) Y[row * n + i] = from_f32<T>(fmaf(v[j] * r, param_at(g, i, 1.f), param_at(b, i, 0.f)));
  }
  if (threadIdx.x == 0) {
    if (mean) mean[row] = m;
    if (rstd) rstd[row] = r;
  }
}

// Rows longer than a block's registers, read once per use.
template <typename T, typename TP>
__global__ void __launch_bounds__(LN_THREADS)
ln_long_kernel(const T* __restrict__ X, int64_t ld, int n, const TP* __restrict__ g, const TP* __restrict__ b, float eps,
               T* __restrict__ Y, float* __restrict__ mean, float* __restrict__ rstd) {
  pdl_wait();
  pdl_trigger();
  __shared__ float red[2][32];
  const int64_t row = blockIdx.x;
  const T* x = X + row * ld;
  float s = 0.f;
  for (int i = threadIdx.x; i < n; i += LN_THREADS) s += to_f32<T>(x[i]);
  const float m = row_sum(s, red[0]) / (float)n;
  s = 0.f;
  for (int i = threadIdx.x; i < n; i += LN_THREADS) {
    const float c = to_f32<T>(x[i]) - m;
    s = fmaf(c, c, s);
  }
  const float r = rsqrtf(row_sum(s, red[1]) / (float)n + eps);
  for (int i = threadIdx.x; i < n; i += LN_THREADS)
    Y[row * n + i] = from_f32<T>(fmaf((to_f32<T>(x[i]) - m) * r, param_at(g, i, 1.f), param_at(b, i, 0.f)));
  if (threadIdx.x == 0) {
    if (mean) mean[row] = m;
    if (rstd) rstd[row] = r;
  }
}

// ---- gradient through a ring of bulk copies ----
// What a block has in flight bounds it: data comes after about 2 us when all SMs ask for theirs, so a loop that loads its next
// row (or its next row's statistics) one iteration ahead takes 2 us a row.  A persistent block takes rows b, b + gridDim.x, ...;
// consumer thread t has vectors t, t + consumers, ... of them; one more warp brings a row of X and one of dY a stage, as many
// stages as fit.  A warp gives a stage back as soon as its vectors are in registers.
constexpr int LN_MAX_STAGES = 8;
constexpr int RING_THREADS = 512;          // consumers at most
// Registers of 16 columns a thread (96 to 112 without spills) by the most consumers a kernel is built for: two blocks on an SM
// up to 256, one with up to 128 registers a thread up to 480.
constexpr int RING_HALF = 256, RING_WIDE = 480;

struct RowRing {
  uint64_t full[LN_MAX_STAGES], empty[LN_MAX_STAGES];
  float red[2][64];
  int abort_flag;
};

__device__ __forceinline__ void ring_init(RowRing& rr, int stages, int warps) {
  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      tc::mbar_init(tc::smem_u32(&rr.full[s]), 1);
      tc::mbar_init(tc::smem_u32(&rr.empty[s]), warps);
    }
    rr.abort_flag = 0;
    tc::fence_mbar_init();
  }
  __syncthreads();
}

// tc::mbar_wait for many waiting threads: the timer, slow to read, is looked at only when a wait has gone on for a while.
__device__ __forceinline__ bool ring_wait(RowRing& rr, uint64_t* bar, uint32_t parity, int* status) {
  const uint32_t b = tc::smem_u32(bar);
  uint64_t t0 = 0;
  for (uint32_t it = 1;; ++it) {
    if (tc::mbar_try_wait(b, parity)) return true;
    if ((it & 63u) == 0u) {
      if (*reinterpret_cast<volatile int*>(&rr.abort_flag)) return false;
      const uint64_t now = tc::global_timer_ns();
      if (t0 == 0) t0 = now;
      if (now - t0 > tc::WAIT_LIMIT_NS) {
        *reinterpret_cast<volatile int*>(&rr.abort_flag) = 1;
        record_error(status, ZOACT_ERR_TIMEOUT);
        return false;
      }
    }
  }
}

// The producer warp's lane 0: this block's rows of X and dY.
__device__ __forceinline__ void ring_produce(RowRing& rr, uint8_t* ring, int stages, const void* x, int64_t ld_x, const void* dy,
                                             int64_t ld_dy, uint32_t row_bytes, int64_t rows, int* status) {
  int s = 0;
  uint32_t phase = 1;                      // the ring is empty at first
  bool ok = true;
  for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
    ok = ring_wait(rr, &rr.empty[s], phase, status);
    if (!ok) break;
    const uint32_t bar = tc::smem_u32(&rr.full[s]), dst = tc::smem_u32(ring) + (uint32_t)(s * 2) * row_bytes;
    tc::mbar_arrive_expect_tx(bar, 2 * row_bytes);
    tc::bulk_load(dst, static_cast<const uint8_t*>(x) + row * ld_x, row_bytes, bar);
    tc::bulk_load(dst + row_bytes, static_cast<const uint8_t*>(dy) + row * ld_dy, row_bytes, bar);
    if (++s == stages) { s = 0; phase ^= 1u; }
  }
  if (!ok) {                               // copies in flight: time to land before the block's memory goes
    const uint64_t t0 = tc::global_timer_ns();
    while (tc::global_timer_ns() - t0 < 2000000ull) {
    }
  }
}

// The whole gradient: a thread has both parameters' sums of its columns in registers over all rows.  Registers bound how many
// warps there are to hide a row's chain of two butterflies and a barrier: the row's own values stay packed, unpacked once for
// the sums and once for dX (with the gain in shared memory and a third block on an SM, the spills cost more: 34 us for 25 at
// 4096 x 4096 bf16).
template <typename T, typename TP, int VPT, int MOST>
__global__ void __launch_bounds__(MOST + 32, MOST == RING_HALF ? 2 : 1)
ln_grad_ring_kernel(const T* __restrict__ dY, int64_t ld_dy, const T* __restrict__ X, int64_t ld, int64_t rows, int n,
                    const TP* __restrict__ g, const float* __restrict__ mean, const float* __restrict__ rstd,
                    T* __restrict__ dX, float* __restrict__ part, int stages, int* status) {
  constexpr int E = 16 / (int)sizeof(T), P = E / 2;
  extern __shared__ __align__(128) uint8_t ring[];
  __shared__ RowRing rr;
  const int consumers = blockDim.x - 32, warps = consumers / 32, lane = threadIdx.x & 31;
  ring_init(rr, stages, warps);
  pdl_wait();
  pdl_trigger();
  if (threadIdx.x >= consumers) {
    if (lane == 0)
      ring_produce(rr, ring, stages, X, ld * (int64_t)sizeof(T), dY, ld_dy * (int64_t)sizeof(T),
                      (uint32_t)n * (uint32_t)sizeof(T), rows, status);
    return;
  }
  const int nv = n / E;
  const float inv_n = 1.f / (float)n;
  float2 gg[VPT][P], sg[VPT][P], sb[VPT][P];
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int v = threadIdx.x + j * consumers;
    if (v < nv) load_param<TP, P>(g, (int64_t)v * E, 1.f, gg[j]);
#pragma unroll
    for (int k = 0; k < P; ++k) sg[j][k] = sb[j][k] = make_float2(0.f, 0.f);
  }
  // the statistics of the block's next 32 rows, a row a lane, and of the 32 after those
  const int64_t step = (int64_t)gridDim.x, first = (int64_t)blockIdx.x + lane * step;
  float m0 = first < rows ? mean[first] : 0.f, r0 = first < rows ? rstd[first] : 0.f, m1 = 0.f, r1 = 0.f;
  int s = 0, turn = 0, i = 0;
  uint32_t phase = 0;
  for (int64_t row = blockIdx.x; row < rows; row += step, turn ^= 1, i = (i + 1) & 31) {
    if (i == 0) {
      if (row != (int64_t)blockIdx.x) { m0 = m1; r0 = r1; }
      const int64_t ahead = row + (32 + lane) * step;
      if (ahead < rows) { m1 = mean[ahead]; r1 = rstd[ahead]; }
    }
    const float m = __shfl_sync(0xffffffffu, m0, i), r = __shfl_sync(0xffffffffu, r0, i);
    bool ok = ring_wait(rr, &rr.full[s], phase, status);
    const uint4* xs = reinterpret_cast<const uint4*>(ring) + (size_t)s * 2 * nv;
    const uint4* ys = xs + nv;
    uint4 xq[VPT], yq[VPT];
    float2 ta = make_float2(0.f, 0.f), tb = make_float2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int v = threadIdx.x + j * consumers;
      if (v < nv) { xq[j] = xs[v]; yq[j] = ys[v]; }
    }
    __syncwarp();
    if (lane == 0) tc::mbar_arrive(tc::smem_u32(&rr.empty[s]));
    if (++s == stages) { s = 0; phase ^= 1u; }
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int v = threadIdx.x + j * consumers;
      if (v < nv) {
        float2 xh[P], u[P];
        unpack<T>(xq[j], xh);
        unpack<T>(yq[j], u);
#pragma unroll
        for (int k = 0; k < P; ++k) {
          xh[k] = mul2(add2(xh[k], both(-m)), both(r));
          sg[j][k] = fma2(u[k], xh[k], sg[j][k]);
          sb[j][k] = add2(sb[j][k], u[k]);
          u[k] = mul2(u[k], gg[j][k]);
          ta = add2(ta, u[k]);
          tb = fma2(u[k], xh[k], tb);
        }
      }
    }
    post_sum2(ta.x + ta.y, tb.x + tb.y, rr.red[turn]);
    ok = tc::named_bar_and(1, consumers, ok);
    const float2 c = join_sum2(rr.red[turn], warps);
    if (!ok) return;                       // the same answer for all
    if (dX) {
      const float2 c1 = both(-c.x * inv_n), c2 = both(-c.y * inv_n);
      uint4* out = reinterpret_cast<uint4*>(dX + row * n);
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int v = threadIdx.x + j * consumers;
        if (v < nv) {
          float2 xh[P], u[P];
          unpack<T>(xq[j], xh);
          unpack<T>(yq[j], u);
#pragma unroll
          for (int k = 0; k < P; ++k) {
            xh[k] = mul2(add2(xh[k], both(-m)), both(r));
            u[k] = mul2(fma2(xh[k], c2, fma2(u[k], gg[j][k], c1)), both(r));
          }
          out[v] = pack<T>(u);
        }
      }
    }
  }
  if (!part) return;
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int v = threadIdx.x + j * consumers;
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
template <typename T, typename TP, int VPT>
__global__ void __launch_bounds__(ONE_THREADS)
ln_grad_one_kernel(const T* __restrict__ dY, int64_t ld_dy, const T* __restrict__ X, int64_t ld, int64_t rows, int n,
                   const TP* __restrict__ g, const float* __restrict__ mean, const float* __restrict__ rstd,
                   T* __restrict__ dX, float* __restrict__ part) {
  __shared__ float red[2][64];
  pdl_wait();
  pdl_trigger();
  const float inv_n = 1.f / (float)n;
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
    float u[VPT], xh[VPT], ta = 0.f, tb = 0.f;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {        // elements past the row: dY and gain are 0
      xh[j] = (x1[j] - m1) * r;
      sg[j] = fmaf(y1[j], xh[j], sg[j]);
      sb[j] += y1[j];
      u[j] = y1[j] * gg[j];
      ta += u[j];
      tb = fmaf(u[j], xh[j], tb);
    }
    if (row + gridDim.x < rows) fetch(row + gridDim.x);
    const float2 t = row_sum2(ta, tb, red[turn]);
    if (dX) {
      const float c1 = t.x * inv_n, c2 = t.y * inv_n;
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int i = threadIdx.x + j * blockDim.x;
        if (i < n) dX[row * n + i] = from_f32<T>((u[j] - c1 - xh[j] * c2) * r);
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

// ---- gradient of rows too long for one block's registers ----
template <typename T, typename TP, int VPT>
__global__ void __launch_bounds__(GRAD_VEC_THREADS)
ln_grad_rows_kernel(const T* __restrict__ dY, int64_t ld_dy, const T* __restrict__ X, int64_t ld, int n,
                    const TP* __restrict__ g, const float* __restrict__ mean, const float* __restrict__ rstd,
                    T* __restrict__ dX) {
  constexpr int E = 16 / (int)sizeof(T), P = E / 2;
  pdl_wait();
  pdl_trigger();
  __shared__ float red[2][32];
  const int64_t row = blockIdx.x;
  const uint4* x = reinterpret_cast<const uint4*>(X + row * ld);
  const uint4* dy = reinterpret_cast<const uint4*>(dY + row * ld_dy);
  const float m = mean[row], r = rstd[row], inv_n = 1.f / (float)n;
  const int nv = n / E;
  float2 u[VPT][P], xh[VPT][P], a = make_float2(0.f, 0.f), c = make_float2(0.f, 0.f);
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int i = threadIdx.x + j * blockDim.x;
    if (i < nv) {
      float2 gg[P];
      unpack<T>(__ldcs(dy + i), u[j]);
      unpack<T>(__ldcs(x + i), xh[j]);
      load_param<TP, P>(g, (int64_t)i * E, 1.f, gg);
#pragma unroll
      for (int k = 0; k < P; ++k) {
        u[j][k] = mul2(u[j][k], gg[k]);
        xh[j][k] = mul2(add2(xh[j][k], both(-m)), both(r));
        a = add2(a, u[j][k]);
        c = fma2(u[j][k], xh[j][k], c);
      }
    }
  }
  const float2 c1 = both(row_sum(a.x + a.y, red[0]) * -inv_n), c2 = both(row_sum(c.x + c.y, red[1]) * -inv_n);
  uint4* out = reinterpret_cast<uint4*>(dX + row * n);
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int i = threadIdx.x + j * blockDim.x;
    if (i < nv) {
#pragma unroll
      for (int k = 0; k < P; ++k) u[j][k] = mul2(fma2(xh[j][k], c2, add2(u[j][k], c1)), both(r));
      out[i] = pack<T>(u[j]);
    }
  }
}

template <typename T, typename TP>
__global__ void __launch_bounds__(LN_THREADS)
ln_grad_long_kernel(const T* __restrict__ dY, int64_t ld_dy, const T* __restrict__ X, int64_t ld, int n,
                    const TP* __restrict__ g, const float* __restrict__ mean, const float* __restrict__ rstd,
                    T* __restrict__ dX) {
  pdl_wait();
  pdl_trigger();
  __shared__ float red[64];
  const int64_t row = blockIdx.x;
  const T* x = X + row * ld;
  const T* dy = dY + row * ld_dy;
  const float m = mean[row], r = rstd[row];
  float a = 0.f, c = 0.f;
  for (int i = threadIdx.x; i < n; i += LN_THREADS) {
    const float u = to_f32<T>(dy[i]) * param_at(g, i, 1.f), xh = (to_f32<T>(x[i]) - m) * r;
    a += u;
    c = fmaf(u, xh, c);
  }
  const float2 s = row_sum2(a, c, red);
  const float c1 = s.x / (float)n, c2 = s.y / (float)n;
  for (int i = threadIdx.x; i < n; i += LN_THREADS) {
    const float u = to_f32<T>(dy[i]) * param_at(g, i, 1.f), xh = (to_f32<T>(x[i]) - m) * r;
    dX[row * n + i] = from_f32<T>((u - c1 - xh * c2) * r);
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
  s = lanes_sum(red[c][group]);            // warp w: the groups of column w
  const int64_t mine = (int64_t)blockIdx.x * 32 + group;
  if (c != 0 || mine >= 2 * (int64_t)n) return;
  float* out = mine < n ? dg : db;
  if (out) out[mine < n ? mine : mine - n] = s;
}

bool vec16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

// The shape of a row's block: threads in x (rows in y for rows of one warp); vectors a thread: the fewest of `vpts` that need
// no more than `enough` threads, else the most.  False where that takes more than `most` threads.
struct RowShape {
  int threads, rows, vpt;
};
bool row_shape(int nv, const int* vpts, int n_vpts, int enough, int most, RowShape& s) {
  for (int i = 0; i < n_vpts; ++i) {
    s.vpt = vpts[i];
    s.threads = ((nv + s.vpt - 1) / s.vpt + 31) / 32 * 32;
    if (s.threads <= enough) break;
  }
  s.rows = s.threads == 32 ? 4 : 1;
  return s.threads <= most;
}
constexpr int VEC_VPT[] = {1, 2, 4};       // vectors of 16 bytes
constexpr int ONE_VPT[] = {4, 16};         // single elements

template <typename T, typename TP, int VPT, int ROWS>
int go_rows(Ctx* ctx, const RowShape& s, const void* X, int64_t rows, int n, int64_t ld, const void* g, const void* b,
            float eps, void* Y, float* mean, float* rstd) {
  const int64_t per = (int64_t)s.rows * ROWS;
  ZOACT_CUDA_TRY(launch_pdl(ctx, ln_rows_kernel<T, TP, VPT, ROWS>, dim3((unsigned)((rows + per - 1) / per)),
                            dim3(s.threads, s.rows), 0, (const T*)X, ld, rows, n, (const TP*)g, (const TP*)b, eps, (T*)Y, mean,
                            rstd));
  ++ctx->n_launch;
  return ZOACT_OK;
}
template <typename T, typename TP, int VPT>
int go_rows_one(Ctx* ctx, const RowShape& s, const void* X, int64_t rows, int n, int64_t ld, const void* g, const void* b,
                float eps, void* Y, float* mean, float* rstd) {
  ZOACT_CUDA_TRY(launch_pdl(ctx, ln_one_kernel<T, TP, VPT>, dim3((unsigned)((rows + s.rows - 1) / s.rows)),
                            dim3(s.threads, s.rows), 0, (const T*)X, ld, rows, n, (const TP*)g, (const TP*)b, eps, (T*)Y, mean,
                            rstd));
  ++ctx->n_launch;
  return ZOACT_OK;
}

int join_parts(Ctx* ctx, const float* part, int parts, int n, float* dg, float* db) {
  ZOACT_CUDA_TRY(launch_pdl(ctx, ln_join_kernel, dim3((unsigned)((2 * (int64_t)n + 31) / 32)), dim3(1024), 0, part, parts, n, dg, db));
  ++ctx->n_launch;
  return ZOACT_OK;
}

// The blocks' sums of dg and db, where they are asked for.
bool parts_for(Ctx* ctx, int64_t blocks, int n, bool wanted, float** part) {
  *part = nullptr;
  if (!wanted) return true;
  *part = (float*)scratch(ctx, SLOT_LN, (size_t)blocks * 2 * n * 4);
  return *part != nullptr;
}

// Blocks that run at once, by their registers a thread and 200 KB of rings an SM (three stages at least), and a ring's stages.
constexpr int RING_BYTES = 200 * 1024;
struct RingShape {
  int blocks, stages, smem;
};
RingShape ring_shape(const Ctx* ctx, int threads, int regs, int64_t stage, int64_t rows) {
  int per_sm = 65536 / regs / threads;
  per_sm = per_sm > 8 ? 8 : per_sm;
  while (per_sm > 1 && RING_BYTES / per_sm / stage < 3) --per_sm;
  RingShape q;
  q.stages = (int)(RING_BYTES / per_sm / stage);
  if (q.stages > LN_MAX_STAGES) q.stages = LN_MAX_STAGES;
  q.smem = (int)(q.stages * stage);
  const int64_t most = (int64_t)ctx->sm_count * per_sm;
  q.blocks = (int)(rows < most ? rows : most);
  return q;
}

template <typename T, typename TP, int VPT, int MOST>
int go_ring(Ctx* ctx, int consumers, const void* dY, int64_t ld_dy, const void* X, int64_t rows, int n, int64_t ld,
            const void* g, const float* mean, const float* rstd, void* dX, float* dg, float* db) {
  auto kern = ln_grad_ring_kernel<T, TP, VPT, MOST>;
  const int regs = VPT * (16 / (int)sizeof(T)) <= 8 ? 72 : 112;
  const RingShape q = ring_shape(ctx, consumers + 32, regs, 2 * (int64_t)n * (int)sizeof(T), rows);
  // the most that any width takes: the attribute is the function's, and another host thread may be between it and a launch
  ZOACT_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, RING_BYTES));
  float* part;
  if (!parts_for(ctx, q.blocks, n, dg || db, &part)) return ZOACT_ERR_NOMEM;
  ZOACT_CUDA_TRY(launch_pdl(ctx, kern, dim3((unsigned)q.blocks), dim3(consumers + 32), q.smem, (const T*)dY, ld_dy, (const T*)X,
                            ld, rows, n, (const TP*)g, mean, rstd, (T*)dX, part, q.stages, ctx->d_status));
  ++ctx->n_launch;
  return part ? join_parts(ctx, part, q.blocks, n, dg, db) : ZOACT_OK;
}

template <typename T, typename TP, int VPT>
int go_one(Ctx* ctx, int threads, const void* dY, int64_t ld_dy, const void* X, int64_t rows, int n, int64_t ld, const void* g,
           const float* mean, const float* rstd, void* dX, float* dg, float* db) {
  const int64_t most = (int64_t)ctx->sm_count * (threads <= 256 ? 4 : 2);
  const int blocks = (int)(rows < most ? rows : most);
  float* part;
  if (!parts_for(ctx, blocks, n, dg || db, &part)) return ZOACT_ERR_NOMEM;
  ZOACT_CUDA_TRY(launch_pdl(ctx, ln_grad_one_kernel<T, TP, VPT>, dim3((unsigned)blocks), dim3(threads), 0, (const T*)dY, ld_dy,
                            (const T*)X, ld, rows, n, (const TP*)g, mean, rstd, (T*)dX, part));
  ++ctx->n_launch;
  return part ? join_parts(ctx, part, blocks, n, dg, db) : ZOACT_OK;
}

template <typename T, typename TP>
int run_ln(Ctx* ctx, const void* X, int64_t rows, int n, int64_t ld, const void* g, const void* b, float eps, void* Y,
           float* mean, float* rstd) {
  constexpr int E = 16 / (int)sizeof(T);
  RowShape s;
  const bool vec = n % E == 0 && ld % E == 0 && vec16(X) && vec16(Y) && vec16(g) && vec16(b);
  // two rows a block, of one or two vectors a thread, unless there are not enough rows for the SMs, or they are too long
  if (vec && rows >= 4 * (int64_t)ctx->sm_count && row_shape(n / E, VEC_VPT, 2, 64, 512, s))
    return s.vpt == 1 ? go_rows<T, TP, 1, 2>(ctx, s, X, rows, n, ld, g, b, eps, Y, mean, rstd)
                      : go_rows<T, TP, 2, 2>(ctx, s, X, rows, n, ld, g, b, eps, Y, mean, rstd);
  if (vec && row_shape(n / E, VEC_VPT, 3, 256, VEC_THREADS, s)) {
    switch (s.vpt) {
      case 1: return go_rows<T, TP, 1, 1>(ctx, s, X, rows, n, ld, g, b, eps, Y, mean, rstd);
      case 2: return go_rows<T, TP, 2, 1>(ctx, s, X, rows, n, ld, g, b, eps, Y, mean, rstd);
      default: return go_rows<T, TP, 4, 1>(ctx, s, X, rows, n, ld, g, b, eps, Y, mean, rstd);
    }
  }
  if (row_shape(n, ONE_VPT, 2, 256, ONE_THREADS, s))
    return s.vpt == 4 ? go_rows_one<T, TP, 4>(ctx, s, X, rows, n, ld, g, b, eps, Y, mean, rstd)
                      : go_rows_one<T, TP, 16>(ctx, s, X, rows, n, ld, g, b, eps, Y, mean, rstd);
  ZOACT_CUDA_TRY(launch_pdl(ctx, ln_long_kernel<T, TP>, dim3((unsigned)rows), dim3(LN_THREADS), 0, (const T*)X, ld, n,
                            (const TP*)g, (const TP*)b, eps, (T*)Y, mean, rstd));
  ++ctx->n_launch;
  return ZOACT_OK;
}

template <typename T, typename TP>
int run_ln_grad(Ctx* ctx, const void* dY, int64_t ld_dy, const void* X, int64_t rows, int n, int64_t ld, const void* g,
                const float* mean, const float* rstd, void* dX, float* dg, float* db) {
  constexpr int E = 16 / (int)sizeof(T);
  RowShape s;
  const bool vec = n % E == 0 && ld % E == 0 && ld_dy % E == 0 && vec16(X) && vec16(dY) && vec16(dX) && vec16(g);
  // up to 16 columns a thread: 16-bit rows to 8192, fp32 rows to 7680
  if (rows > 0 && vec && row_shape(n / E, VEC_VPT, 2, E == 8 ? 256 : RING_THREADS, RING_THREADS, s)) {
    if (s.vpt == 1) return go_ring<T, TP, 1, RING_THREADS>(ctx, s.threads, dY, ld_dy, X, rows, n, ld, g, mean, rstd, dX, dg, db);
    if (s.threads <= RING_HALF) return go_ring<T, TP, 2, RING_HALF>(ctx, s.threads, dY, ld_dy, X, rows, n, ld, g, mean, rstd, dX, dg, db);
    return s.threads <= RING_WIDE ? go_ring<T, TP, 2, RING_WIDE>(ctx, s.threads, dY, ld_dy, X, rows, n, ld, g, mean, rstd, dX, dg, db)
                                  : go_ring<T, TP, 2, RING_THREADS>(ctx, s.threads, dY, ld_dy, X, rows, n, ld, g, mean, rstd, dX, dg, db);
  }
  if constexpr (E == 4) {
    if (rows > 0 && vec && row_shape(n / E, VEC_VPT, 3, RING_HALF, RING_WIDE, s))
      return go_ring<T, TP, 4, RING_WIDE>(ctx, s.threads, dY, ld_dy, X, rows, n, ld, g, mean, rstd, dX, dg, db);
  }
  if (rows > 0 && !vec && row_shape(n, ONE_VPT, 2, 256, ONE_THREADS, s))
    return s.vpt == 4 ? go_one<T, TP, 4>(ctx, s.threads, dY, ld_dy, X, rows, n, ld, g, mean, rstd, dX, dg, db)
                      : go_one<T, TP, 16>(ctx, s.threads, dY, ld_dy, X, rows, n, ld, g, mean, rstd, dX, dg, db);
  if (dX && rows > 0) {
    if (vec && row_shape(n / E, VEC_VPT, 3, 0, GRAD_VEC_THREADS, s))
      ZOACT_CUDA_TRY(launch_pdl(ctx, ln_grad_rows_kernel<T, TP, 4>, dim3((unsigned)rows), dim3(s.threads), 0, (const T*)dY, ld_dy,
                                (const T*)X, ld, n, (const TP*)g, mean, rstd, (T*)dX));
    else
      ZOACT_CUDA_TRY(launch_pdl(ctx, ln_grad_long_kernel<T, TP>, dim3((unsigned)rows), dim3(LN_THREADS), 0, (const T*)dY, ld_dy,
                                (const T*)X, ld, n, (const TP*)g, mean, rstd, (T*)dX));
    ++ctx->n_launch;
  }
  if (!dg && !db) return ZOACT_OK;
  // ranges of at least 16 rows, as many as give an SM four blocks
  const int cols = (n + LN_THREADS - 1) / LN_THREADS;
  int64_t ranges = (4 * (int64_t)ctx->sm_count + cols - 1) / cols;
  const int64_t by_rows = (rows + 15) / 16;
  ranges = ranges < by_rows ? ranges : by_rows;
  if (ranges < 1) ranges = 1;
  const int64_t per = (rows + ranges - 1) / ranges;
  float* part;
  if (!parts_for(ctx, ranges, n, true, &part)) return ZOACT_ERR_NOMEM;
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
