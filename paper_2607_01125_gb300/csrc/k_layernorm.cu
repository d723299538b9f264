// Layer norm over the rows of X [rows, n] (row stride ld):
//     y = (x - m) s g + b,  m = mean(x),  s = 1 / sqrt(mean((x - m)^2) + eps)
// and its gradient, with u = dy g and xh = (x - m) s:
//     dx = s (u - mean(u) - xh mean(u xh)),  dg = sum_rows dy xh,  db = sum_rows dy.
#include "internal.h"

namespace zoact {
namespace {

constexpr int LN_THREADS = 256;

__device__ __forceinline__ float ln_block_sum(float v, float* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __syncthreads();
  if (lane == 0) red[warp] = v;
  __syncthreads();
  float s = 0.f;
  for (int w = 0; w < LN_THREADS / 32; ++w) s += red[w];
  return s;
}

template <typename TP>
__device__ __forceinline__ float param_at(const TP* p, int i, float none) { return p ? to_f32<TP>(p[i]) : none; }

template <typename T, typename TP>
__global__ void __launch_bounds__(LN_THREADS)
ln_kernel(const T* __restrict__ X, int64_t ld, int n, const TP* __restrict__ g, const TP* __restrict__ b, float eps,
          T* __restrict__ Y, float* __restrict__ mean, float* __restrict__ rstd) {
  pdl_wait();                              // the input rows written by the previous kernel
  pdl_trigger();
  __shared__ float red[LN_THREADS / 32];
  const int64_t row = blockIdx.x;
  const T* x = X + row * ld;
  float s = 0.f;
  for (int i = threadIdx.x; i < n; i += LN_THREADS) s += to_f32<T>(x[i]);
  const float m = ln_block_sum(s, red) / (float)n;
  float q = 0.f;
  for (int i = threadIdx.x; i < n; i += LN_THREADS) {
    const float c = to_f32<T>(x[i]) - m;
    q = fmaf(c, c, q);
  }
  const float r = 1.f / sqrtf(ln_block_sum(q, red) / (float)n + eps);
  for (int i = threadIdx.x; i < n; i += LN_THREADS)
    Y[row * n + i] = from_f32<T>(fmaf((to_f32<T>(x[i]) - m) * r, param_at(g, i, 1.f), param_at(b, i, 0.f)));
  if (threadIdx.x == 0) {
    if (mean) mean[row] = m;
    if (rstd) rstd[row] = r;
  }
}

template <typename T, typename TP>
__global__ void __launch_bounds__(LN_THREADS)
ln_grad_x_kernel(const T* __restrict__ dY, int64_t ld_dy, const T* __restrict__ X, int64_t ld, int n,
                 const TP* __restrict__ g, const float* __restrict__ mean, const float* __restrict__ rstd,
                 T* __restrict__ dX) {
  pdl_wait();
  pdl_trigger();
  __shared__ float red[LN_THREADS / 32];
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
  a = ln_block_sum(a, red) / (float)n;
  c = ln_block_sum(c, red) / (float)n;
  for (int i = threadIdx.x; i < n; i += LN_THREADS) {
    const float u = to_f32<T>(dy[i]) * param_at(g, i, 1.f), xh = (to_f32<T>(x[i]) - m) * r;
    dX[row * n + i] = from_f32<T>((u - a - xh * c) * r);
  }
}

// Column sums, one thread per column, rows in order.
template <typename T>
__global__ void __launch_bounds__(LN_THREADS)
ln_grad_p_kernel(const T* __restrict__ dY, int64_t ld_dy, const T* __restrict__ X, int64_t ld, int64_t rows, int n,
                 const float* __restrict__ mean, const float* __restrict__ rstd, float* __restrict__ dg,
                 float* __restrict__ db) {
  pdl_wait();
  pdl_trigger();
  const int i = blockIdx.x * LN_THREADS + threadIdx.x;
  if (i >= n) return;
  float sg = 0.f, sb = 0.f;
  for (int64_t row = 0; row < rows; ++row) {
    const float dy = to_f32<T>(dY[row * ld_dy + i]);
    sg = fmaf(dy, (to_f32<T>(X[row * ld + i]) - mean[row]) * rstd[row], sg);
    sb += dy;
  }
  if (dg) dg[i] = sg;
  if (db) db[i] = sb;
}

template <typename T, typename TP>
int run_ln(Ctx* ctx, const void* X, int64_t rows, int n, int64_t ld, const void* g, const void* b, float eps, void* Y,
           float* mean, float* rstd) {
  ZOACT_CUDA_TRY(launch_pdl(ctx, ln_kernel<T, TP>, dim3((unsigned)rows), dim3(LN_THREADS), 0, (const T*)X, ld, n,
                            (const TP*)g, (const TP*)b, eps, (T*)Y, mean, rstd));
  ++ctx->n_launch;
  return ZOACT_OK;
}

template <typename T, typename TP>
int run_ln_grad(Ctx* ctx, const void* dY, int64_t ld_dy, const void* X, int64_t rows, int n, int64_t ld, const void* g,
                const float* mean, const float* rstd, void* dX, float* dg, float* db) {
  if (dX && rows > 0) {
    ZOACT_CUDA_TRY(launch_pdl(ctx, ln_grad_x_kernel<T, TP>, dim3((unsigned)rows), dim3(LN_THREADS), 0, (const T*)dY, ld_dy,
                              (const T*)X, ld, n, (const TP*)g, mean, rstd, (T*)dX));
    ++ctx->n_launch;
  }
  if (dg || db) {
    ZOACT_CUDA_TRY(launch_pdl(ctx, ln_grad_p_kernel<T>, dim3((unsigned)((n + LN_THREADS - 1) / LN_THREADS)), dim3(LN_THREADS),
                              0, (const T*)dY, ld_dy, (const T*)X, ld, rows, n, mean, rstd, dg, db));
    ++ctx->n_launch;
  }
  return ZOACT_OK;
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
