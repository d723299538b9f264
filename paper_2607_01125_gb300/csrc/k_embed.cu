// The embedding at the input of a language model: scaled rows of a table by
// token id, and the table's gradient.  A negative id is a token without a row
// (padding): its output is zero and it adds nothing to the gradient.
#include "internal.h"

namespace zoact {
namespace {

constexpr int EMB_THREADS = 256;

template <typename T>
__global__ void __launch_bounds__(EMB_THREADS)
embed_kernel(const T* __restrict__ E, const void* __restrict__ ids, int id64, int64_t vocab, int d, float scale,
             T* __restrict__ Y, int* status) {
  pdl_wait();                              // ids and table as earlier kernels left them
  pdl_trigger();
  const int64_t t = blockIdx.x;
  const int64_t id = load_id(ids, id64, t);
  const bool ok = id >= 0 && id < vocab;
  if (id >= vocab && threadIdx.x == 0) record_error(status, ZOACT_ERR_INVALID_ARG);
  const T* e = E + (ok ? id : 0) * d;
  for (int i = threadIdx.x; i < d; i += EMB_THREADS)
    Y[t * d + i] = from_f32<T>(ok ? to_f32<T>(e[i]) * scale : 0.f);
}

// One block per table row: the ids are searched in token order, so the sum's order is fixed.
template <typename T, typename TE>
__global__ void __launch_bounds__(EMB_THREADS)
embed_grad_kernel(const T* __restrict__ dY, int64_t n_tok, int d, const void* __restrict__ ids, int id64, int64_t vocab,
                  float scale, TE* __restrict__ dE, int accumulate, int* status) {
  pdl_wait();
  pdl_trigger();
  __shared__ int hit[EMB_THREADS];
  const int64_t v = blockIdx.x;
  bool any = false;
  for (int c0 = 0; c0 < d; c0 += EMB_THREADS) {
    const int c = c0 + threadIdx.x;
    float sum = 0.f;
    for (int64_t t0 = 0; t0 < n_tok; t0 += EMB_THREADS) {
      const int64_t t = t0 + threadIdx.x;
      const int64_t id = t < n_tok ? load_id(ids, id64, t) : -1;
      if (id >= vocab && v == 0) record_error(status, ZOACT_ERR_INVALID_ARG);
      hit[threadIdx.x] = id == v;
      if (__syncthreads_or(id == v)) {
        any = true;
        for (int k = 0; k < EMB_THREADS; ++k)
          if (hit[k] && c < d) sum += to_f32<T>(dY[(t0 + k) * d + c]);
      }
      __syncthreads();
    }
    if (c < d && (any || !accumulate)) {
      const float old = accumulate ? to_f32<TE>(dE[v * d + c]) : 0.f;
      dE[v * d + c] = from_f32<TE>(fmaf(scale, sum, old));
    }
  }
}

template <typename T>
int run_embed(Ctx* ctx, const void* E, int64_t vocab, int d, const void* ids, int id64, int64_t n, float scale, void* Y) {
  ZOACT_CUDA_TRY(launch_pdl(ctx, embed_kernel<T>, dim3((unsigned)n), dim3(EMB_THREADS), 0, (const T*)E, ids, id64, vocab,
                            d, scale, (T*)Y, ctx->d_status));
  ++ctx->n_launch;
  return ZOACT_OK;
}

template <typename T, typename TE>
int run_embed_grad(Ctx* ctx, const void* dY, int64_t n, int d, const void* ids, int id64, int64_t vocab, float scale,
                   void* dE, int accumulate) {
  ZOACT_CUDA_TRY(launch_pdl(ctx, embed_grad_kernel<T, TE>, dim3((unsigned)vocab), dim3(EMB_THREADS), 0, (const T*)dY, n, d,
                            ids, id64, vocab, scale, (TE*)dE, accumulate, ctx->d_status));
  ++ctx->n_launch;
  return ZOACT_OK;
}

}  // namespace

int launch_embed(Ctx* ctx, const void* E, int dtype, int64_t vocab, int d, const void* ids, int id64, int64_t n,
                 float scale, void* Y) {
  if (n == 0) return ZOACT_OK;
  switch (dtype) {
    case ZOACT_DT_FP32: return run_embed<float>(ctx, E, vocab, d, ids, id64, n, scale, Y);
    case ZOACT_DT_BF16: return run_embed<__nv_bfloat16>(ctx, E, vocab, d, ids, id64, n, scale, Y);
    default: return run_embed<__half>(ctx, E, vocab, d, ids, id64, n, scale, Y);
  }
}

int launch_embed_grad(Ctx* ctx, const void* dY, int dtype, int64_t n, int d, const void* ids, int id64, int64_t vocab,
                      float scale, void* dE, int edtype, int accumulate) {
  if (n == 0 && accumulate) return ZOACT_OK;
  const bool f32 = edtype == ZOACT_DT_FP32;
  switch (dtype) {
    case ZOACT_DT_FP32: return run_embed_grad<float, float>(ctx, dY, n, d, ids, id64, vocab, scale, dE, accumulate);
    case ZOACT_DT_BF16:
      return f32 ? run_embed_grad<__nv_bfloat16, float>(ctx, dY, n, d, ids, id64, vocab, scale, dE, accumulate)
                 : run_embed_grad<__nv_bfloat16, __nv_bfloat16>(ctx, dY, n, d, ids, id64, vocab, scale, dE, accumulate);
    default:
      return f32 ? run_embed_grad<__half, float>(ctx, dY, n, d, ids, id64, vocab, scale, dE, accumulate)
                 : run_embed_grad<__half, __half>(ctx, dY, n, d, ids, id64, vocab, scale, dE, accumulate);
  }
}

}  // namespace zoact
