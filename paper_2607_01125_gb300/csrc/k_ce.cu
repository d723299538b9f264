// Softmax cross entropy of hidden states H [rows, d] against a head W [vocab, d], without keeping the logits z = H W^T:
//     lse_t = log sum_v exp z_tv,   loss_t = lse_t - z_t,target(t),   L_b = sum_t loss_t / N  (block b's counted rows)
// and the gradient of s L by H and W.  With G = exp(z - lse) - onehot(target) on counted rows (0 on the others),
//     dH = s/N G W,   dW = s/N G^T H.
// A row whose target is negative has loss 0 and is not counted.
#include <type_traits>

#include "ce_tc.h"

namespace zoact {
namespace {

constexpr int TS = 64;              // tile of rows and of columns
constexpr int TK = 16;
constexpr int CE_THREADS = 256;     // 4 x 4 outputs a thread

enum { MODE_CE = 0, MODE_G = 1, MODE_OUT = 2 };

struct GemmArgs {
  int64_t M, N, K;
  int64_t sam, sak, sbn, sbk;       // element strides of A [M, K] and B [N, K]
  // MODE_CE
  float2* part;                     // [column tile][M]: maximum and sum of exp(z - maximum)
  float* zt;                        // [M] the target's logit
  const void* targets;
  int id64;
  int64_t T;
  // MODE_G
  const float2* stat;               // [M] the row's maximum and log sum exp(z - maximum)
  float* G;
  int64_t ldg;
  // MODE_OUT
  const float* alpha;               // device
  const float* add;                 // [M, N] or nullptr
  void* out;                        // [M, N]
};

__device__ __forceinline__ int64_t target_of(const GemmArgs& a, int64_t row, int64_t vocab) {
  const int64_t t = load_id(a.targets, a.id64, row % a.T);
  return t >= 0 && t < vocab ? t : -1;
}

// D[m, n] = sum_k A[m, k] B[n, k] in fp32, 64 x 64 a block; sums of 1024 products are added up by themselves (one chain
// over a vocabulary of 2^20 erred by 3e-4 of the terms' magnitudes).
template <int MODE, typename TA, typename TB, typename TO>
__global__ void __launch_bounds__(CE_THREADS)
ce_gemm_kernel(const TA* __restrict__ A, const TB* __restrict__ B, const GemmArgs a) {
  pdl_wait();
  pdl_trigger();
  __shared__ float sa[TK][TS + 1], sb[TK][TS + 1];
  const int64_t m0 = (int64_t)blockIdx.y * TS, n0 = (int64_t)blockIdx.x * TS;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float acc[4][4] = {}, sum[4][4] = {};
  for (int64_t k0 = 0; k0 < a.K; k0 += TK) {
    for (int e = threadIdx.x; e < TS * TK; e += CE_THREADS) {
      const bool ak = a.sak == 1, bk = a.sbk == 1;       // the contiguous index varies fastest over the threads
      const int am = ak ? e / TK : e % TS, ai = ak ? e % TK : e / TS;
      const int bn = bk ? e / TK : e % TS, bi = bk ? e % TK : e / TS;
      sa[ai][am] = m0 + am < a.M && k0 + ai < a.K ? to_f32<TA>(A[(m0 + am) * a.sam + (k0 + ai) * a.sak]) : 0.f;
      sb[bi][bn] = n0 + bn < a.N && k0 + bi < a.K ? to_f32<TB>(B[(n0 + bn) * a.sbn + (k0 + bi) * a.sbk]) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < TK; ++k) {
      float x[4], y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) { x[i] = sa[k][ty * 4 + i]; y[i] = sb[k][tx * 4 + i]; }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(x[i], y[j], acc[i][j]);
    }
    __syncthreads();
    if (k0 / TK % 64 == 63 || k0 + TK >= a.K) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) { sum[i][j] += acc[i][j]; acc[i][j] = 0.f; }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t m = m0 + ty * 4 + i;
    const bool mok = m < a.M;
    if (MODE == MODE_CE) {
      float mx = -INFINITY, s = 0.f;
      const int64_t t = mok ? target_of(a, m, a.N) : -1;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int64_t n = n0 + tx * 4 + j;
        if (n >= a.N) continue;
        mx = fmaxf(mx, sum[i][j]);
        if (n == t) a.zt[m] = sum[i][j];
      }
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (n0 + tx * 4 + j < a.N) s += expf(sum[i][j] - mx);
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      if (mok && tx == 0) a.part[(int64_t)blockIdx.x * a.M + m] = make_float2(mx, s);
    } else if (MODE == MODE_G) {
      if (!mok) continue;
      const int64_t t = target_of(a, m, a.N);
      const float2 st = a.stat[m];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int64_t n = n0 + tx * 4 + j;
        if (n < a.N) a.G[m * a.ldg + n] = t < 0 ? 0.f : n == t ? expm1f((sum[i][j] - st.x) - st.y) : expf((sum[i][j] - st.x) - st.y);
      }
    } else {
      if (!mok) continue;
      const float f = *a.alpha;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int64_t n = n0 + tx * 4 + j;
        if (n >= a.N) continue;
        const float v = sum[i][j] * f + (a.add ? a.add[m * a.N + n] : 0.f);
        reinterpret_cast<TO*>(a.out)[m * a.N + n] = from_f32<TO>(v);
      }
    }
  }
}

// The tiles' maxima m_i and sums s_i of a row joined: m, log s with s = sum s_i exp(m_i - m) (a row that the model predicts
// well has s = 1 + many terms that fp32 alone would drop one by one), lse = m + log s and loss = lse - z_t.
// The gradient takes z - lse as (z - m) - log s, exact where z = m.
// All of it in fp32 with what the additions round off beside the sum (fp64 FMAs run at 1/64 of the rate: with them this kernel
// took 24 us for 2048 rows of 1002 tiles).  A block has ROWS rows; 1024 / ROWS groups of threads take their tiles in turn,
// and a warp a row joins the groups.
struct MaxSum {
  float m, hi, lo;                         // sum of exp(z - m): hi + lo
};
__device__ __forceinline__ MaxSum join_sums(const MaxSum& a, const MaxSum& b) {
  MaxSum c;
  c.m = fmaxf(a.m, b.m);
  const float fa = a.m == c.m ? 1.f : expf(a.m - c.m), fb = b.m == c.m ? 1.f : expf(b.m - c.m);
  const float x = a.hi * fa, y = b.hi * fb;
  c.hi = x + y;
  c.lo = a.lo * fa + b.lo * fb + (x >= y ? (x - c.hi) + y : (y - c.hi) + x);      // what hi rounded off
  return c;
}

template <int ROWS>
__global__ void __launch_bounds__(1024)
ce_join_kernel(const float2* __restrict__ part, int64_t tiles, int64_t part_ld, int64_t rows, const float* __restrict__ zt,
               const void* __restrict__ targets, int id64, int64_t T, int64_t vocab, float2* __restrict__ stat,
               float* __restrict__ lse, float* __restrict__ loss, int* status) {
  pdl_wait();
  pdl_trigger();
  constexpr int GROUPS = 1024 / ROWS;
  static_assert(GROUPS % 32 == 0 && ROWS <= 32, "a warp joins a row's groups");
  __shared__ float mx[ROWS][GROUPS + 1], hi[ROWS][GROUPS + 1], lo[ROWS][GROUPS + 1];
  {
    const int r = threadIdx.x % ROWS, group = threadIdx.x / ROWS;
    const int64_t row = (int64_t)blockIdx.x * ROWS + r;
    MaxSum a = {-INFINITY, 0.f, 0.f};
    if (row < rows) {
#pragma unroll 8
      for (int64_t i = group; i < tiles; i += GROUPS) {
        const float2 p = part[i * part_ld + row];
        a = join_sums(a, MaxSum{p.x, p.y, 0.f});
      }
    }
    mx[r][group] = a.m;
    hi[r][group] = a.hi;
    lo[r][group] = a.lo;
  }
  __syncthreads();
  const int r = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * ROWS + r;
  if (r >= ROWS || row >= rows) return;
  MaxSum a = {mx[r][lane], hi[r][lane], lo[r][lane]};
#pragma unroll
  for (int g = 32; g < GROUPS; g += 32) a = join_sums(a, MaxSum{mx[r][lane + g], hi[r][lane + g], lo[r][lane + g]});
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const MaxSum b = {__shfl_xor_sync(0xffffffffu, a.m, o), __shfl_xor_sync(0xffffffffu, a.hi, o),
                      __shfl_xor_sync(0xffffffffu, a.lo, o)};
    a = (lane & o) ? join_sums(b, a) : join_sums(a, b);              // one order for both
  }
  if (lane != 0) return;
  const float ls = logf(a.hi) + a.lo / a.hi;
  const float l = a.m + ls;
  stat[row] = make_float2(a.m, ls);
  lse[row] = l;
  const int64_t t = load_id(targets, id64, row % T);
  if (t >= vocab) record_error(status, ZOACT_ERR_INVALID_ARG);
  loss[row] = t >= 0 && t < vocab ? l - zt[row] : 0.f;
}

// alpha = scale / N, N the number of counted rows (at least 1): the factor of the gradient's products.
__global__ void __launch_bounds__(1024)
ce_alpha_kernel(const void* __restrict__ targets, int id64, int64_t T, int64_t vocab, float scale, float* alpha) {
  pdl_wait();
  pdl_trigger();
  __shared__ int red[32];
  int n = 0;
  for (int64_t t = threadIdx.x; t < T; t += 1024) {
    const int64_t id = load_id(targets, id64, t);
    n += id >= 0 && id < vocab;
  }
  n = __reduce_add_sync(0xffffffffu, n);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = n;
  __syncthreads();
  if (threadIdx.x < 32) {
    n = __reduce_add_sync(0xffffffffu, red[threadIdx.x]);
    if (threadIdx.x == 0) *alpha = (float)((double)scale / (double)(n > 1 ? n : 1));
  }
}

// What a chunk of rows kept of its logits, 4096 (m_tile - z) in 16 bits, to G = exp(z - lse) - onehot in the operands' type,
// in place.  The fixed point errs by 1.2e-4 of the exponential at most, a third of fp16's rounding (exp(z - m_tile) in fp16
// would have rounded twice; beyond 16 below the tile's largest nothing is kept).  fp16's G is scaled by 2^15 (undone in
// the products' scale): 1 / vocab would lie among its subnormals.  The target's element is expm1(z_t - lse): p - 1 from a
// rounded p would lose what is left of it where the model is nearly right.
constexpr float G_SCALE_FP16 = 32768.f;

__device__ __forceinline__ float exp2_ftz(float x) {
  float e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x));
  return e;
}

// Thread: 8 entries of SCALE_ROWS rows, loaded together; block: 32 SCALE_ROWS rows of one block of 64 entries (blockIdx.x
// their group, blockIdx.y the block).
constexpr int SCALE_ROWS = 4;

template <typename T>
__global__ void __launch_bounds__(CE_THREADS)
ce_scale_kernel(void* __restrict__ G, int64_t blk0, int64_t rows, const float2* __restrict__ part, int64_t part_ld,
                const float2* __restrict__ stat, const float* __restrict__ zt, const void* __restrict__ targets, int id64,
                int64_t vocab) {
  pdl_wait();
  pdl_trigger();
  constexpr float scale = std::is_same<T, __half>::value ? G_SCALE_FP16 : 1.f;
  const int64_t blk = blk0 + blockIdx.y, v0 = blk * 64 + threadIdx.x % 8 * 8;
  const int64_t row0 = (int64_t)blockIdx.x * (32 * SCALE_ROWS) + threadIdx.x / 8;
  uint4* g = reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(G) + (blk * rows + row0) * 64 + threadIdx.x % 8 * 8);
  constexpr int STEP = 32 * 64 / 8;        // from a row to the thread's next one, in vectors
  uint4 q[SCALE_ROWS];
  int64_t t[SCALE_ROWS];
  float c[SCALE_ROWS];
#pragma unroll
  for (int k = 0; k < SCALE_ROWS; ++k) {
    const int64_t row = row0 + 32 * k;
    t[k] = -1;
    if (row < rows) {
      t[k] = load_id(targets, id64, row);
      q[k] = g[k * STEP];
      const float2 st = __ldg(stat + row);
      c[k] = (__ldg(&part[blk / (ce::V_TILE / 64) * part_ld + row].x) - st.x) - st.y;
    }
  }
#pragma unroll
  for (int k = 0; k < SCALE_ROWS; ++k) {
    const int64_t row = row0 + 32 * k;
    if (row >= rows) return;
    if (t[k] >= 0 && t[k] < vocab) {
      uint32_t* w = reinterpret_cast<uint32_t*>(&q[k]);
      const float none = c[k] == c[k] ? 0.f : c[k];      // a row that is not finite stays so
      const float c2 = c[k] * 1.44269504f;
      float e[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        // 2^23 + the fixed point, by its bytes: the conversion instruction shares the exponential's unit
        const uint32_t bits = __byte_perm(w[i / 2], 0x4b000000u, i & 1 ? 0x7632 : 0x7610);
        const float x = __uint_as_float(bits) - 8388608.f;
        e[i] = bits == 0x4b00ffffu ? none : exp2_ftz(fmaf(x, -1.44269504f / 4096.f, c2)) * scale;
      }
      if (t[k] >= v0 && t[k] < v0 + 8) {
        const float2 st = stat[row];
        const float g_t = expm1f((zt[row] - st.x) - st.y) * scale;
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = t[k] == v0 + i ? g_t : e[i];
      }
      if (v0 + 8 > vocab) {                              // the last block's rest
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = v0 + i < vocab ? e[i] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        T o[2] = {from_f32<T>(e[2 * i]), from_f32<T>(e[2 * i + 1])};
        w[i] = *reinterpret_cast<const uint32_t*>(o);
      }
    } else {
      q[k] = make_uint4(0, 0, 0, 0);
    }
    g[k * STEP] = q[k];
  }
}

// Block b: L_b = sum / N and D_b = sum over t of (loss_b - loss_0) / N, in fp64 and in a fixed order.
//   mean [nb] (or nullptr); est: 1 = the pair's {L+, L-, D, a}, 2 = {L_0 .. L_q, a_1 .. a_q}, 0 = none.
__global__ void __launch_bounds__(1024)
ce_finish_kernel(const float* __restrict__ loss, int64_t T, int nb, const void* __restrict__ targets, int id64,
                 int64_t vocab, double* mean, int est, double step, double* out, int* status) {
  pdl_wait();
  pdl_trigger();
  __shared__ double red[3][32];
  const int b = blockIdx.x;
  const int other = est == 1 ? 1 : 0;       // the pair's D is L+ - L-, the others' L_b - L_0
  double s = 0.0, dd = 0.0, n = 0.0;
  for (int64_t t = threadIdx.x; t < T; t += 1024) {
    const int64_t id = load_id(targets, id64, t);
    if (id < 0 || id >= vocab) continue;
    const double l = loss[b * T + t];
    n += 1.0;
    s += l;
    if (est) dd += l - (double)loss[other * T + t];
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    s += __shfl_xor_sync(0xffffffffu, s, o);
    dd += __shfl_xor_sync(0xffffffffu, dd, o);
    n += __shfl_xor_sync(0xffffffffu, n, o);
  }
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (lane == 0) { red[0][warp] = s; red[1][warp] = dd; red[2][warp] = n; }
  __syncthreads();
  if (threadIdx.x != 0) return;
  s = dd = n = 0.0;
  for (int w = 0; w < 32; ++w) { s += red[0][w]; dd += red[1][w]; n += red[2][w]; }
  const double den = n > 0.0 ? n : 1.0;
  const double L = s / den, D = dd / den;
  if (mean) mean[b] = L;
  bool fine = isfinite(L);
  if (est == 1) {
    out[b] = L;
    if (b == 0) {
      const double e = D / (2.0 * step);
      out[2] = D;
      out[3] = e;
      fine = fine && isfinite(e);
    }
  } else if (est == 2) {
    out[b] = L;
    if (b > 0) {
      const double e = D / step;
      out[nb + b - 1] = e;
      fine = fine && isfinite(e);
    }
  }
  if (!fine) record_error(status, ZOACT_ERR_NONFINITE);
}

struct CeScratch {
  float* alpha;
  float *zt, *lse, *loss;
  float2 *stat, *part;
  int64_t part_ld;
};

// part_rows: rows whose statistics are held at a time.
bool ce_scratch(Ctx* ctx, int64_t rows, int64_t part_rows, int64_t tiles, CeScratch& s) {
  const size_t r = (size_t)((rows + 3) / 4 * 4);
  char* p = (char*)scratch(ctx, SLOT_CE, 256 + r * 4 * 5 + (size_t)tiles * part_rows * sizeof(float2));
  if (!p) return false;
  s.alpha = (float*)p;
  s.zt = (float*)(p + 256);
  s.lse = s.zt + r;
  s.loss = s.lse + r;
  s.stat = (float2*)(s.loss + r);
  s.part = s.stat + r;
  s.part_ld = part_rows;
  return true;
}

template <int MODE, typename TA, typename TB, typename TO>
int gemm(Ctx* ctx, const void* A, const void* B, const GemmArgs& a) {
  const dim3 grid((unsigned)((a.N + TS - 1) / TS), (unsigned)((a.M + TS - 1) / TS));
  ZOACT_CUDA_TRY(launch_pdl(ctx, ce_gemm_kernel<MODE, TA, TB, TO>, grid, dim3(CE_THREADS), 0, (const TA*)A, (const TB*)B, a));
  ++ctx->n_launch;
  return ZOACT_OK;
}

// Join rows [r0, r0 + n), whose statistics lie at the beginning of s.part.
int join(Ctx* ctx, const CeArgs& c, const CeScratch& s, int64_t tiles, int64_t r0, int64_t n, float* lse, float* loss) {
  // with several blocks the rows are all there; a chunk of rows (one block) takes its own targets
  const void* targets = (const char*)c.targets + r0 * (c.id64 ? 8 : 4);
  constexpr int ROWS = 8;
  ZOACT_CUDA_TRY(launch_pdl(ctx, ce_join_kernel<ROWS>, dim3((unsigned)((n + ROWS - 1) / ROWS)), dim3(1024), 0,
                            (const float2*)s.part, tiles, s.part_ld, n, (const float*)s.zt + r0, targets, c.id64, c.T, c.vocab, s.stat + r0, lse + r0,
                            loss + r0, ctx->d_status));
  ++ctx->n_launch;
  return ZOACT_OK;
}

int make_alpha(Ctx* ctx, const CeArgs& c, const CeScratch& s, float scale) {
  ZOACT_CUDA_TRY(launch_pdl(ctx, ce_alpha_kernel, dim3(1), dim3(1024), 0, c.targets, c.id64, c.T, c.vocab, scale, s.alpha));
  ++ctx->n_launch;
  return ZOACT_OK;
}

template <typename T>
int run_forward(Ctx* ctx, const CeArgs& c, const CeScratch& s, int64_t tiles, float* lse, float* loss) {
  GemmArgs a = {};
  a.M = c.rows; a.N = c.vocab; a.K = c.d;
  a.sam = c.d; a.sak = 1; a.sbn = c.d; a.sbk = 1;
  a.part = s.part; a.zt = s.zt; a.targets = c.targets; a.id64 = c.id64; a.T = c.T;
  const int st = gemm<MODE_CE, T, T, T>(ctx, c.H, c.W, a);
  if (st) return st;
  return join(ctx, c, s, tiles, 0, c.rows, lse, loss);
}

template <typename T, typename TG>
int run_backward(Ctx* ctx, const CeArgs& c, const CeScratch& s, void* dH, void* dW,
                 int accumulate) {
  const size_t most = (size_t)1 << 31;
  int64_t chunk = (int64_t)(most / ((size_t)c.vocab * 4)) / TS * TS;
  if (chunk < TS) chunk = TS;
  if (chunk > c.rows) chunk = c.rows;
  float* G = (float*)scratch(ctx, SLOT_CE_G, (size_t)chunk * c.vocab * 4);
  if (!G) return ZOACT_ERR_NOMEM;
  float* dWf = nullptr;             // fp32 sums of several chunks of rows
  if (dW && sizeof(TG) != 4 && chunk < c.rows) {
    dWf = (float*)scratch(ctx, SLOT_CE_DW, (size_t)c.vocab * c.d * 4);
    if (!dWf) return ZOACT_ERR_NOMEM;
  }
  for (int64_t r0 = 0; r0 < c.rows; r0 += chunk) {
    const int64_t n = c.rows - r0 < chunk ? c.rows - r0 : chunk;
    const T* H = (const T*)c.H + r0 * c.d;
    GemmArgs a = {};
    a.M = n; a.N = c.vocab; a.K = c.d;
    a.sam = c.d; a.sak = 1; a.sbn = c.d; a.sbk = 1;
    a.targets = (const char*)c.targets + r0 * (c.id64 ? 8 : 4); a.id64 = c.id64; a.T = c.T;
    a.stat = s.stat + r0; a.G = G; a.ldg = c.vocab;
    int st = gemm<MODE_G, T, T, T>(ctx, H, c.W, a);
    if (st) return st;
    a.alpha = s.alpha;
    if (dH) {
      a.M = n; a.N = c.d; a.K = c.vocab;
      a.sam = c.vocab; a.sak = 1; a.sbn = 1; a.sbk = c.d;
      a.out = (T*)dH + r0 * c.d; a.add = nullptr;
      st = gemm<MODE_OUT, float, T, T>(ctx, G, c.W, a);
      if (st) return st;
    }
    if (dW) {
      a.M = c.vocab; a.N = c.d; a.K = n;
      a.sam = 1; a.sak = c.vocab; a.sbn = 1; a.sbk = c.d;
      const bool last = r0 + n == c.rows;
      if (dWf) {
        a.add = r0 ? dWf : nullptr;
        a.out = last ? dW : dWf;
      } else {
        a.out = dW;
        a.add = r0 || accumulate ? (const float*)dW : nullptr;   // several chunks or accumulate: dW is fp32
      }
      st = dWf && !last ? gemm<MODE_OUT, float, T, float>(ctx, G, H, a) : gemm<MODE_OUT, float, T, TG>(ctx, G, H, a);
      if (st) return st;
    }
  }
  return ZOACT_OK;
}

// The losses' means and estimates.
int finish(Ctx* ctx, const CeArgs& c, const float* loss) {
  if (!c.mean && !c.est) return ZOACT_OK;
  ZOACT_CUDA_TRY(launch_pdl(ctx, ce_finish_kernel, dim3((unsigned)c.nb), dim3(1024), 0, loss, c.T, c.nb, c.targets, c.id64,
                            c.vocab, c.mean, c.est, (double)c.step, c.out, ctx->d_status));
  ++ctx->n_launch;
  return ZOACT_OK;
}

template <typename T>
__global__ void __launch_bounds__(CE_THREADS) ce_round_kernel(const float4* __restrict__ x, int64_t n4, T* __restrict__ y) {
  pdl_wait();
  pdl_trigger();
  for (int64_t i = (int64_t)blockIdx.x * CE_THREADS + threadIdx.x; i < n4; i += (int64_t)gridDim.x * CE_THREADS) {
    const float4 v = x[i];
    T o[4] = {from_f32<T>(v.x), from_f32<T>(v.y), from_f32<T>(v.z), from_f32<T>(v.w)};
    *reinterpret_cast<uint2*>(y + 4 * i) = *reinterpret_cast<const uint2*>(o);
  }
}

// 16-bit operands: the products on the tensor cores.  Where the gradient is asked for, chunk by chunk of rows: logits, whose
// exponentials are kept in 16 bits, the rows' sums, G in place, and its two products.
template <typename T>
int run_tc(Ctx* ctx, const CeArgs& c) {
  using ce::Operand;
  const int64_t tiles = (c.vocab + ce::V_TILE - 1) / ce::V_TILE, blocks = (c.vocab + 63) / 64;
  const bool grad = c.dH || c.dW;
  int64_t chunk = c.rows;
  if (grad) {
    chunk = (int64_t)(((size_t)1 << 31) / ((size_t)blocks * 128)) / 256 * 256;
    if (chunk < 256) chunk = 256;
    if (chunk > c.rows) chunk = c.rows;
  }
  CeScratch s;
  if (!ce_scratch(ctx, c.rows, chunk, tiles, s)) return ZOACT_ERR_NOMEM;
  float* lse = c.lse ? c.lse : s.lse;
  float* loss = c.loss ? c.loss : s.loss;
  const Operand W = {c.W, c.dtype, c.vocab, c.d, c.d, 1, c.vocab * c.d};
  int st;
  if (!grad) {
    const Operand H = {c.H, c.dtype, c.rows, c.d, c.d, 1, c.rows * c.d};
    st = ce::launch_logits(ctx, W, H, s.part, s.part_ld, s.zt, c.targets, c.id64, c.T, ce::KEEP_NONE, ce::Blocks{});
    if (!st) st = join(ctx, c, s, tiles, 0, c.rows, lse, loss);
    return st ? st : finish(ctx, c, loss);
  }
  void* G = scratch(ctx, SLOT_CE_G, (size_t)chunk * blocks * 128);
  if (!G) return ZOACT_ERR_NOMEM;
  // several chunks add to dW in fp32: a 16-bit dW is rounded from the whole sum
  const bool parts = chunk < c.rows;
  float* dWf = nullptr;
  if (c.dW && parts && c.wgdtype != ZOACT_DT_FP32) {
    dWf = (float*)scratch(ctx, SLOT_CE_DW, (size_t)c.vocab * c.d * 4);
    if (!dWf) return ZOACT_ERR_NOMEM;
  }
  st = make_alpha(ctx, c, s, c.dtype == ZOACT_DT_FP16 ? c.grad_scale / G_SCALE_FP16 : c.grad_scale);
  if (st) return st;
  for (int64_t r0 = 0; r0 < c.rows; r0 += chunk) {
    const int64_t n = c.rows - r0 < chunk ? c.rows - r0 : chunk;
    const Operand H = {(const T*)c.H + r0 * c.d, c.dtype, n, c.d, c.d, 1, n * c.d};
    const ce::Blocks Gm = {G, c.dtype, n, c.vocab, 1};
    const void* targets = (const char*)c.targets + r0 * (c.id64 ? 8 : 4);
    st = ce::launch_logits(ctx, W, H, s.part, s.part_ld, s.zt + r0, targets, c.id64, c.T, ce::KEEP_LOG, Gm);
    if (!st) st = join(ctx, c, s, tiles, r0, n, lse, loss);
    if (st) return st;
    const int64_t row_groups = (n + 32 * SCALE_ROWS - 1) / (32 * SCALE_ROWS);
    for (int64_t b = 0; b < blocks; b += 65535) {
      const int64_t nb = blocks - b < 65535 ? blocks - b : 65535;
      ZOACT_CUDA_TRY(launch_pdl(ctx, ce_scale_kernel<T>, dim3((unsigned)row_groups, (unsigned)nb), dim3(CE_THREADS), 0, G, b, n,
                                (const float2*)s.part, s.part_ld, (const float2*)s.stat + r0, (const float*)s.zt + r0, targets,
                                c.id64, c.vocab));
      ++ctx->n_launch;
    }
    if (c.dH) st = ce::launch_by_h(ctx, W, Gm, s.alpha, (T*)c.dH + r0 * c.d, c.dtype);
    if (!st && c.dW)
      st = ce::launch_by_w(ctx, Gm, H, s.alpha, dWf ? (void*)dWf : c.dW, dWf ? ZOACT_DT_FP32 : c.wgdtype,
                           r0 > 0 || c.accumulate);
    if (st) return st;
  }
  if (dWf) {
    const int64_t total = c.vocab * c.d / 4;        // d is a multiple of 8
    const int64_t blocks = (total + CE_THREADS - 1) / CE_THREADS;
    ZOACT_CUDA_TRY(launch_pdl(ctx, ce_round_kernel<T>, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(CE_THREADS), 0,
                              (const float4*)dWf, total, (T*)c.dW));
    ++ctx->n_launch;
  }
  return finish(ctx, c, loss);
}

// fp32 operands.
int run_fp32(Ctx* ctx, const CeArgs& c) {
  const int64_t tiles = (c.vocab + TS - 1) / TS;
  CeScratch s;
  if (!ce_scratch(ctx, c.rows, c.rows, tiles, s)) return ZOACT_ERR_NOMEM;
  float* lse = c.lse ? c.lse : s.lse;
  float* loss = c.loss ? c.loss : s.loss;
  int st = run_forward<float>(ctx, c, s, tiles, lse, loss);
  if (!st) st = finish(ctx, c, loss);
  if (st || (!c.dH && !c.dW)) return st;
  st = make_alpha(ctx, c, s, c.grad_scale);
  return st ? st : run_backward<float, float>(ctx, c, s, c.dH, c.dW, c.accumulate);
}

}  // namespace

int launch_ce(Ctx* ctx, const CeArgs& c) {
  if (c.rows == 0) {                       // no token: losses of 0, no gradient
    if (c.dW && !c.accumulate)
      ZOACT_CUDA_TRY(cudaMemsetAsync(c.dW, 0, (size_t)c.vocab * c.d * dtype_size(c.wgdtype), ctx->stream));
    return finish(ctx, c, nullptr);
  }
  switch (c.dtype) {
    case ZOACT_DT_FP32: return run_fp32(ctx, c);
    case ZOACT_DT_BF16: return run_tc<__nv_bfloat16>(ctx, c);
    default: return run_tc<__half>(ctx, c);
  }
}

}  // namespace zoact
