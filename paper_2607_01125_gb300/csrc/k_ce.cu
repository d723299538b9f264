// Softmax cross entropy of hidden states H [rows, d] against a head W [vocab, d], without keeping the logits z = H W^T:
//     lse_t = log sum_v exp z_tv,   loss_t = lse_t - z_t,target(t),   L_b = sum_t loss_t / N  (block b's counted rows)
// and the gradient of s L by H and W.  With G = exp(z - lse) - onehot(target) on counted rows (0 on the others),
//     dH = s/N G W,   dW = s/N G^T H.
// A row whose target is negative has loss 0 and is not counted.
#include <type_traits>

#include "ce_tc.h"

namespace zoact {
namespace {

constexpr int CE_THREADS = 256;

// The tiles' maxima m_i and sums s_i of a row, which are without its target, and the target's logit z_t (as one more of them, with
// a sum of 1) joined: m, log s with s = sum s_i exp(m_i - m), lse = m + log s and loss = (m - z_t) + log s.  A row that the
// model predicts well has s = 1 + many terms that fp32 alone would drop one by one: these are summed first.
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
    constexpr int AHEAD = 8;               // tiles loaded together
    for (int64_t i0 = group; i0 < tiles && row < rows; i0 += AHEAD * GROUPS) {
      float2 p[AHEAD];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        const int64_t i = i0 + k * GROUPS;
        p[k] = i < tiles ? part[i * part_ld + row] : make_float2(-INFINITY, 0.f);
      }
      float m = a.m;
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) m = fmaxf(m, p[k].x);
      const float f = a.m == m ? 1.f : expf(a.m - m);
      a.m = m;
      a.hi *= f;
      a.lo *= f;
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        const float y = p[k].x == m ? p[k].y : p[k].y * expf(p[k].x - m);
        const float t = a.hi + y, b = t - a.hi;
        a.lo += (a.hi - (t - b)) + (y - b);                          // what t rounded off
        a.hi = t;
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
  const int64_t t = load_id(targets, id64, row % T);
  if (t >= vocab) record_error(status, ZOACT_ERR_INVALID_ARG);
  const bool counted = t >= 0 && t < vocab;
  const float z = counted ? zt[row] : 0.f;
  if (counted) a = join_sums(a, MaxSum{z, 1.f, 0.f});
  const float ls = logf(a.hi) + a.lo / a.hi;
  stat[row] = make_float2(a.m, ls);
  lse[row] = a.m + ls;
  loss[row] = counted ? (a.m - z) + ls : 0.f;      // not lse - z: lse's rounding would stay in a small loss
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

// What a chunk of rows kept of its logits, 2048 (m_tile - z) in 16 bits, to G = exp(z - lse) - onehot in the operands' type,
// in place.  The fixed point errs by 2.4e-4 of the exponential at most, half of fp16's rounding (exp(z - m_tile) in fp16 would
// have rounded twice).  It reaches 32 below the largest of the tile's entries other than the target.  fp16's G is scaled by 2^15
// (undone in the products' scale): 1 / vocab would lie among its subnormals.  The target's element is expm1(z_t - lse): p - 1
// from a rounded p would lose what is left of it where the model is nearly right.
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
        e[i] = bits == 0x4b00ffffu ? none : exp2_ftz(fmaf(x, -1.44269504f / ce::LOG_STEPS, c2)) * scale;
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

// Block b: L_b = sum / N and D_b = sum over t of (loss_b - loss_0) / N, in a fixed order: pairs of fp32 whose additions keep what
// they round off (about 48 bits), since fp64's run at 1/64 of the rate (64 rows took 11.4 us with them), and fp64 from the
// block's sums on.
//   mean [nb] (or nullptr); est: 1 = the pair's {L+, L-, D, a}, 2 = {L_0 .. L_q, a_1 .. a_q}, 0 = none.
constexpr int FINISH_THREADS = 512;

struct Twofold {
  float hi = 0.f, lo = 0.f;
  __device__ __forceinline__ void add(float h, float l) {
    const float s = hi + h, b = s - hi, e = (hi - (s - b)) + (h - b) + (lo + l);
    hi = isfinite(s) ? s + e : s;
    lo = isfinite(s) ? s - hi + e : 0.f;
  }
  __device__ __forceinline__ double value() const { return (double)hi + (double)lo; }
};

__global__ void __launch_bounds__(FINISH_THREADS)
ce_finish_kernel(const float* __restrict__ loss, int64_t T, int nb, const void* __restrict__ targets, int id64,
                 int64_t vocab, double* mean, int est, double step, double* out, int* status) {
  pdl_wait();
  pdl_trigger();
  constexpr int WARPS = FINISH_THREADS / 32, AHEAD = 4;
  __shared__ Twofold red[2][WARPS];
  __shared__ int count[WARPS];
  const int b = blockIdx.x;
  const int other = est == 1 ? 1 : 0;       // the pair's D is L+ - L-, the others' L_b - L_0
  Twofold s, dd;
  int n = 0;
  for (int64_t t0 = threadIdx.x; t0 < T; t0 += AHEAD * FINISH_THREADS) {
    int64_t id[AHEAD];
    float l[AHEAD], o[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int64_t t = t0 + k * FINISH_THREADS;
      id[k] = -1;
      if (t < T) {
        id[k] = load_id(targets, id64, t);
        l[k] = loss[b * T + t];
        if (est) o[k] = loss[other * T + t];
      }
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (id[k] < 0 || id[k] >= vocab) continue;
      ++n;
      s.add(l[k], 0.f);
      if (est) {
        const float d = l[k] - o[k], c = d - l[k];
        dd.add(d, (l[k] - (d - c)) - (o[k] + c));                    // the difference's own rounding
      }
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    s.add(__shfl_xor_sync(0xffffffffu, s.hi, o), __shfl_xor_sync(0xffffffffu, s.lo, o));
    if (est) dd.add(__shfl_xor_sync(0xffffffffu, dd.hi, o), __shfl_xor_sync(0xffffffffu, dd.lo, o));
  }
  n = __reduce_add_sync(0xffffffffu, n);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (lane == 0) { red[0][warp] = s; red[1][warp] = dd; count[warp] = n; }
  __syncthreads();
  if (threadIdx.x >= 2) return;             // thread 0: the mean; 1: the difference and the estimate
  Twofold sum;
  int64_t all = 0;
#pragma unroll
  for (int w = 0; w < WARPS; ++w) {
    sum.add(red[threadIdx.x][w].hi, red[threadIdx.x][w].lo);
    all += count[w];
  }
  const double v = sum.value() / (double)(all > 0 ? all : 1);
  bool fine = isfinite(v);
  if (threadIdx.x == 0) {
    if (mean) mean[b] = v;
    if (est) out[b] = v;
  } else if (est == 1) {
    if (b == 0) {
      const double e = v / (2.0 * step);
      out[2] = v;
      out[3] = e;
      fine = fine && isfinite(e);
    }
  } else if (est == 2 && b > 0) {
    const double e = v / step;
    out[nb + b - 1] = e;
    fine = fine && isfinite(e);
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

// The losses' means and estimates.
int finish(Ctx* ctx, const CeArgs& c, const float* loss) {
  if (!c.mean && !c.est) return ZOACT_OK;
  ZOACT_CUDA_TRY(launch_pdl(ctx, ce_finish_kernel, dim3((unsigned)c.nb), dim3(FINISH_THREADS), 0, loss, c.T, c.nb, c.targets, c.id64,
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

// What a finite x has beyond the bf16 range, taken off it: the largest value of bf16, 3.3895e38, is the first part of what lies
// above it (rounded to the nearest, the part would be infinite).  0 for all others; an infinity stays one.
__device__ __forceinline__ float take_excess(float& x) {
  constexpr float MOST = 3.38953139e38f;
  const float all = x;
  if (fabsf(x) > MOST && fabsf(x) < INFINITY) x = copysignf(MOST, x);
  return all - x;
}

// fp32 operands in three bf16 parts: rows of W and then of H [., d] to [3][rows][ld] each, ld = d rounded up to 8 (what lies
// past d is not read).  Four elements a thread.
__global__ void __launch_bounds__(CE_THREADS)
ce_split_kernel(const float* __restrict__ W, int64_t w_rows, uint16_t* __restrict__ W3, const float* __restrict__ H,
                int64_t h_rows, uint16_t* __restrict__ H3, int d, int ld) {
  pdl_wait();
  pdl_trigger();
  const int c4 = d / 4;
  const int64_t total = (w_rows + h_rows) * c4;
  for (int64_t i = (int64_t)blockIdx.x * CE_THREADS + threadIdx.x; i < total; i += (int64_t)gridDim.x * CE_THREADS) {
    int64_t row = i / c4;
    const int c = (int)(i - row * c4) * 4;
    const bool of_w = row < w_rows;
    if (!of_w) row -= w_rows;
    float4 v = *reinterpret_cast<const float4*>((of_w ? W : H) + row * d + c);
    uint16_t* o = (of_w ? W3 : H3) + row * ld + c;
    const int64_t part = (of_w ? w_rows : h_rows) * ld;
    const float4 more = make_float4(take_excess(v.x), take_excess(v.y), take_excess(v.z), take_excess(v.w));
#pragma unroll
    for (int p = 0; p < 3; ++p) {
      if (p == 1) v = make_float4(v.x + more.x, v.y + more.y, v.z + more.z, v.w + more.w);
      const uint32_t lo = next_part_bf16x2(v.x, v.y), hi = next_part_bf16x2(v.z, v.w);
      *reinterpret_cast<uint2*>(o + p * part) = make_uint2(lo, hi);
    }
  }
}

// fp32: the kept logits of a chunk of rows, [blocks][rows][64], to G = exp(z - lse) - onehot in three bf16 parts of the same
// layout.  Thread: 4 entries of a row.
__global__ void __launch_bounds__(CE_THREADS)
ce_split_g_kernel(const float* __restrict__ Z, uint16_t* __restrict__ G, int64_t blocks, int64_t rows,
                  const float2* __restrict__ stat, const float* __restrict__ zt, const void* __restrict__ targets, int id64,
                  int64_t vocab) {
  pdl_wait();
  pdl_trigger();
  const int64_t n4 = blocks * rows * 16;
  for (int64_t i = (int64_t)blockIdx.x * CE_THREADS + threadIdx.x; i < n4; i += (int64_t)gridDim.x * CE_THREADS) {
    const int64_t line = i / 16, blk = line / rows, row = line - blk * rows, v0 = blk * 64 + (i - line * 16) * 4;
    const int64_t t = load_id(targets, id64, row);
    float e[4] = {0.f, 0.f, 0.f, 0.f};
    if (t >= 0 && t < vocab && v0 < vocab) {
      const float4 z = *reinterpret_cast<const float4*>(Z + i * 4);
      const float2 st = stat[row];
      const float x[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const bool of_target = v0 + k == t;
        const float y = ((of_target ? zt[row] : x[k]) - st.x) - st.y;
        e[k] = v0 + k >= vocab ? 0.f : of_target ? expm1f(y) : expf(y);
      }
    }
#pragma unroll
    for (int p = 0; p < 3; ++p) {
      const uint32_t lo = next_part_bf16x2(e[0], e[1]), hi = next_part_bf16x2(e[2], e[3]);
      *reinterpret_cast<uint2*>(G + (p * blocks * rows + line) * 64 + (i - line * 16) * 4) = make_uint2(lo, hi);
    }
  }
}

unsigned stride_blocks(const Ctx* ctx, int64_t items) {
  const int64_t blocks = (items + CE_THREADS - 1) / CE_THREADS, most = (int64_t)ctx->sm_count * 32;
  return (unsigned)(blocks < most ? blocks : most);
}

// What the rows [r0, r0 + n) of a 16-bit call keep of their logits, to G.
template <typename T>
int make_g(Ctx* ctx, const CeArgs& c, const CeScratch& s, const ce::Blocks& G, int64_t r0, int64_t n, const void* targets) {
  const int64_t row_groups = (n + 32 * SCALE_ROWS - 1) / (32 * SCALE_ROWS), blocks = G.blocks();
  for (int64_t b = 0; b < blocks; b += 65535) {
    const int64_t nb = blocks - b < 65535 ? blocks - b : 65535;
    ZOACT_CUDA_TRY(launch_pdl(ctx, ce_scale_kernel<T>, dim3((unsigned)row_groups, (unsigned)nb), dim3(CE_THREADS), 0, G.p, b, n,
                              (const float2*)s.part, s.part_ld, (const float2*)s.stat + r0, (const float*)s.zt + r0, targets,
                              c.id64, c.vocab));
    ++ctx->n_launch;
  }
  return ZOACT_OK;
}

// The products on the tensor cores; fp32 operands in three bf16 parts.  Where the gradient is asked for, chunk by chunk of
// rows: logits, of which 16 bits (fp32: all) are kept, the rows' sums, G, and its two products.
template <typename T>
int run(Ctx* ctx, const CeArgs& c) {
  using ce::Operand;
  constexpr bool F32 = sizeof(T) == 4;
  constexpr int PARTS = F32 ? 3 : 1;
  const int optype = F32 ? ZOACT_DT_BF16 : c.dtype;
  const int64_t tiles = (c.vocab + ce::V_TILE - 1) / ce::V_TILE, blocks = (c.vocab + 63) / 64;
  const bool grad = c.dH || c.dW;
  const size_t row_bytes = (size_t)blocks * 64 * (F32 ? 10 : 2);       // of G (fp32: the logits and three parts)
  int64_t chunk = c.rows;
  if (grad) {
    chunk = (int64_t)(((size_t)1 << 31) / row_bytes) / 256 * 256;
    if (chunk < 256) chunk = 256;
    if (chunk > c.rows) chunk = c.rows;
  }
  CeScratch s;
  if (!ce_scratch(ctx, c.rows, chunk, tiles, s)) return ZOACT_ERR_NOMEM;
  float* lse = c.lse ? c.lse : s.lse;
  float* loss = c.loss ? c.loss : s.loss;
  Operand W = {c.W, optype, c.vocab, c.d, c.d, 1, c.vocab * c.d}, H = {c.H, optype, c.rows, c.d, c.d, 1, c.rows * c.d};
  const bool few = F32 && ce::few_rows(ctx, c.rows, c.vocab, c.d);
  if (F32 && (grad || !few)) {
    const int64_t ld = (c.d + 7) / 8 * 8;
    uint16_t* W3 = (uint16_t*)scratch(ctx, SLOT_CE_SPLIT, (size_t)(c.vocab + c.rows) * ld * 6);
    if (!W3) return ZOACT_ERR_NOMEM;
    uint16_t* H3 = W3 + 3 * c.vocab * ld;
    ZOACT_CUDA_TRY(launch_pdl(ctx, ce_split_kernel, dim3(stride_blocks(ctx, (c.vocab + c.rows) * (c.d / 4))), dim3(CE_THREADS), 0,
                              (const float*)c.W, c.vocab, W3, (const float*)c.H, c.rows, H3, c.d, (int)ld));
    ++ctx->n_launch;
    W = {W3, optype, c.vocab, c.d, ld, 3, c.vocab * ld};
    H = {H3, optype, c.rows, c.d, ld, 3, c.rows * ld};
  }
  // the logits of rows [r0, r0 + h.rows), kept in G as asked for
  auto logits = [&](const Operand& h, int64_t r0, const void* targets, int keep, const ce::Blocks& G) {
    if (few)
      return ce::launch_logits_few(ctx, (const float*)c.W, c.vocab, (const float*)c.H + r0 * c.d, h.rows, c.d, s.part, s.part_ld,
                                   s.zt + r0, targets, c.id64, c.T, keep, G);
    return ce::launch_logits(ctx, W, h, s.part, s.part_ld, s.zt + r0, targets, c.id64, c.T, keep, G);
  };
  int st;
  if (!grad) {
    st = logits(H, 0, c.targets, ce::KEEP_NONE, ce::Blocks{});
    if (!st) st = join(ctx, c, s, tiles, 0, c.rows, lse, loss);
    return st ? st : finish(ctx, c, loss);
  }
  char* kept = (char*)scratch(ctx, SLOT_CE_G, (size_t)chunk * row_bytes);
  if (!kept) return ZOACT_ERR_NOMEM;
  // several chunks add to dW in fp32: a 16-bit dW is rounded from the whole sum
  float* dWf = nullptr;
  if (c.dW && chunk < c.rows && c.wgdtype != ZOACT_DT_FP32) {
    dWf = (float*)scratch(ctx, SLOT_CE_DW, (size_t)c.vocab * c.d * 4);
    if (!dWf) return ZOACT_ERR_NOMEM;
  }
  st = make_alpha(ctx, c, s, c.dtype == ZOACT_DT_FP16 ? c.grad_scale / G_SCALE_FP16 : c.grad_scale);
  if (st) return st;
  for (int64_t r0 = 0; r0 < c.rows; r0 += chunk) {
    const int64_t n = c.rows - r0 < chunk ? c.rows - r0 : chunk;
    Operand Hc = H;
    Hc.p = (const uint16_t*)H.p + r0 * H.ld;
    Hc.rows = n;
    ce::Blocks G = {kept, optype, n, c.vocab, PARTS};
    const void* targets = (const char*)c.targets + r0 * (c.id64 ? 8 : 4);
    st = logits(Hc, r0, targets, F32 ? ce::KEEP_Z : ce::KEEP_LOG, G);
    if (!st) st = join(ctx, c, s, tiles, r0, n, lse, loss);
    if (st) return st;
    if constexpr (F32) {
      G.p = kept + (size_t)blocks * n * 64 * 4;
      ZOACT_CUDA_TRY(launch_pdl(ctx, ce_split_g_kernel, dim3(stride_blocks(ctx, blocks * n * 16)), dim3(CE_THREADS), 0,
                                (const float*)kept, (uint16_t*)G.p, blocks, n, (const float2*)s.stat + r0, (const float*)s.zt + r0,
                                targets, c.id64, c.vocab));
      ++ctx->n_launch;
    } else {
      st = make_g<T>(ctx, c, s, G, r0, n, targets);
    }
    if (!st && c.dH) st = ce::launch_by_h(ctx, W, G, s.alpha, (T*)c.dH + r0 * c.d, c.dtype);
    if (!st && c.dW)
      st = ce::launch_by_w(ctx, G, Hc, targets, c.id64, s.alpha, dWf ? (void*)dWf : c.dW,
                           dWf ? ZOACT_DT_FP32 : c.wgdtype, r0 > 0 || c.accumulate);
    if (st) return st;
  }
  if constexpr (!F32) {
    if (dWf) {
      const int64_t total = c.vocab * c.d / 4;      // d is a multiple of 8
      ZOACT_CUDA_TRY(launch_pdl(ctx, ce_round_kernel<T>, dim3(stride_blocks(ctx, total)), dim3(CE_THREADS), 0, (const float4*)dWf,
                                total, (T*)c.dW));
      ++ctx->n_launch;
    }
  }
  return finish(ctx, c, loss);
}

}  // namespace

int launch_ce(Ctx* ctx, const CeArgs& c) {
  if (c.rows == 0) {                       // no token: losses of 0, no gradient
    if (c.dW && !c.accumulate)
      ZOACT_CUDA_TRY(cudaMemsetAsync(c.dW, 0, (size_t)c.vocab * c.d * dtype_size(c.wgdtype), ctx->stream));
    return finish(ctx, c, nullptr);
  }
  switch (c.dtype) {
    case ZOACT_DT_FP32: return run<float>(ctx, c);
    case ZOACT_DT_BF16: return run<__nv_bfloat16>(ctx, c);
    default: return run<__half>(ctx, c);
  }
}

}  // namespace zoact
