// Rotary positions: the pair (a, b) of frequency f in every head of row r turns by the angle position f,
//     a' = a cos - b sin,  b' = a sin + b cos        (inverse: by the opposite angle, which is the gradient).
//
// The angle is kept in turns, as a 64-bit fraction of one: a position times the frequency's fraction (zoact_rope_init), modulo
// 2^64, is the fraction of a turn that the rotation leaves -- an exact product, so that a far position loses nothing to the
// reduction that a 32-bit angle would (position 10^6 in fp32: 0.03 radians).  Its two top bits are the quadrant, and the rest
// goes to sine and cosine as a fraction of at most 1/8 turn.
//
// Bound by memory: every element is read and written once.  A block makes the sines and cosines of its rows once, in shared
// memory, for all of a row's heads, and then moves 16 bytes of both halves (or of neighbouring pairs) at a time, two of a
// thread's pieces in flight (four: 40 us for 35 at the first size below, the same at the second).
//
// Measured (GB300): 8192 rows of 40 heads of 128 in bf16 34.9 us (4.8 TB/s; a copy of as much takes 28.7), 3001 rows of 80 heads
// of 80, 32 of them turned, in fp16 20.3 to 21.2 us (3.7 TB/s).
#include <cmath>

#include "internal.h"

namespace zoact {
namespace {

constexpr int THREADS = 256, TABLE = 1024;      // TABLE: sines and cosines of a block

struct Turns {
  uint64_t t[ZOACT_ROPE_MAX / 2];
};

// (cos, sin) of a fraction of a turn.
__device__ __forceinline__ float2 cos_sin_turns(uint64_t t) {
  const uint32_t quadrant = (uint32_t)((t + (1ull << 61)) >> 62) & 3u;
  const int32_t rest = (int32_t)(uint32_t)((t - ((uint64_t)quadrant << 62)) >> 32);     // +- 1/8 turn, in 2^-32 turns
  float s, c;
  sincospif((float)rest * 0x1p-31f, &s, &c);
  if (quadrant & 1u) {
    const float k = c;
    c = -s;
    s = k;
  }
  return quadrant & 2u ? make_float2(-c, -s) : make_float2(c, s);
}

template <typename T, int N> struct alignas(sizeof(T) * N) Vec { T v[N]; };

// A piece of a head: what is read for it, and turned in place.
template <typename T, int V, bool HALF> struct Piece {
  static constexpr int W = HALF || V > 1 ? V : 2;              // elements of one half, or of neighbouring pairs
  Vec<T, W> a, b;
  __device__ __forceinline__ void load(const T* x, int nf) {
    if constexpr (!HALF && V == 1) {
      a.v[0] = x[0];
      a.v[1] = x[1];
    } else {
      a = *reinterpret_cast<const Vec<T, W>*>(x);
      if constexpr (HALF) b = *reinterpret_cast<const Vec<T, W>*>(x + nf);
    }
  }
  __device__ __forceinline__ void turn(const float2* cs) {
    if constexpr (HALF) {
#pragma unroll
      for (int j = 0; j < W; ++j) {
        const float2 w = cs[j];
        const float u = to_f32<T>(a.v[j]), v = to_f32<T>(b.v[j]);
        a.v[j] = from_f32<T>(u * w.x - v * w.y);
        b.v[j] = from_f32<T>(u * w.y + v * w.x);
      }
    } else {
#pragma unroll
      for (int j = 0; j < W; j += 2) {
        const float2 w = cs[j / 2];
        const float u = to_f32<T>(a.v[j]), v = to_f32<T>(a.v[j + 1]);
        a.v[j] = from_f32<T>(u * w.x - v * w.y);
        a.v[j + 1] = from_f32<T>(u * w.y + v * w.x);
      }
    }
  }
  __device__ __forceinline__ void store(T* y, int nf) const {
    if constexpr (!HALF && V == 1) {
      y[0] = a.v[0];
      y[1] = a.v[1];
    } else {
      *reinterpret_cast<Vec<T, W>*>(y) = a;
      if constexpr (HALF) *reinterpret_cast<Vec<T, W>*>(y + nf) = b;
    }
  }
};

// V elements at a time (V = 1: any alignment).  np: pieces of a head that turn; nc: pieces behind them that are copied.  MANY
// pieces of a thread are read before the first is written (X may be Y, which the compiler has to allow for).
constexpr int MANY = 2;
template <typename T, int V, bool HALF>
__global__ void __launch_bounds__(THREADS)
rope_kernel(const T* X, int64_t ld_x, T* Y, int64_t ld_y, int64_t rows, int head_dim, int rot, int np, Divisor pieces, Divisor per_row,
            const void* __restrict__ positions, int id64, uint32_t n_pos, int rows_block, int inverse,
            const __grid_constant__ Turns turns) {
  using P = Piece<T, V, HALF>;
  __shared__ float2 table[TABLE];
  pdl_wait();
  pdl_trigger();
  const int64_t r0 = (int64_t)blockIdx.x * rows_block;
  const int nr = (int)(rows - r0 < rows_block ? rows - r0 : rows_block), nf = rot / 2;
  for (int i = threadIdx.x; i < nr * nf; i += THREADS) {
    const int r = i / nf, f = i - r * nf;
    const uint64_t pos = (uint64_t)load_id(positions, id64, (uint32_t)((uint64_t)(r0 + r) % n_pos));
    const float2 cs = cos_sin_turns(pos * turns.t[f]);
    table[i] = make_float2(cs.x, inverse ? -cs.y : cs.y);
  }
  __syncthreads();
  const int total = nr * per_row.d;
  for (int i0 = threadIdx.x; i0 < total; i0 += MANY * THREADS) {
    P v[MANY];
    int64_t to[MANY];
    int cs[MANY];                              // the first of its cosines and sines, or -1: copied
#pragma unroll
    for (int k = 0; k < MANY; ++k) {
      const int i = min(i0 + k * THREADS, total - 1);
      int in_row, p;
      const int r = per_row.div(i, in_row), head = pieces.div(in_row, p);
      const bool copy = p >= np;
      const int d = copy ? rot + (p - np) * V : p * P::W;
      const int64_t at = (int64_t)head * head_dim + d;
      const T* x = X + (r0 + r) * ld_x + at;
      to[k] = (r0 + r) * ld_y + at;
      cs[k] = copy ? -1 : r * nf + (HALF ? d : d / 2);
      if (copy) {
        const Vec<T, V> c = *reinterpret_cast<const Vec<T, V>*>(x);
#pragma unroll
        for (int j = 0; j < V; ++j) v[k].a.v[j] = c.v[j];
      } else {
        v[k].load(x, nf);
      }
    }
#pragma unroll
    for (int k = 0; k < MANY; ++k) {
      if (i0 + k * THREADS >= total) break;
      if (cs[k] < 0) {
        Vec<T, V> c;
#pragma unroll
        for (int j = 0; j < V; ++j) c.v[j] = v[k].a.v[j];
        *reinterpret_cast<Vec<T, V>*>(Y + to[k]) = c;
      } else {
        v[k].turn(table + cs[k]);
        v[k].store(Y + to[k], nf);
      }
    }
  }
}

template <typename T, bool HALF>
int launch(Ctx* ctx, const RopeArgs& a, const Turns& turns) {
  const int nf = a.rope->rot / 2, rest = a.head_dim - a.rope->rot;
  constexpr int V = 16 / (int)sizeof(T);
  const auto lies = [&](const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld % V == 0; };
  const bool vec = lies(a.X, a.ld_x) && lies(a.Y, a.ld_y) && a.head_dim % V == 0 && (HALF ? nf : 2 * nf) % V == 0;
  const int v = vec ? V : 1;
  const int np = HALF ? nf / v : vec ? 2 * nf / v : nf, nc = a.X == a.Y ? 0 : rest / v;
  // Rows of a block: as many as the table holds, fewer where the SMs would not have two blocks each.
  int rows_block = TABLE / nf < 8 ? TABLE / nf : 8;
  while (rows_block > 1 && a.rows < (int64_t)2 * ctx->sm_count * rows_block) rows_block /= 2;
  const int64_t blocks = (a.rows + rows_block - 1) / rows_block;
  const auto run = [&](auto kern) {
    return launch_pdl(ctx, kern, dim3((unsigned)blocks), dim3(THREADS), 0, (const T*)a.X, a.ld_x, (T*)a.Y, a.ld_y, a.rows,
                      a.head_dim, a.rope->rot, np, Divisor(np + nc), Divisor(a.heads * (np + nc)), a.positions, a.id64,
                      (uint32_t)a.n_pos, rows_block, a.inverse, turns);
  };
  ZOACT_CUDA_TRY(vec ? run(rope_kernel<T, V, HALF>) : run(rope_kernel<T, 1, HALF>));
  ++ctx->n_launch;
  return ZOACT_OK;
}

}  // namespace

int launch_rope(Ctx* ctx, const RopeArgs& a) {
  if (a.rows == 0) return ZOACT_OK;
  Turns turns = {};
  for (int i = 0; i < a.rope->rot / 2; ++i) turns.t[i] = a.rope->turns[i];
  const bool half = a.rope->layout == ZOACT_ROPE_HALF;
  switch (a.dtype) {
    case ZOACT_DT_FP32: return half ? launch<float, true>(ctx, a, turns) : launch<float, false>(ctx, a, turns);
    case ZOACT_DT_BF16: return half ? launch<__nv_bfloat16, true>(ctx, a, turns) : launch<__nv_bfloat16, false>(ctx, a, turns);
    default: return half ? launch<__half, true>(ctx, a, turns) : launch<__half, false>(ctx, a, turns);
  }
}

}  // namespace zoact

// Frequencies in radians a position: base^(-2 i / rot), scaled for contexts longer than the original length.
extern "C" int zoact_rope_init(zoact_rope* rope, int32_t rot, int32_t layout, double base, int32_t scaling, double factor,
                               double low, double high, int64_t original) {
  if (!rope || rot < 2 || rot % 2 != 0 || (layout != ZOACT_ROPE_HALF && layout != ZOACT_ROPE_INTERLEAVED))
    return ZOACT_ERR_INVALID_ARG;
  if (rot > ZOACT_ROPE_MAX) return ZOACT_ERR_UNSUPPORTED;
  if (!(base > 1.0) || !std::isfinite(base) || scaling < ZOACT_ROPE_PLAIN || scaling > ZOACT_ROPE_PARTS)
    return ZOACT_ERR_INVALID_ARG;
  if (scaling != ZOACT_ROPE_PLAIN && (!(factor > 0.0) || !std::isfinite(factor))) return ZOACT_ERR_INVALID_ARG;
  if (scaling == ZOACT_ROPE_PARTS && (!(high > low) || !std::isfinite(low) || !std::isfinite(high) || original <= 0))
    return ZOACT_ERR_INVALID_ARG;
  const double two_pi = 6.283185307179586476925;
  if (scaling == ZOACT_ROPE_BASE && rot > 2) base *= std::pow(factor, (double)rot / (rot - 2));
  if (!std::isfinite(base) || !(base > 0.0)) return ZOACT_ERR_INVALID_ARG;
  zoact_rope r = {};
  r.rot = rot;
  r.layout = layout;
  for (int i = 0; i < ZOACT_ROPE_MAX / 2; ++i) {
    double f = 0.0;
    if (i < rot / 2) f = std::pow(base, -2.0 * i / rot);
    if (scaling == ZOACT_ROPE_LINEAR) f /= factor;
    if (scaling == ZOACT_ROPE_PARTS) {
      const double turns = (double)original * f / two_pi;
      const double keep = std::fmin(std::fmax((turns - low) / (high - low), 0.0), 1.0);
      f *= keep + (1.0 - keep) / factor;
    }
    if (!std::isfinite(f)) return ZOACT_ERR_INVALID_ARG;
    const double t = f / two_pi, part = t - std::floor(t);          // below 1: its 53 bits are part of the 64
    r.turns[i] = (uint64_t)std::ldexp(part, 64);
  }
  *rope = r;
  return ZOACT_OK;
}
