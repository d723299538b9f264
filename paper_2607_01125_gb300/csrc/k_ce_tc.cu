// Launches of the cross entropy's tensor-core products.
#include "ce_tc.h"
#include "ce_tc_kernel.cuh"

namespace zoact {
namespace ce {
namespace {

// K-blocks of 64 that the tensor core sums by itself: its cut-off costs about 1.6e-8 of the sum for each 16 products.  Logits
// end in fp32 (8 blocks: 5e-7); the product by H ends in 16 bits (64: 4e-6).
constexpr int LOGIT_GROUP = 8, BY_H_GROUP = 64;

int encode(CUtensorMap* map, const Operand& o, int box_rows) {
  return encode_tmap_3d_16bit(map, o.p, o.dtype, o.parts, o.rows, o.cols, o.ld, o.part_stride, box_rows);
}

template <int EPI, bool A_MN, bool B_MN, typename TO>
int launch(Ctx* ctx, const Maps& tm, const Params& p) {
  auto kern = ce_tc_kernel<EPI, A_MN, B_MN, TO>;
  ZOACT_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_BYTES));
  const int64_t units = p.tail_first + (int64_t)(p.num_m * p.num_n - p.tail_first) * p.tail_split;
  const int pairs = ctx->sm_count / 2;
  const int clusters = units < pairs ? (int)units : pairs;
  ZOACT_CUDA_TRY(launch_pdl(ctx, kern, dim3(2 * clusters), dim3(THREADS), SMEM_BYTES, tm, p));
  ++ctx->n_launch;
  ZOACT_CHECK_LAUNCH();
  return ZOACT_OK;
}

int up32(int64_t n) { return n >= BN ? BN : (int)((n + 31) / 32 * 32); }

// Rows per tile of m_tiles x rows outputs: the fewest waves of pairs, a tile's time taken as its width plus a part that
// does not depend on it.
int tile_rows(const Ctx* ctx, int64_t m_tiles, int64_t rows) {
  const int pairs = ctx->sm_count / 2;
  int best = up32(rows);
  double least = 0.0;
  for (int bn = best; bn >= 32; bn -= 32) {
    const int64_t tiles = m_tiles * ((rows + bn - 1) / bn);
    const double cost = (double)((tiles + pairs - 1) / pairs) * (bn + 32);
    if (least == 0.0 || cost < 0.99 * least) {
      least = cost;
      best = bn;
    }
  }
  return best;
}

// The sum of a tail tile's pieces in K order, scaled: out[n, m] from [piece][tile][bn][256].
template <typename TO>
__global__ void __launch_bounds__(256)
ce_tail_kernel(const float* __restrict__ part, int tail_first, int tail, int split, int num_n, int bn, int64_t M, int64_t N,
               const double* __restrict__ count, float scale, TO* __restrict__ out) {
  pdl_wait();
  pdl_trigger();
  const int t = tail_first + blockIdx.x, mb = t / num_n, nb = t - mb * num_n;
  const int64_t m = (int64_t)mb * 2 * BM + threadIdx.x, n = (int64_t)nb * bn + blockIdx.y;
  if (m >= M || n >= N) return;
  const float* src = part + ((size_t)blockIdx.x * bn + blockIdx.y) * (2 * BM) + threadIdx.x;
  const size_t step = (size_t)tail * bn * (2 * BM);
  float s = 0.f;
#pragma unroll 4
  for (int j = 0; j < split; ++j) s += __ldcg(src + j * step);
  out[n * M + m] = from_f32<TO>(s * (float)((double)scale / fmax(*count, 1.0)));
}

// Tiles that fill no whole wave of pairs, cut along K: the pieces whose rounds of 1 / split tile, with the time to write
// and read their fp32 sums, are the shortest.
int tail_pieces(int64_t tail, int64_t kblocks, int pairs, int bn) {
  int best = 1;
  double least = 0.0;
  for (int s = 1; s <= 32 && (s == 1 || kblocks / s >= 8); ++s) {
    const double rounds = (double)((tail * s + pairs - 1) / pairs) / s;
    // in K-blocks of a tile (about 0.3 us for 256 rows): 2 x 4 bytes of 256 bn sums a piece at 6 TB/s, over all pairs
    const double io = s == 1 ? 0.0 : tail * s * 2048.0 * bn / 6e6 / 0.3 + 10.0;
    const double cost = rounds * kblocks + io;
    if (s == 1 || cost < 0.98 * least) {
      least = cost;
      best = s;
    }
  }
  return best;
}

template <typename TO>
int run_by_h(Ctx* ctx, const Maps& tm, Params& p, const double* count, float scale, void* out) {
  const int tiles = p.num_m * p.num_n, pairs = ctx->sm_count / 2, tail = tiles % pairs;
  p.tail_first = tiles;
  p.tail_split = 1;
  if (tail > 0) {
    p.tail_split = tail_pieces(tail, (int64_t)p.num_kb * p.products, pairs, p.bn);
    if (p.tail_split > 1) {
      p.tail_first = tiles - tail;
      p.tail_part = (float*)scratch(ctx, SLOT_CE_TAIL, (size_t)tail * p.tail_split * p.bn * 2 * BM * 4);
      if (!p.tail_part) { p.tail_first = tiles; p.tail_split = 1; }
    }
  }
  const int st = launch<EPI_COL, true, false, TO>(ctx, tm, p);
  if (st || p.tail_split == 1) return st;
  ZOACT_CUDA_TRY(launch_pdl(ctx, ce_tail_kernel<TO>, dim3((unsigned)tail, (unsigned)p.bn), dim3(256), 0, (const float*)p.tail_part,
                            p.tail_first, tail, p.tail_split, p.num_n, p.bn, p.M, p.N, count, scale, (TO*)out));
  ++ctx->n_launch;
  return ZOACT_OK;
}

}  // namespace

int launch_logits(Ctx* ctx, const Operand& W, const Operand& H, float2* part, int64_t part_ld, float* zt, const void* targets,
                  int id64, int64_t T, int keep, void* G, int64_t ldg) {
  Params p = {};
  p.M = W.rows; p.N = H.rows;
  p.num_m = (int)((p.M + 2 * BM - 1) / (2 * BM));
  p.bn = tile_rows(ctx, p.num_m, p.N);
  p.num_n = (int)((p.N + p.bn - 1) / p.bn);
  p.num_kb = (int)((W.cols + BK - 1) / BK);
  p.products = W.parts == 3 ? 6 : 1;
  p.group_kb = LOGIT_GROUP;
  p.tail_first = p.num_m * p.num_n; p.tail_split = 1;
  p.bf16 = W.dtype == ZOACT_DT_BF16; p.status = ctx->d_status;
  p.part = part; p.part_ld = part_ld; p.zt = zt; p.targets = targets; p.id64 = id64; p.T = T; p.G = G; p.ldg = ldg;
  Maps tm;
  int st = encode(&tm.a, W, BM);
  if (!st) st = encode(&tm.b, H, p.bn / 2);
  if (st) return st;
  tm.out = tm.a;
  switch (keep) {
    case KEEP_LOG: return launch<EPI_LOG, false, false, float>(ctx, tm, p);
    case KEEP_Z: return launch<EPI_Z, false, false, float>(ctx, tm, p);
    default: return launch<EPI_LSE, false, false, float>(ctx, tm, p);
  }
}

int launch_by_h(Ctx* ctx, const Operand& W, const Operand& G, const double* count, float scale, void* out, int dtype) {
  Params p = {};
  p.M = W.cols; p.N = G.rows;
  p.num_m = (int)((p.M + 2 * BM - 1) / (2 * BM));
  p.num_kb = (int)((W.rows + BK - 1) / BK);
  p.products = W.parts == 3 ? 6 : 1;
  p.group_kb = BY_H_GROUP;
  // the tail is cut along K: only the rows' padding counts
  p.bn = tile_rows(ctx, 1 << 20, p.N);
  p.num_n = (int)((p.N + p.bn - 1) / p.bn);
  p.bf16 = W.dtype == ZOACT_DT_BF16; p.status = ctx->d_status;
  p.count = count; p.scale = scale; p.out = out;
  Maps tm;
  int st = encode(&tm.a, W, 64);
  if (!st) st = encode(&tm.b, G, p.bn / 2);
  if (st) return st;
  tm.out = tm.a;
  switch (dtype) {
    case ZOACT_DT_FP32: return run_by_h<float>(ctx, tm, p, count, scale, out);
    case ZOACT_DT_BF16: return run_by_h<__nv_bfloat16>(ctx, tm, p, count, scale, out);
    default: return run_by_h<__half>(ctx, tm, p, count, scale, out);
  }
}

int launch_by_w(Ctx* ctx, const Operand& G, const Operand& H, const double* count, float scale, void* out, int dtype, int add) {
  Params p = {};
  p.M = G.cols; p.N = H.cols;
  p.num_m = (int)((p.M + 2 * BM - 1) / (2 * BM));
  p.bn = p.N > 128 ? 256 : 128;      // whole boxes of 64 for each CTA
  p.num_n = (int)((p.N + p.bn - 1) / p.bn);
  p.num_kb = (int)((H.rows + BK - 1) / BK);
  p.products = H.parts == 3 ? 6 : 1;
  p.group_kb = p.num_kb * p.products;
  p.tail_first = p.num_m * p.num_n; p.tail_split = 1;
  p.bf16 = H.dtype == ZOACT_DT_BF16; p.status = ctx->d_status;
  p.count = count; p.scale = scale; p.out = out; p.add = add;
  Maps tm;
  int st = encode(&tm.a, G, 64);
  if (!st) st = encode(&tm.b, H, 64);
  if (!st) st = encode_tmap_store(&tm.out, out, dtype, p.M, p.N, 128 / (int)dtype_size(dtype), BM, true);
  if (st) return st;
  switch (dtype) {
    case ZOACT_DT_FP32: return launch<EPI_ROW, true, true, float>(ctx, tm, p);
    case ZOACT_DT_BF16: return launch<EPI_ROW, true, true, __nv_bfloat16>(ctx, tm, p);
    default: return launch<EPI_ROW, true, true, __half>(ctx, tm, p);
  }
}

}  // namespace ce
}  // namespace zoact
