// Launches of the cross entropy's tensor-core products.
#include "ce_tc.h"
#include "ce_tc_kernel.cuh"

namespace zoact {
namespace ce {
namespace {

// K-blocks of 64 that the tensor core sums by itself, at most: its cut-off costs about 1.6e-8 of the sum for each 16 products,
// and reading a group's sum about 300 cycles of it.  Logits end in fp32: log-sum-exps err by 4e-7 (d 4096) to 6e-7 (5120) with 8
// blocks, half of that with 4 (333 rows 174 us for 163, 4096 rows 2.26 ms for 2.10), 8e-7 with 12 (333 rows 2% faster).
// Products of G, itself rounded to 16 bits, take 64 (4e-6), a dW in fp32 among them; fp32 operands, whose six products are
// summed alike, 4 (3e-7).
constexpr int LOGIT_GROUP = 8, GRAD_GROUP = 64, FP32_GROUP = 4;
// Rows on the M side are taken up to this much more padding: their epilogue has no reduction over lanes.  Loss and dH of a
// 4096 x 128256 head in bf16, rows on N / on M: 100 rows 357 us / 368, 200 rows 412 / 410, 400 rows 683 / 699, 512 rows
// 761 / 749, 1024 rows 1469 / 1404, 2048 rows 2795 / 2668; 333 rows of 5120 x 50272 in fp16 326 / 349.
constexpr double ROWS_M_GAIN = 1.15;
// fp32 rows that are multiplied as they are: up to this many (a head is then read as it is at most three times; loss by parts /
// as they are, 20000 x 1024: 8 rows 88 us / 28.6, 24 rows 88 / 47.5, 32 rows 88 / 64), or as many as fill no more than a
// block on each SM (128 rows of 256 against 1009 entries: 16.0 us / 10.8, of 4096: 103 / 49); and their shared memory at most.
constexpr int FEW_ROWS = 24, FEW_SMEM = 160 * 1024;
// K-blocks below which the product by W stores through shared memory (epi_row).
constexpr int STAGED_BELOW = 14;

int even_groups(int kb, int most) {
  const int groups = (kb + most - 1) / most;
  return (kb + groups - 1) / groups;
}

int encode(CUtensorMap* map, const Operand& o, int box_rows) {
  return encode_tmap_3d_16bit(map, o.p, o.dtype, o.parts, o.rows, o.cols, o.ld, o.part_stride, box_rows);
}
int encode(CUtensorMap* map, const Blocks& g, int box_rows) {
  return encode_tmap_3d_16bit(map, g.p, g.dtype, g.blocks() * g.parts, g.rows, 64, 64, g.rows * 64, box_rows);
}

template <int EPI, bool ROWS_M, typename TO>
int launch(Ctx* ctx, const Maps& tm, Params p) {
  p.stages = ring_bytes(EPI) / stage_bytes(p.bn);
  if (p.stages > MAX_STAGES) p.stages = MAX_STAGES;
  auto kern = ce_tc_kernel<EPI, ROWS_M, TO>;
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

// The time of `tiles` tiles of 2 BM x bn in whole waves of pairs, in units of one column: a tile's time is taken as its width
// plus a part that does not depend on it (a K-block of 64, 333 rows: 217 ns at 96 columns, 244 at 128, 306 at 192, 340 at 256).
double wave_cost(const Ctx* ctx, int64_t tiles, int bn) {
  const int pairs = ctx->sm_count / 2;
  return (double)((tiles + pairs - 1) / pairs) * (bn + 128);
}

// Rows per tile of m_tiles x rows outputs, the rows on the N side.
int tile_rows(const Ctx* ctx, int64_t m_tiles, int64_t rows, double* cost) {
  int best = up32(rows);
  double least = 0.0;
  for (int bn = best; bn >= 32; bn -= 32) {
    const double c = wave_cost(ctx, m_tiles * ((rows + bn - 1) / bn), bn);
    if (least == 0.0 || c < 0.99 * least) {
      least = c;
      best = bn;
    }
  }
  if (cost) *cost = least;
  return best;
}

// Accumulators: as many as fit in TMEM.
int buffers(int bn) { return TMEM_COLS / bn < MAX_BUF ? TMEM_COLS / bn : MAX_BUF; }

// The sum of a tail tile's pieces in K order, scaled: out[n, m] from [piece][tile][bn][256].
template <typename TO>
__global__ void __launch_bounds__(256)
ce_tail_kernel(const float* __restrict__ part, int tail_first, int tail, int split, int num_n, int bn, int64_t M, int64_t N,
               const float* __restrict__ alpha, TO* __restrict__ out) {
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
  out[n * M + m] = from_f32<TO>(s * __ldg(alpha));
}

// Logits of a few fp32 rows, each read of W's used for FEW rows: a block has V_TILE entries of the vocabulary, a warp four of
// them at a time, its lanes their columns; H's rows lie in shared memory.  Splitting W for the tensor cores reads and writes
// 2.5 times its bytes before the product reads them again: see FEW_ROWS.  Two blocks an SM (128 registers) carry a head of
// little more than one block each: 20000 x 1024 28 us for 38 with one (50272 x 4096, 8 rows: 199 for 185).
constexpr int FEW = 8, FEW_THREADS = 256, FEW_ENTRIES = 4;
static_assert(FEW * FEW_ENTRIES == 32 && FEW == FEW_THREADS / 32, "a lane a sum, a warp a row");

__global__ void __launch_bounds__(FEW_THREADS, 2)
ce_few_kernel(const float* __restrict__ W, int64_t vocab, const float* __restrict__ H, int64_t rows, int d, int groups,
              float2* __restrict__ part, int64_t part_ld, float* __restrict__ zt, const void* __restrict__ targets, int id64,
              int64_t T, float* __restrict__ Z) {
  pdl_wait();
  pdl_trigger();
  extern __shared__ __align__(16) uint8_t few_smem[];
  float* hs = reinterpret_cast<float*>(few_smem);                    // [FEW][d]
  __shared__ float z[V_TILE][FEW + 1];
  const int64_t tile = blockIdx.x / groups, r0 = (int64_t)(blockIdx.x - tile * groups) * FEW, v0 = tile * V_TILE;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c4 = d / 4;
  for (int i = threadIdx.x; i < FEW * c4; i += FEW_THREADS) {
    const int r = i / c4;
    reinterpret_cast<float4*>(hs)[i] =
        r0 + r < rows ? reinterpret_cast<const float4*>(H + (r0 + r) * d)[i - r * c4] : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  __syncthreads();
  for (int e0 = warp * FEW_ENTRIES; e0 < V_TILE; e0 += FEW_ENTRIES * FEW_THREADS / 32) {
    const float4* w[FEW_ENTRIES];
#pragma unroll
    for (int i = 0; i < FEW_ENTRIES; ++i) {
      const int64_t v = v0 + e0 + i;
      w[i] = reinterpret_cast<const float4*>(W + (v < vocab ? v : vocab - 1) * d);
    }
    float acc[FEW_ENTRIES * FEW];
#pragma unroll
    for (int k = 0; k < FEW_ENTRIES * FEW; ++k) acc[k] = 0.f;
#pragma unroll 4
    for (int c = lane; c < c4; c += 32) {
      float4 x[FEW_ENTRIES];
#pragma unroll
      for (int i = 0; i < FEW_ENTRIES; ++i) x[i] = __ldcs(w[i] + c);
#pragma unroll
      for (int r = 0; r < FEW; ++r) {
        const float4 h = reinterpret_cast<const float4*>(hs)[r * c4 + c];
#pragma unroll
        for (int i = 0; i < FEW_ENTRIES; ++i)
          acc[i * FEW + r] = fmaf(x[i].x, h.x, fmaf(x[i].y, h.y, fmaf(x[i].z, h.z, fmaf(x[i].w, h.w, acc[i * FEW + r]))));
      }
    }
    const float sum = columns_over_lanes<false>(acc, lane);
    z[e0 + lane / FEW][lane % FEW] = sum;
  }
  __syncthreads();
  const int64_t row = r0 + warp;
  if (row >= rows) return;
  const int64_t t = load_id(targets, id64, row % T) - v0, blocks = (vocab + 63) / 64;
  float x[V_TILE / 32], m = -INFINITY, s = 0.f;
#pragma unroll
  for (int k = 0; k < V_TILE / 32; ++k) {
    const int e = k * 32 + lane;
    x[k] = v0 + e < vocab ? z[e][warp] : -INFINITY;
    if (e == t && v0 + e < vocab) {                                  // the target leaves by itself
      zt[row] = x[k];
      x[k] = -INFINITY;
    }
    m = fmaxf(m, x[k]);
    if (Z && (v0 + e) / 64 < blocks) Z[((v0 + e) / 64 * rows + row) * 64 + (e & 63)] = x[k];
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
#pragma unroll
  for (int k = 0; k < V_TILE / 32; ++k) s += expf(x[k] - exp_base(m));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (lane == 0) part[tile * part_ld + row] = make_float2(m, s);
}

// Tiles that fill no whole wave of pairs, cut along K: the pieces whose rounds of 1 / split tile, with the time to write
// and read their fp32 sums, are the shortest.
int tail_pieces(int64_t tail, int64_t kblocks, int pairs, int bn) {
  int best = 1;
  double least = 0.0;
  for (int s = 1; s <= 32 && (s == 1 || kblocks / s >= 8); ++s) {
    const double rounds = (double)((tail * s + pairs - 1) / pairs) / s;
    // in K-blocks of a tile (about 0.3 us for 256 rows): 4 bytes of 256 bn sums a piece read at 3 TB/s, over all pairs
    const double io = s == 1 ? 0.0 : tail * s * 1024.0 * bn / 3e6 / 0.3 + 10.0;
    const double cost = rounds * kblocks + io;
    if (s == 1 || cost < 0.98 * least) {
      least = cost;
      best = s;
    }
  }
  return best;
}

template <typename TO>
int run_by_h(Ctx* ctx, const Maps& tm, Params& p, const float* alpha, void* out) {
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
  const int st = launch<EPI_COL, false, TO>(ctx, tm, p);
  if (st || p.tail_split == 1) return st;
  ZOACT_CUDA_TRY(launch_pdl(ctx, ce_tail_kernel<TO>, dim3((unsigned)tail, (unsigned)p.bn), dim3(256), 0, (const float*)p.tail_part,
                            p.tail_first, tail, p.tail_split, p.num_n, p.bn, p.M, p.N, alpha, (TO*)out));
  ++ctx->n_launch;
  return ZOACT_OK;
}

}  // namespace

int launch_logits(Ctx* ctx, const Operand& W, const Operand& H, float2* part, int64_t part_ld, float* zt, const void* targets,
                  int id64, int64_t T, int keep, const Blocks& G) {
  Params p = {};
  const int64_t v_tiles = (W.rows + 2 * BM - 1) / (2 * BM), r_tiles = (H.rows + 2 * BM - 1) / (2 * BM);
  double lanes_cost = 0.0;
  p.bn = tile_rows(ctx, v_tiles, H.rows, &lanes_cost);
  // rows on the M side unless their padding to 256 costs more than the shuffles of the other form
  const bool rows_m = wave_cost(ctx, r_tiles * v_tiles, BN) <= ROWS_M_GAIN * lanes_cost;
  if (rows_m) p.bn = BN;
  p.M = rows_m ? H.rows : W.rows;
  p.N = rows_m ? W.rows : H.rows;
  p.num_m = (int)(rows_m ? r_tiles : v_tiles);
  p.num_n = (int)((p.N + p.bn - 1) / p.bn);
  p.num_kb = (int)((W.cols + BK - 1) / BK);
  p.products = W.parts == 3 ? 6 : 1;
  p.group_kb = even_groups(p.num_kb * p.products, p.products > 1 ? FP32_GROUP : LOGIT_GROUP);
  p.nbuf = buffers(p.bn);
  p.tail_first = p.num_m * p.num_n; p.tail_split = 1;
  p.bf16 = W.dtype == ZOACT_DT_BF16; p.status = ctx->d_status;
  p.part = part; p.part_ld = part_ld; p.zt = zt; p.targets = targets; p.id64 = id64; p.T = (uint32_t)T;
  p.rows = H.rows; p.vocab = W.rows; p.G = G.p;
  p.n_first = !rows_m;
  Maps tm;
  int st = encode(&tm.a, rows_m ? H : W, BM);
  if (!st) st = encode(&tm.b, rows_m ? W : H, p.bn / 2);
  if (!st && keep == KEEP_LOG) st = encode(&tm.out, G, BM);
  if (st) return st;
  if (keep != KEEP_LOG) tm.out = tm.a;
  switch (keep) {
    case KEEP_LOG: return rows_m ? launch<EPI_LOG, true, float>(ctx, tm, p) : launch<EPI_LOG, false, float>(ctx, tm, p);
    case KEEP_Z: return rows_m ? launch<EPI_Z, true, float>(ctx, tm, p) : launch<EPI_Z, false, float>(ctx, tm, p);
    default: return rows_m ? launch<EPI_LSE, true, float>(ctx, tm, p) : launch<EPI_LSE, false, float>(ctx, tm, p);
  }
}

bool few_rows(const Ctx* ctx, int64_t rows, int64_t vocab, int d) {
  const int64_t blocks = (vocab + V_TILE - 1) / V_TILE * ((rows + FEW - 1) / FEW);
  return (rows <= FEW_ROWS || blocks <= ctx->sm_count) && (int64_t)FEW * d * 4 <= FEW_SMEM;
}

int launch_logits_few(Ctx* ctx, const float* W, int64_t vocab, const float* H, int64_t rows, int d, float2* part,
                      int64_t part_ld, float* zt, const void* targets, int id64, int64_t T, int keep, const Blocks& G) {
  const int groups = (int)((rows + FEW - 1) / FEW);
  const int64_t blocks = (vocab + V_TILE - 1) / V_TILE * groups;
  ZOACT_CUDA_TRY(cudaFuncSetAttribute(ce_few_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, FEW_SMEM));
  ZOACT_CUDA_TRY(launch_pdl(ctx, ce_few_kernel, dim3((unsigned)blocks), dim3(FEW_THREADS), (size_t)FEW * d * 4, W, vocab, H, rows,
                            d, groups, part, part_ld, zt, targets, id64, T, keep == KEEP_Z ? (float*)G.p : (float*)nullptr));
  ++ctx->n_launch;
  return ZOACT_OK;
}

int launch_by_h(Ctx* ctx, const Operand& W, const Blocks& G, const float* alpha, void* out, int dtype) {
  Params p = {};
  p.M = W.cols; p.N = G.rows;
  p.num_m = (int)((p.M + 2 * BM - 1) / (2 * BM));
  p.num_kb = (int)G.blocks();
  p.g_blocks = p.num_kb;
  p.products = W.parts == 3 ? 6 : 1;
  p.group_kb = even_groups(p.num_kb * p.products, p.products > 1 ? FP32_GROUP : GRAD_GROUP);
  // the tail is cut along K: only the rows' padding counts
  p.bn = tile_rows(ctx, 1 << 20, p.N, nullptr);
  p.nbuf = buffers(p.bn);
  p.num_n = (int)((p.N + p.bn - 1) / p.bn);
  p.n_first = 1;
  p.bf16 = W.dtype == ZOACT_DT_BF16; p.status = ctx->d_status;
  p.alpha = alpha; p.out = out;
  Maps tm;
  int st = encode(&tm.a, W, 64);
  if (!st) st = encode(&tm.b, G, p.bn / 2);
  if (st) return st;
  tm.out = tm.a;
  switch (dtype) {
    case ZOACT_DT_FP32: return run_by_h<float>(ctx, tm, p, alpha, out);
    case ZOACT_DT_BF16: return run_by_h<__nv_bfloat16>(ctx, tm, p, alpha, out);
    default: return run_by_h<__half>(ctx, tm, p, alpha, out);
  }
}

// Rows of H to columns: [parts][rows][cols] (rows ld_in apart) to [parts][cols][ld_out], 64 x 64 a block.  Rows without a
// target become zeros: G's zeros would not take a NaN or an infinity out of the sum over the rows.
__global__ void __launch_bounds__(256)
ce_transpose_kernel(const uint16_t* __restrict__ in, int64_t rows, int cols, int64_t ld_in, int64_t part_in,
                    uint16_t* __restrict__ out, int64_t ld_out, const void* __restrict__ targets, int id64, int64_t vocab) {
  pdl_wait();
  pdl_trigger();
  __shared__ uint16_t t[64][66];
  __shared__ bool counted[64];
  const int64_t r0 = (int64_t)blockIdx.x * 64, c0 = (int64_t)blockIdx.y * 64;
  in += blockIdx.z * part_in;
  out += (int64_t)blockIdx.z * cols * ld_out;
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
  uint32_t in_w[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int64_t r = r0 + y + 8 * k, c = c0 + 2 * x;
    in_w[k] = 0;
    if (r < rows && c < cols) in_w[k] = *reinterpret_cast<const uint32_t*>(in + r * ld_in + c);      // cols is even
  }
  if (threadIdx.x < 64) {
    const int64_t id = r0 + threadIdx.x < rows ? load_id(targets, id64, r0 + threadIdx.x) : -1;
    counted[threadIdx.x] = id >= 0 && id < vocab;
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const uint32_t w = counted[y + 8 * k] ? in_w[k] : 0;
    t[y + 8 * k][2 * x] = (uint16_t)w;
    t[y + 8 * k][2 * x + 1] = (uint16_t)(w >> 16);
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int64_t c = c0 + y + 8 * k, r = r0 + 2 * x;
    if (c < cols && r < ld_out)            // ld_out is even; past `rows` zeros, which are not read
      *reinterpret_cast<uint32_t*>(out + c * ld_out + r) = (uint32_t)t[2 * x][y + 8 * k] | (uint32_t)t[2 * x + 1][y + 8 * k] << 16;
  }
}

int launch_by_w(Ctx* ctx, const Blocks& G, const Operand& H, const void* targets, int id64, const float* alpha, void* out,
                int dtype, int add) {
  const int64_t ld = (H.rows + 7) / 8 * 8;
  uint16_t* T = (uint16_t*)scratch(ctx, SLOT_CE_HT, (size_t)H.parts * H.cols * ld * 2);
  if (!T) return ZOACT_ERR_NOMEM;
  ZOACT_CUDA_TRY(launch_pdl(ctx, ce_transpose_kernel, dim3((unsigned)((H.rows + 63) / 64), (unsigned)((H.cols + 63) / 64), H.parts),
                            dim3(256), 0, (const uint16_t*)H.p, H.rows, (int)H.cols, H.ld, H.part_stride, T, ld,
                            targets, id64, G.vocab));
  ++ctx->n_launch;
  const Operand HT = {T, H.dtype, H.cols, H.rows, ld, H.parts, H.cols * ld};
  Params p = {};
  p.M = G.vocab; p.N = H.cols;
  p.num_m = (int)((p.M + 2 * BM - 1) / (2 * BM));
  p.bn = up32(p.N);
  p.nbuf = 2;
  p.num_n = (int)((p.N + p.bn - 1) / p.bn);
  p.n_first = 1;
  p.num_kb = (int)((H.rows + BK - 1) / BK);
  p.g_blocks = (int)G.blocks();
  p.products = H.parts == 3 ? 6 : 1;
  p.group_kb = even_groups(p.num_kb * p.products, p.products > 1 ? FP32_GROUP : GRAD_GROUP);
  p.tail_first = p.num_m * p.num_n; p.tail_split = 1;
  p.bf16 = H.dtype == ZOACT_DT_BF16; p.status = ctx->d_status;
  p.alpha = alpha; p.out = out; p.add = add;
  p.out_32 = ((uintptr_t)out & 31) == 0 && p.N * (int64_t)dtype_size(dtype) % 32 == 0;
  const bool staged = p.num_kb * p.products < STAGED_BELOW;
  Maps tm;
  int st = encode(&tm.a, G, 64);
  if (!st) st = encode(&tm.b, HT, p.bn / 2);
  if (!st && staged) st = encode_tmap_store(&tm.out, out, dtype, p.M, p.N, 128 / (int)dtype_size(dtype), BM, true);
  if (st) return st;
  if (!staged) tm.out = tm.a;
  switch (dtype) {
    case ZOACT_DT_FP32: return staged ? launch<EPI_ROW_STAGED, false, float>(ctx, tm, p) : launch<EPI_ROW, false, float>(ctx, tm, p);
    case ZOACT_DT_BF16:
      return staged ? launch<EPI_ROW_STAGED, false, __nv_bfloat16>(ctx, tm, p) : launch<EPI_ROW, false, __nv_bfloat16>(ctx, tm, p);
    default: return staged ? launch<EPI_ROW_STAGED, false, __half>(ctx, tm, p) : launch<EPI_ROW, false, __half>(ctx, tm, p);
  }
}

}  // namespace ce
}  // namespace zoact
