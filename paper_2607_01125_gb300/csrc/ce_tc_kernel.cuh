// The three products of the cross entropy over a vocabulary on CTA pairs (tcgen05 cta_group::2):
//
//   logits   z   = H W^T     M = rows,  N = vocab, K = d      epilogue: maximum and sum of exponentials per row, a thread a row
//            z^T = W H^T     M = vocab, N = rows,  K = d      the same over the accumulator's lanes, for few or ragged rows
//   by H     dH^T = W^T G^T  M = d,     N = rows,  K = vocab  epilogue: transposed store, or K pieces of the last tiles
//   by W     dW = G^T H      M = vocab, N = d,     K = rows   epilogue: row-major store
//
// Rows on the N side make the padding of a ragged or small batch cheap (tiles of 32 to 256 rows in steps of 32); there the
// logits' statistics reduce by a butterfly of shuffles that leaves lane l with column l of 32, which a thread that owns a
// row does without: a tile's epilogue took 13 000 cycles with shuffles, more than two groups of the main loop.
// W is read as it lies: as rows of 64 elements, and by columns as M-major tiles, 64 x 64 boxes whose descriptors step by boxes
// along M and by 8 K rows along K.  G, which only these kernels see, lies in blocks of 64 vocabulary entries,
// [block][row][64]: every box of it is contiguous, and M-major for the product by W.  H is small and is transposed for that one
// (read by columns as an N-major tile beside the M-major one, it ran at 1630 TFLOP/s).
// fp32 operands come as three bf16 parts each (24 bits); six products of parts run as six passes over K into one accumulator.
//
// The tensor core cuts its running fp32 sum off at every step of 16 products instead of rounding it: 4096 products of logits
// came out 4e-6 low, five times what fp32 FMAs err by.  K is therefore taken in groups (Params::group_kb) whose sums the
// epilogue adds up in registers, rounded; a group's sum is read while the next one runs into the other accumulator.
//
// Roles, barriers and bounded waits are those of the pair forward on CTA pairs: a TMA producer in each CTA, one MMA issuer
// in the leader, eight epilogue warps in each (two warpgroups), two to four accumulators in TMEM (as many as fit).
//
// Measured (bf16, 4096 x 128256 unless said): 32 rows 154 us, W at 6.8 TB/s; 4096 rows 2.10 ms with the tensor pipe 98% busy;
// with gradients 2048 rows 1.11 / 1.13 / 1.05 ms (93 to 97%, under the power cap), 333 rows of 5120 x 50272 in fp16
// 142 to 155 / 128 to 132 / 147 to 149 us (60 / 70 / 56%: 384 rows of MMA for 333, and the last one's stores); fp32, 1024 rows of
// 4096 x 50272 1.70 ms the loss and 4.84 ms with gradients (1.5 PFLOP/s of the six products).
#pragma once
#include "pair_tc2_kernel.cuh"

namespace zoact {
namespace ce {

constexpr int BM = 128, BN = 256, BK = 64;                // BM: rows of a CTA, a pair has 2 BM
constexpr int A_BYTES = BM * BK * 2;
// The ring: stages of A and bn / 2 rows of B, as many as fit (6 at bn = 256, 10 at 32).
constexpr int MAX_STAGES = 10;
__host__ __device__ constexpr int stage_bytes(int bn) { return A_BYTES + bn / 2 * BK * 2; }
constexpr int BOX_BYTES = 64 * BK * 2;                    // an M- or N-major box
constexpr int EPI_THREADS = 256, EPI_BASE = 128, THREADS = EPI_BASE + EPI_THREADS;
// Registers: 384 threads are launched with 168 each; the first warpgroup (producer, issuer) gives back what the epilogue's
// two take for a tile's sums: 56 + 2 x 224 = 3 x 168.
constexpr int REGS_ISSUE = 56, REGS_EPI = 224;
constexpr int TMEM_COLS = 512, MAX_BUF = 4;
constexpr int STG_BYTES = 16384;                          // a staging buffer (128 rows x 128 bytes)
enum Epi {
  EPI_LSE = 0,   // the rows' statistics
  EPI_LOG,       // and the tile's maximum - z as 16-bit fixed point
  EPI_Z,         // and z in fp32
  EPI_COL,       // D^T scaled
  EPI_ROW,       // D scaled, from registers
  EPI_ROW_STAGED // the same through shared memory
};

// Epilogue area beside the ring: a staging buffer for each warpgroup, or two.
__host__ __device__ constexpr int aux_bytes(int epi) { return epi == EPI_ROW_STAGED ? 4 * STG_BYTES : 2 * STG_BYTES; }
__host__ __device__ constexpr int ring_bytes(int epi) { return 229376 - aux_bytes(epi); }
constexpr int SMEM_BYTES = 1024 + 229376 + 256;
static_assert(SMEM_BYTES <= 232448, "dynamic shared memory above the 227 KB a CTA may use");

struct Maps {
  CUtensorMap a, b, out;
};

struct Params {
  int num_m, num_n, num_kb, products, bn;
  int n_first;                      // tile order: along N first (the operand of M streams, that of N stays in L2), or along M
  int group_kb;                     // K-blocks of one accumulation on the tensor core
  int tail_first, tail_split;       // tiles from tail_first on run as tail_split pieces of K each
  int64_t M, N;
  int g_blocks;                     // blocks of 64 vocabulary entries of one part of G
  int bf16;
  int* status;
  int nbuf, stages;                 // accumulators in TMEM, stages of the ring
  // logits: row r's target is targets[r % T]
  float2* part;                     // [ceil(vocab / 128)][part_ld]: maximum and sum of exp(z - maximum)
  int64_t part_ld;
  float* zt;
  const void* targets;
  int id64;
  uint32_t T;
  int64_t rows, vocab;
  void* G;                          // EPI_LOG, EPI_Z: [ceil(vocab / 64)][rows][64]
  // products by H and W: out = alpha D
  const float* alpha;
  void* out;                        // EPI_COL: [N, M]
  float* tail_part;                 // pieces of the tail's tiles: [piece][tile][bn][256]
  int add, out_32;                  // EPI_ROW: add to out (fp32); out and its rows lie on 32 bytes
};

struct Shared {
  uint64_t full[MAX_STAGES], empty[MAX_STAGES], tmem_full[MAX_BUF], tmem_empty[MAX_BUF], drain;
  uint32_t tmem_base;
  int abort_flag, epi_ok;
};
static_assert(sizeof(Shared) <= 256, "barrier block outgrew its shared-memory slot");

struct Unit {
  int m, n, kb0, kb1, slot;         // slot: index of a piece, or -1 for a whole tile
};

__device__ __forceinline__ bool unit_at(const Params& p, int u, Unit& w) {
  const int tiles = p.num_m * p.num_n, tail = tiles - p.tail_first, K = p.num_kb * p.products;
  int t = u;
  w.kb0 = 0; w.kb1 = K; w.slot = -1;
  if (u >= p.tail_first) {
    const int s = u - p.tail_first;
    if (s >= tail * p.tail_split) return false;
    const int j = s / tail;         // pieces of one K range run together: they share their operands' lines in L2
    t = p.tail_first + (s - j * tail);
    if (p.tail_split > 1) {
      w.kb0 = (int)((int64_t)j * K / p.tail_split);
      w.kb1 = (int)((int64_t)(j + 1) * K / p.tail_split);
      w.slot = s;
    }
  }
  if (p.n_first) {
    w.m = t / p.num_n;
    w.n = t - w.m * p.num_n;
  } else {
    w.n = t / p.num_m;
    w.m = t - w.n * p.num_m;
  }
  return true;
}

__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap* map, int32_t x, int32_t y, int32_t z,
                                                 uint32_t bar_cluster) {
  asm volatile(
      "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], "
      "[%5];" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar_cluster)
      : "memory");
}
// Add the box in shared memory to the tensor's elements (fp32), each once.
__device__ __forceinline__ void tma_add_2d(const CUtensorMap* map, int32_t x, int32_t y, uint32_t src) {
  asm volatile("cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x),
               "r"(y), "r"(src)
               : "memory");
}

// Low words of the operands' descriptors at `tile` (both with 128-byte swizzling; the high words are constants), and what a
// step of 16 in K adds.  K-major: rows of BK elements, 1024 bytes for 8 rows.  M-major: boxes of 64 elements x BK rows of K,
// BOX_BYTES apart along M, 1024 bytes for 8 rows of K.
constexpr uint32_t SDESC_HI = (1024u >> 4) | 1u << 14 | 2u << 29;
__device__ __forceinline__ uint32_t sdesc_lo(uint32_t tile, bool mn) {
  return tile >> 4 | (mn ? (uint32_t)(BOX_BYTES >> 4) << 16 : 1u << 16);
}
__device__ __forceinline__ uint64_t sdesc(uint32_t lo) { return (uint64_t)SDESC_HI << 32 | lo; }
__host__ __device__ constexpr uint32_t sdesc_step(bool mn) { return mn ? 2048u >> 4 : 32u >> 4; }

// One lane of a converged warp, the same one each time.
__device__ __forceinline__ bool elect_one() {
  uint32_t is;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
  return is != 0;
}
// A wait of a whole warp (in every lane, with one answer).
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* status) {
  return __all_sync(0xffffffffu, tc::mbar_wait(bar, parity, abort_flag, status));
}

// Reduce 32 columns over the warp's 32 lanes: lane l returns column l's maximum (sum).  x is overwritten.
template <bool MAX>
__device__ __forceinline__ float columns_over_lanes(float* x, int lane) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const bool up = lane & o;
#pragma unroll
    for (int i = 0; i < o; ++i) {
      const float send = up ? x[i] : x[i + o], keep = up ? x[i + o] : x[i];
      const float got = __shfl_xor_sync(0xffffffffu, send, o);
      x[i] = MAX ? fmaxf(keep, got) : keep + got;
    }
  }
  return x[0];
}

// The accumulators in turn.
struct Ring {
  int buf = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void next(int nbuf) {
    if (++buf == nbuf) { buf = 0; phase ^= 1u; }
  }
};

// Wait until accumulator r.buf is complete (pairtc::epi_wait_full), and give it back to the issuer once every epilogue
// thread of this CTA has read it.
__device__ __forceinline__ bool acc_wait(const Params& p, Shared* ss, const Ring& r, int etid, volatile int* abort_flag) {
  return pairtc::epi_wait_full(ss, r.buf, r.phase, abort_flag, p.status, etid);
}
__device__ __forceinline__ void acc_free(Shared* ss, const Ring& r, int etid) {
  tc::tc_fence_before();
  tc::named_bar_sync(3, EPI_THREADS);
  if (etid == 0) pairtc::tc2::arrive_cluster(pairtc::tc2::map_to(tc::smem_u32(&ss->tmem_empty[r.buf]), 0));
}

// A warp's part of an accumulator tile: 32 lanes, and its warpgroup's 32-column chunks: the half's own 128 columns
// (ADJACENT), or chunks half, half + 2, ...
constexpr int CHUNKS = BN / 64;
struct Part {
  float x[CHUNKS][32];
};
template <bool ADJACENT>
__device__ __forceinline__ int chunk_of(int half, int i) { return ADJACENT ? half * CHUNKS + i : half + 2 * i; }

// The sums over a unit's K groups, each read from its accumulator as soon as it is complete.  False: the wait gave up.
template <bool ADJACENT>
__device__ __forceinline__ bool sum_groups(const Params& p, Shared* ss, const Unit& w, int etid, int half, uint32_t t_quad,
                                           volatile int* abort_flag, Ring& r, Part& a) {
  const int nch = p.bn / 32;
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
    for (int j = 0; j < 32; ++j) a.x[i][j] = 0.f;
#pragma unroll 1
  for (int kb = w.kb0; kb < w.kb1; kb += p.group_kb) {
    if (!acc_wait(p, ss, r, etid, abort_flag)) return false;
    const uint32_t t = t_quad + (uint32_t)(r.buf * p.bn);
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      const int c = chunk_of<ADJACENT>(half, i);
      if (c < nch) {
        float y[32];
        tc::tmem_ld32(t + (uint32_t)(c * 32), y);
#pragma unroll
        for (int j = 0; j < 32; ++j) a.x[i][j] += y[j];
      }
    }
    acc_free(ss, r, etid);
    r.next(p.nbuf);
  }
  return true;
}

// Fixed point of the tile's maximum - z: 1 / LOG_STEPS, up to 32 (below exp(-32) of the tile's largest: 65535, no value);
// rounded in the low bits of a sum with 2^23.  x = z - maximum.
__device__ __forceinline__ uint32_t log_fixed(float x) {
  return __float_as_uint(fminf(x * -LOG_STEPS, 65535.f) + 8388608.f) & 0xffffu;
}
__device__ __forceinline__ float exp_of(float x) { return pairtc::exp2_sfu(x * 1.44269504f); }
// What a tile's exponentials are taken from: its maximum m, or 0 where all of its logits are minus infinity (the difference of
// two of these would be NaN; from 0 each exponential is 0, and the tile leaves a sum of 0).
__device__ __forceinline__ float exp_base(float m) { return m == -INFINITY ? 0.f : m; }

// One tile of logits, M = rows: a thread has a row and the 128 vocabulary entries of its warpgroup from v0.  A row's target leaves
// by itself (zt) and is none of its tile's entries: beside its exponential, a nearly sure row's others would be rounded off.
template <int EPI>
__device__ __forceinline__ void epi_rows(const Params& p, const Maps& tm, uint8_t* stg, Part& a, int etid, int half, int row_in_cta,
                                         int64_t m0, int64_t v0, bool& pending) {
  const int64_t row = m0 + row_in_cta;
  const bool ok = row < p.rows;
  const int64_t left = p.vocab - v0;
  const int nv = left >= 128 ? 128 : left > 0 ? (int)left : 0;          // uniform
  if (nv < 128) {
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
      for (int j = 0; j < 32; ++j)
        if (i * 32 + j >= nv) a.x[i][j] = -INFINITY;
  }
  const int64_t t = ok ? load_id(p.targets, p.id64, (uint32_t)row % p.T) - v0 : -1;
  if (t >= 0 && t < nv) {                                               // seldom
    float z = 0.f;
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
      for (int j = 0; j < 32; ++j) {
        if (i * 32 + j != (int)t) continue;
        z = a.x[i][j];
        a.x[i][j] = -INFINITY;
      }
    p.zt[row] = z;
  }
  if (EPI == EPI_Z && ok) {
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      if (i * 32 >= nv) continue;
      float4* g = reinterpret_cast<float4*>(reinterpret_cast<float*>(p.G) + (((v0 / 64 + i / 2) * p.rows + row) * 64 + (i & 1) * 32));
#pragma unroll
      for (int j = 0; j < 8; ++j) g[j] = make_float4(a.x[i][4 * j], a.x[i][4 * j + 1], a.x[i][4 * j + 2], a.x[i][4 * j + 3]);
    }
  }
  float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i)
#pragma unroll
    for (int j = 0; j < 32; ++j) mx[j & 3] = fmaxf(mx[j & 3], a.x[i][j]);
  const float m = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])), from = exp_base(m);
  float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) {
#pragma unroll
    for (int j = 0; j < 32; ++j) a.x[i][j] -= from;
    if (EPI == EPI_LOG && (i & 1) == 0) {           // a box of 64 entries: wait until the last one has been read
      if ((etid & 127) == 0 && pending) tc::bulk_wait_read0();
      tc::named_bar_sync(4 + half, 128);
    }
    if (EPI == EPI_LOG) {
      const uint32_t sbuf = tc::smem_u32(stg + half * STG_BYTES);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        uint32_t q[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) q[k] = log_fixed(a.x[i][8 * g + 2 * k]) | log_fixed(a.x[i][8 * g + 2 * k + 1]) << 16;
        tc::st_shared_v4(sbuf + pairtc::sw128_off(row_in_cta, (i & 1) * 4 + g), make_uint4(q[0], q[1], q[2], q[3]));
      }
      if (i & 1) {
        tc::fence_proxy_async_smem();
        tc::named_bar_sync(4 + half, 128);
        if ((etid & 127) == 0 && (i / 2) * 64 < nv && m0 < p.rows) {
          tc::tma_store_3d(&tm.out, 0, (int32_t)m0, (int32_t)(v0 / 64 + i / 2), sbuf);
          tc::bulk_commit();
          pending = true;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 32; ++j) s[j & 3] += exp_of(a.x[i][j]);
  }
  if (ok && nv > 0) p.part[v0 / BM * p.part_ld + row] = make_float2(m, (s[0] + s[1]) + (s[2] + s[3]));
}

// Exchange area of the epilogue below, per warpgroup: [quad][column of its chunks], and each warp's copy of the columns'
// maxima for broadcast reads.
struct Exchange {
  float mx[2][4][128], sum[2][4][128], all[8][128];
};
static_assert(sizeof(Exchange) <= aux_bytes(0), "exchange area");

// One tile of logits, M = vocab: this CTA's 128 entries from m0 and the tile's rows from n0; warp `quad` takes 32 entries.
template <int EPI>
__device__ __forceinline__ void epi_lanes(const Params& p, Exchange* ex, Part& a, int half, int quad, int lane, int64_t m0,
                                          int64_t n0) {
  const int nch = p.bn / 32;
  const int64_t v = m0 + quad * 32 + lane, vb = m0 + quad * 32;
  const bool vok = v < p.vocab;
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) {
    const int c = chunk_of<false>(half, i);
    if (c >= nch) continue;
    // the target's logit, where one of these rows has its target among this warp's entries (seldom)
    const int64_t n = n0 + c * 32 + lane;
    const int64_t t = n < p.rows ? load_id(p.targets, p.id64, (uint32_t)n % p.T) : -1;
    unsigned hits = __ballot_sync(0xffffffffu, t >= vb && t < vb + 32 && t < p.vocab);
    while (hits) {
      const int l = __ffs(hits) - 1;
      hits &= hits - 1;
      const int src = (int)(__shfl_sync(0xffffffffu, t, l) - vb);
      float z = 0.f;
#pragma unroll
      for (int j = 0; j < 32; ++j) {
        if (j != l) continue;
        z = a.x[i][j];
        if (lane == src) a.x[i][j] = -INFINITY;
      }
      if (lane == src) p.zt[n0 + c * 32 + l] = z;
    }
    float y[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) y[j] = vok ? a.x[i][j] : -INFINITY;
    ex->mx[half][quad][i * 32 + lane] = columns_over_lanes<true>(y, lane);
  }
  tc::named_bar_sync(4 + half, 128);
  float* all = ex->all[half * 4 + quad];
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) {
    const int k = i * 32 + lane;
    if (chunk_of<false>(half, i) < nch)
      all[k] = exp_base(fmaxf(fmaxf(ex->mx[half][0][k], ex->mx[half][1][k]), fmaxf(ex->mx[half][2][k], ex->mx[half][3][k])));
  }
  __syncwarp();
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) {
    const int c = chunk_of<false>(half, i);
    if (c >= nch) continue;
    const int64_t n = n0 + c * 32;
    const int nv = (int)(p.rows - n < 32 ? p.rows - n : 32);
    const int64_t at = ((v >> 6) * p.rows + n) * 64 + (v & 63);       // a row is 64 elements from the next
    if (EPI == EPI_Z && vok) {
      float* g = reinterpret_cast<float*>(p.G) + at;
#pragma unroll
      for (int j = 0; j < 32; ++j)
        if (j < nv) g[j * 64] = a.x[i][j];
    }
#pragma unroll
    for (int j = 0; j < 32; j += 4) {
      const float4 m = *reinterpret_cast<const float4*>(all + i * 32 + j);
      a.x[i][j] -= m.x;
      a.x[i][j + 1] -= m.y;
      a.x[i][j + 2] -= m.z;
      a.x[i][j + 3] -= m.w;
    }
    if (EPI == EPI_LOG && vok) {
      uint16_t* g = reinterpret_cast<uint16_t*>(p.G) + at;
#pragma unroll
      for (int j = 0; j < 32; ++j)
        if (j < nv) g[j * 64] = (uint16_t)log_fixed(a.x[i][j]);
    }
#pragma unroll
    for (int j = 0; j < 32; ++j) a.x[i][j] = vok ? exp_of(a.x[i][j]) : 0.f;
    ex->sum[half][quad][i * 32 + lane] = columns_over_lanes<false>(a.x[i], lane);
  }
  tc::named_bar_sync(4 + half, 128);
  // chunk i's statistics by warp i of the warpgroup
  const int c = chunk_of<false>(half, quad), k = quad * 32 + lane;
  const int64_t n = n0 + c * 32 + lane;
  if (c < nch && n < p.rows && m0 < p.vocab) {
    const float s = (ex->sum[half][0][k] + ex->sum[half][1][k]) + (ex->sum[half][2][k] + ex->sum[half][3][k]);
    p.part[m0 / BM * p.part_ld + n] = make_float2(s == 0.f ? -INFINITY : all[k], s);     // a sum of 0: see exp_base
  }
}

// D^T scaled (or a K piece of it, unscaled fp32): a warp stores 32 consecutive elements of each row.
template <typename TO>
__device__ __forceinline__ void epi_col(const Params& p, const Part& a, int half, int row_in_cta, uint32_t rank, int64_t m0,
                                        int64_t n0, int slot, float f) {
  const int nch = p.bn / 32;
  if (slot >= 0) {
    float* d = p.tail_part + ((size_t)slot * p.bn + half * 32) * (2 * BM) + rank * BM + row_in_cta;
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
      if (chunk_of<false>(half, i) >= nch) break;
#pragma unroll
      for (int j = 0; j < 32; ++j) d[(i * 64 + j) * (2 * BM)] = a.x[i][j];
    }
    return;
  }
  if (m0 + row_in_cta >= p.M) return;
  TO* d = reinterpret_cast<TO*>(p.out) + (n0 + half * 32) * p.M + m0 + row_in_cta;
  int left = (int)(p.N - n0 < p.bn ? p.N - n0 : p.bn) - half * 32;      // rows from this warpgroup's first chunk on
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) {
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      if (j < left) *d = from_f32<TO>(a.x[i][j] * f);
      d += p.M;
      asm volatile("" : "+l"(d));          // one address at a time: 32 of them do not fit beside the sums
    }
    d += 32 * p.M;
    left -= 64;
  }
}

// 32 bytes of one thread, or two halves where a row does not lie on 32 bytes.
__device__ __forceinline__ void store_32(void* p, const uint32_t* w, bool whole) {
  if (whole) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                 "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
  } else {
    reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
    reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
  }
}

// D scaled, from registers: a thread has a row's 128 columns of its warpgroup and writes them in whole sectors.  Staged in
// shared memory for bulk stores, a tile's 64 KB of writes and reads there compete with the operands of a long main loop (loss
// and gradient for W alone, 4096 x 128256 in bf16: 1024 rows 1432 us for 1399).  Where K is short the output's bytes are the
// bound, and boxes of 128 rows reach DRAM in better order (1 row: 354 us for 475, 256 rows 464 for 566, 768 rows 1114 for
// 1123), so both stay: see STAGED_BELOW.
template <typename TO>
__device__ __forceinline__ void epi_row(const Params& p, const Part& a, int half, int row_in_cta, int64_t m0, int64_t n0, float f) {
  const int64_t m = m0 + row_in_cta, n = n0 + half * 128;
  if (m >= p.M) return;
  TO* d = reinterpret_cast<TO*>(p.out) + m * p.N + n;
  constexpr int PER = 32 / (int)sizeof(TO);          // elements of a store
  const int left = (int)(p.N - n < 128 ? p.N - n : 128);
  const bool whole = p.out_32 != 0;
#pragma unroll
  for (int i = 0; i < CHUNKS; ++i) {
    if (half * 128 + i * 32 >= p.bn) break;
#pragma unroll
    for (int j = 0; j < 32; j += PER) {
      const int c = i * 32 + j;
      if (c >= left) break;
      uint32_t w[8];
      if constexpr (sizeof(TO) == 2) {
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = pairtc::pack2(a.x[i][j + 2 * k] * f, a.x[i][j + 2 * k + 1] * f, (TO*)nullptr);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = __float_as_uint(a.x[i][j + k] * f);
        if (p.add) {
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (c + k < left) w[k] = __float_as_uint(__uint_as_float(w[k]) + d[c + k]);
        }
      }
      if (c + PER <= left)
        store_32(d + c, w, whole);
      else                                 // the last columns: 16 bytes
        *reinterpret_cast<uint4*>(d + c) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}

// The same through the warpgroup's two staging buffers in boxes of 128 bytes; one thread stores each pair of boxes (16-bit
// outputs are one pair: the only wait is for the tile before).
template <typename TO>
__device__ __forceinline__ void epi_row_staged(const Params& p, const Maps& tm, uint8_t* stg, Part& a, int etid, int half,
                                        int row_in_cta, int64_t m0, int64_t n0, float f, bool& pending) {
  constexpr int CC = 128 / (int)sizeof(TO), PAIRS = 128 / (2 * CC);
  const bool issuer = (etid & 127) == 0;
  const uint32_t sbuf = tc::smem_u32(stg + half * 2 * STG_BYTES);
#pragma unroll
  for (int c = 0; c < PAIRS; ++c) {
    const int64_t n = n0 + half * 128 + c * 2 * CC;
    if (n >= p.N || m0 >= p.M || half * 128 >= p.bn) break;      // uniform over the warpgroup
    if (issuer && pending) tc::bulk_wait_read0();               // the buffers' previous stores have read them
    tc::named_bar_sync(4 + half, 128);
#pragma unroll
    for (int i = c * 2 * CC / 32; i < (c + 1) * 2 * CC / 32; ++i) {
#pragma unroll
      for (int j = 0; j < 32; ++j) a.x[i][j] *= f;
      const int q = i * 32 - c * 2 * CC;
      pairtc::stage_granules<TO, 32>(sbuf + (uint32_t)(q / CC * STG_BYTES), row_in_cta, q % CC, a.x[i], true);
    }
    tc::fence_proxy_async_smem();
    tc::named_bar_sync(4 + half, 128);
    if (issuer) {
      for (int b = 0; b < 2 && n + b * CC < p.N; ++b) {
        if (sizeof(TO) == 4 && p.add) tma_add_2d(&tm.out, (int32_t)(n + b * CC), (int32_t)m0, sbuf + b * STG_BYTES);
        else tc::tma_store_2d(&tm.out, (int32_t)(n + b * CC), (int32_t)m0, sbuf + b * STG_BYTES);
      }
      tc::bulk_commit();
      pending = true;
    }
  }
}

// ROWS_M: the logits' form with rows on the M side.
template <int EPI, bool ROWS_M, typename TO>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS, 1)
ce_tc_kernel(const __grid_constant__ Maps tm, const Params p) {
  namespace tc2 = pairtc::tc2;
  // by H: A = W by columns, B = G by rows; by W: A = G by columns, B = H^T by rows
  constexpr bool BY_W = EPI == EPI_ROW || EPI == EPI_ROW_STAGED, A_MN = EPI == EPI_COL || BY_W;
  constexpr bool A_BLOCKS = BY_W, B_BLOCKS = EPI == EPI_COL;                // G
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* aux = smem + ring_bytes(EPI);
  Shared* ss = reinterpret_cast<Shared*>(aux + aux_bytes(EPI));
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const uint32_t rank = __shfl_sync(0xffffffffu, tc2::cluster_rank(), 0);
  const bool leader = rank == 0;
  volatile int* abort_flag = &ss->abort_flag;

  if (threadIdx.x == 0) {
    for (int s = 0; s < MAX_STAGES; ++s) {
      tc::mbar_init(tc::smem_u32(&ss->full[s]), 2);    // one producer arrival from each CTA (the leader's copy is used)
      tc::mbar_init(tc::smem_u32(&ss->empty[s]), 1);
    }
    for (int b = 0; b < MAX_BUF; ++b) {
      tc::mbar_init(tc::smem_u32(&ss->tmem_full[b]), 1);
      tc::mbar_init(tc::smem_u32(&ss->tmem_empty[b]), 2);
    }
    tc::mbar_init(tc::smem_u32(&ss->drain), 1);
    ss->abort_flag = 0;
    tc::fence_mbar_init();
    tc::prefetch_tmap(&tm.a);
    tc::prefetch_tmap(&tm.b);
    if ((EPI == EPI_LOG && ROWS_M) || EPI == EPI_ROW_STAGED) tc::prefetch_tmap(&tm.out);
  }
  if (warp == 1) {
    tc2::tmem_alloc2(tc::smem_u32(&ss->tmem_base), TMEM_COLS);
    tc2::tmem_relinquish2();
  }
  tc::tc_fence_before();
  __syncthreads();
  tc2::cluster_sync();                    // both CTAs' barriers exist before any remote arrival
  tc::tc_fence_after();
  const uint32_t tmem_base = __shfl_sync(0xffffffffu, ss->tmem_base, 0);
  pdl_wait();
  pdl_trigger();

  const int cluster_id = blockIdx.x >> 1, n_clusters = gridDim.x >> 1;
  const int bh = p.bn / 2, sbytes = stage_bytes(p.bn);
  Unit w;

  if (warp < EPI_BASE / 32) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_ISSUE));
    // Both loops run in whole warps that elect a lane for each copy, MMA and arrival: what the compiler knows to be the
    // warp's own is in the registers that these instructions take.  (One lane's loop took 333 ns a K-block, whatever its
    // size, and a division for the K-block's product 26 of them.)
    if (warp == 0) {
      // ---------------- TMA producer (both CTAs) ----------------
      const uint32_t stage_tx = (uint32_t)(A_BYTES + bh * BK * 2);
      const uint32_t ring = tc::smem_u32(smem), empty = tc::smem_u32(&ss->empty[0]);
      const uint32_t full = tc2::map_to(tc::smem_u32(&ss->full[0]), 0);       // the leader's
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int u = cluster_id; ok && unit_at(p, u, w); u += n_clusters) {
        const int m0 = w.m * 2 * BM + (int)rank * BM, n0 = w.n * p.bn + (int)rank * bh;
        // products of parts (a, b): (0,0) (0,1) (1,0) (0,2) (1,1) (2,0)
        int pr = w.kb0 / p.num_kb, kblk = w.kb0 - pr * p.num_kb;
        for (int kb = w.kb0; kb < w.kb1; ++kb) {
          if (!warp_wait(empty + (uint32_t)stage * 8u, phase ^ 1u, abort_flag, p.status)) { ok = false; break; }
          const uint32_t bar = full + (uint32_t)stage * 8u;
          const uint32_t sa = ring + (uint32_t)(stage * sbytes), sb = sa + A_BYTES;
          const int k = kblk * BK, pa = (0x210100 >> (4 * pr)) & 15, pb = (0x012010 >> (4 * pr)) & 15;
          if (elect_one()) {
            tc2::arrive_expect_tx_cluster(bar, stage_tx);
            if (A_BLOCKS) {
              tma_load_3d_pair(sa, &tm.a, 0, k, m0 / 64 + pa * p.g_blocks, bar);
              tma_load_3d_pair(sa + BOX_BYTES, &tm.a, 0, k, m0 / 64 + 1 + pa * p.g_blocks, bar);
            } else if (A_MN) {
              tma_load_3d_pair(sa, &tm.a, m0, k, pa, bar);
              tma_load_3d_pair(sa + BOX_BYTES, &tm.a, m0 + 64, k, pa, bar);
            } else {
              tma_load_3d_pair(sa, &tm.a, k, m0, pa, bar);
            }
            if (B_BLOCKS) {
              tma_load_3d_pair(sb, &tm.b, 0, n0, kblk + pb * p.g_blocks, bar);
            } else {
              tma_load_3d_pair(sb, &tm.b, k, n0, pb, bar);
            }
          }
          __syncwarp();
          if (++kblk == p.num_kb) { kblk = 0; ++pr; }
          if (++stage == p.stages) { stage = 0; phase ^= 1u; }
        }
      }
      if (!ok) {
        // our copies complete on the leader's barriers; give them time to land before the CTA winds down
        const uint64_t t0 = tc::global_timer_ns();
        while (tc::global_timer_ns() - t0 < 2000000ull) {
        }
      }
    } else if (warp == 1 && leader) {
      // ---------------- MMA issuer (leader CTA) ----------------
      const uint32_t idesc = tc::idesc_f16(2 * BM, p.bn, p.bf16) | (A_MN ? 1u << 15 : 0u);
      const uint32_t ring_a = sdesc_lo(tc::smem_u32(smem), A_MN), ring_b = sdesc_lo(tc::smem_u32(smem) + A_BYTES, false);
      const uint32_t full = tc::smem_u32(&ss->full[0]), empty = tc::smem_u32(&ss->empty[0]);
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true, issued_any = false;
      Ring r;
      for (int u = cluster_id; ok && unit_at(p, u, w); u += n_clusters) {
        for (int g0 = w.kb0; ok && g0 < w.kb1; g0 += p.group_kb) {
          const int g1 = min(g0 + p.group_kb, w.kb1);
          if (!warp_wait(tc::smem_u32(&ss->tmem_empty[r.buf]), r.phase ^ 1u, abort_flag, p.status)) { ok = false; break; }
          tc::tc_fence_after();
          const uint32_t d_tmem = tmem_base + (uint32_t)(r.buf * p.bn);
          for (int kb = g0; kb < g1; ++kb) {
            if (!warp_wait(full + (uint32_t)stage * 8u, phase, abort_flag, p.status)) { ok = false; break; }
            tc::tc_fence_after();
            const uint32_t at = (uint32_t)(stage * sbytes) >> 4;
            if (elect_one()) {
#pragma unroll
              for (int k = 0; k < BK / 16; ++k)
                tc2::mma2_f16(d_tmem, sdesc(ring_a + at + (uint32_t)k * sdesc_step(A_MN)),
                              sdesc(ring_b + at + (uint32_t)k * sdesc_step(false)), idesc, (kb != g0 || k != 0) ? 1u : 0u);
              tc2::commit2_both(empty + (uint32_t)stage * 8u);
            }
            __syncwarp();
            issued_any = true;
            if (++stage == p.stages) { stage = 0; phase ^= 1u; }
          }
          if (!ok) break;
          if (elect_one()) tc2::commit2_both(tc::smem_u32(&ss->tmem_full[r.buf]));
          __syncwarp();
          r.next(p.nbuf);
        }
      }
      if (issued_any) {
        if (elect_one()) tc2::commit2_own(tc::smem_u32(&ss->drain));
        __syncwarp();
        tc::mbar_wait_drain(tc::smem_u32(&ss->drain), 0, 100000000ull);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_EPI));
    // ---------------- epilogue (warps 4..11, both CTAs) ----------------
    const int etid = threadIdx.x - EPI_BASE, half = etid >> 7, quad = warp & 3;
    const int row_in_cta = quad * 32 + lane;
    float f = 0.f;
    if (EPI == EPI_COL || BY_W) f = __ldcg(p.alpha);
    Ring r;
    bool pending = false;
    const uint32_t t_quad = tmem_base + ((uint32_t)(quad * 32) << 16);
    for (int u = cluster_id; unit_at(p, u, w); u += n_clusters) {
      const int64_t m0 = (int64_t)w.m * 2 * BM + (int64_t)rank * BM, n0 = (int64_t)w.n * p.bn;
      Part a;
      if (!sum_groups<ROWS_M || BY_W>(p, ss, w, etid, half, t_quad, abort_flag, r, a)) break;
      if constexpr (EPI == EPI_ROW)
        epi_row<TO>(p, a, half, row_in_cta, m0, n0, f);
      else if constexpr (EPI == EPI_ROW_STAGED)
        epi_row_staged<TO>(p, tm, aux, a, etid, half, row_in_cta, m0, n0, f, pending);
      else if constexpr (EPI == EPI_COL)
        epi_col<TO>(p, a, half, row_in_cta, rank, m0, n0, w.slot, f);
      else if constexpr (ROWS_M)
        epi_rows<EPI>(p, tm, aux, a, etid, half, row_in_cta, m0, n0 + half * 128, pending);
      else
        epi_lanes<EPI>(p, reinterpret_cast<Exchange*>(aux), a, half, quad, lane, m0, n0);
    }
    if (pending) tc::bulk_wait0();
  }

  tc::tc_fence_before();
  __syncthreads();
  tc2::cluster_sync();                    // the peer's MMAs and copies are done before TMEM and smem go away
  if (warp == 1) {
    __syncwarp();
    tc::tc_fence_after();
    tc2::tmem_dealloc2(tmem_base, TMEM_COLS);
  }
}

}  // namespace ce
}  // namespace zoact
