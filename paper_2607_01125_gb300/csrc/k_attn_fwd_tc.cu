// Attention over packed sequences on the tensor cores (16-bit operands, heads of up to 128 columns).
//
// Rows of work are (position, head of the group) pairs, so that the heads that share keys share a tile's reads of them, and a
// tile of a long causal sequence spans few positions.  A CTA runs two tiles of 128 rows against the same blocks of 128 keys:
//     S = Q K^T             both in shared memory, S in TMEM (128 columns)
//     P = exp2(S scale log2 e - m)      a thread a row; P, rounded to the operands' type, over the first 64 columns of S
//     O = O + P V           P from TMEM, V read by rows where it lies, O in TMEM
// with the tiles in alternation: while one tile's warps make P, the tensor core has the other tile's products.  S, P and O of both
// fill the 512 columns.  The running maximum m is only raised where a row's scores exceed it by 2^8 (then O is rescaled, in
// TMEM): P reaches 2^8 at most, and the sum is of what was made with the same m.  In fp16, P is made 2^7 larger, which keeps 7
// more bits of small shares out of its subnormal range, and stays below 2^15.
//
// Queries of up to one tile (single tokens, short sequences): both tiles take the same rows and one half of the key blocks each,
// and the first adds up both.  Longer key ranges than an SM's share come as parts (attn_join.cuh).
//
// Warps: a TMA producer, an MMA issuer, and four for each tile's rows.  The issuer zeroes V's rows behind the last key where a
// step of 16 would take them in (P is 0 there, and 0 times what another sequence left may not be).  Every wait is bounded.
//
// Measured (GB300, bf16, 32 heads on 8 of 128): 8192 tokens 365 us, 1.51 PFLOP/s of useful operations, the tensor pipe busy 69% of
// the cycles; 48 tokens on 820 to 16384 keys 250 to 254 us, 6.7 TB/s; 32 sequences of 256 45.6 us, in units of one or two steps
// whose row warps are never idle: 2700 of a unit's 9000 cycles are its softmax, 3000 its way out.  (Against the same
// kernel then: two threads a row, which agree on the maximum through shared memory in 430 cycles, 8192 tokens 420 us for 386; O stored
// by warps of their own 55 to 61 for 50.5; O's rows made whole lines through shared memory, in the place of Q 52.6 for
// 45.6, with a slot fewer 44.6, but ragged sequences 117 for 115.5.)
#include "attn_join.cuh"
#include "attn_tc.cuh"

namespace zoact {
namespace attn {

namespace {

using namespace tcx;

constexpr int THREADS = 384, REGS_FEW = 88, REGS_ROWS = 208;      // 3 x 168 as launched
static_assert(REGS_FEW + 2 * REGS_ROWS <= 3 * 168, "registers");
constexpr int TMEM_COLS = 512;
constexpr float RAISE = 8.f;

template <int DP> struct Cfg {
  static constexpr int BOXES = DP / 64, TILE_BYTES = BOXES * BOX;
  static constexpr int SLOTS = DP == 128 ? 7 : 12;
  static constexpr int SMEM = 1024 + SLOTS * TILE_BYTES;
};
static_assert(Cfg<128>::SMEM + 1024 <= 232448 && Cfg<64>::SMEM + 1024 <= 232448, "shared memory");

struct Params {
  Work work;
  Slots slots;
  float* merge;             // [SMs][TILE][TC_DIM] and statistics: the second tile's half of the keys
  float2* merge_stat;
  int* status;
  int rep, kv_heads, heads, head_dim, causal, positions;
  float scale_log2;
  void* O;
  int64_t ld_o;
  float* lse;
  int whole;                // rows of O lie on 32 bytes
};

struct Maps { CUtensorMap q, k, v; };

struct Shared {
  uint64_t full[12], empty[12], s_full[2], p_half[2], p_full[2], pv_done[2], merge_full, merge_empty;
  uint64_t join_in[2], join_out[2], drain;
  uint32_t tmem_base;
  int abort_flag, last[2];
};

// The two tiles of a unit of work.
struct Tiles {
  bool halves;              // one tile's rows, the key blocks in halves
  int n0, n1;               // blocks of each tile
  int first1, npos0, npos1; // positions of each tile; the second one's first
  int blocks;
  __device__ __forceinline__ int n(int t) const { return t ? n1 : n0; }
  __device__ __forceinline__ int pos0(int t) const { return t ? first1 : 0; }
  __device__ __forceinline__ int npos(int t) const { return t ? npos1 : npos0; }
  __device__ __forceinline__ Tiles(const Item& w, const Params& p) {
    blocks = (w.nk + BK - 1) / BK;
    halves = w.npos <= p.positions;
    if (halves) {
      first1 = 0;
      npos0 = npos1 = w.npos;
      n0 = (blocks + 1) / 2;
      n1 = blocks - n0;
    } else {
      first1 = p.positions;
      npos0 = p.positions; npos1 = w.npos - p.positions;
      n0 = (visible(w, p.causal, p.positions - 1) + BK - 1) / BK;
      n1 = (visible(w, p.causal, w.npos - 1) + BK - 1) / BK;
    }
  }
  // Loads in order: K, V of each step, of each tile in turn where they have blocks of their own.
  __device__ __forceinline__ int own() const { return blocks == 0 ? 0 : halves ? 1 : 2; }
  __device__ __forceinline__ int loads() const { return halves ? 2 * blocks : 2 * n1; }
  __device__ __forceinline__ int block(int t, int j) const { return halves && t ? n0 + j : j; }
};

// Keys of a block: products over keys run in steps of 16, with zeros behind the last one.
__device__ __forceinline__ int keys_in(const Item& w, int block) { return min(BK, w.nk - block * BK); }

template <int DP, bool BF16>
__global__ void __launch_bounds__(THREADS, 1) fwd_tc_kernel(const __grid_constant__ Maps tm, const __grid_constant__ Params p) {
  using G = Cfg<DP>;
  constexpr int SLOTS = G::SLOTS;
  extern __shared__ uint8_t smem_raw[];
  __shared__ Shared sh;
  const uint32_t smem = (tc::smem_u32(smem_raw) + 1023u) & ~1023u;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  volatile int* abort_flag = &sh.abort_flag;
  const auto bar = [](const uint64_t& b) { return tc::smem_u32(&b); };
  const auto slot = [&](uint32_t s) { return smem + s * (uint32_t)G::TILE_BYTES; };

  if (threadIdx.x == 0) {
    for (int t = 0; t < 2; ++t) {
      tc::mbar_init(bar(sh.s_full[t]), 1);
      tc::mbar_init(bar(sh.p_half[t]), 4);
      tc::mbar_init(bar(sh.p_full[t]), 4);
      tc::mbar_init(bar(sh.pv_done[t]), 1);
      tc::mbar_init(bar(sh.join_in[t]), 4);
      tc::mbar_init(bar(sh.join_out[t]), 1);
    }
    for (int s = 0; s < SLOTS; ++s) {
      tc::mbar_init(bar(sh.full[s]), 1);
      tc::mbar_init(bar(sh.empty[s]), 1);
    }
    tc::mbar_init(bar(sh.merge_full), 4);
    tc::mbar_init(bar(sh.merge_empty), 4);
    tc::mbar_init(bar(sh.drain), 1);
    sh.abort_flag = 0;
    tc::fence_mbar_init();
    tc::prefetch_tmap(&tm.q);
    tc::prefetch_tmap(&tm.k);
    tc::prefetch_tmap(&tm.v);
  }
  if (warp == 1) {
    tc::tmem_alloc(tc::smem_u32(&sh.tmem_base), TMEM_COLS);
    tc::tmem_relinquish();
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, sh.tmem_base, 0);
  pdl_wait();
  pdl_trigger();

  const int total = uniform(work_count(p.work, p.kv_heads, threadIdx.x == 0 && blockIdx.x == 0 ? p.status : nullptr));

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_FEW));
    if (warp == 0) {
      // ---------------- TMA producer ----------------
      Ring ring(SLOTS);
      bool ok = true;
      const uint32_t q_bytes = (uint32_t)(G::BOXES * p.positions * p.rep * 128);
      for (Units U(p.work, total); ok && U.here(); U.next()) {
        const Item& w = U.w;
        const int h = U.h;
        const Tiles T(w, p);
        uint32_t par, own[2] = {0, 0};
        for (int t = 0; ok && t < T.own(); ++t) {
          const uint32_t s = own[t] = ring.take(par);
          ok = warp_wait(bar(sh.empty[s]), par ^ 1u, abort_flag, p.status);
          if (ok && elect_one()) {
            tc::mbar_arrive_expect_tx(bar(sh.full[s]), q_bytes);
            for (int b = 0; b < G::BOXES; ++b)
              tma_load_4d(slot(s) + (uint32_t)(b * BOX), &tm.q, b * 64, 0, h, w.q0 + T.pos0(t), bar(sh.full[s]));
          }
          __syncwarp();
        }
        const auto load = [&](const CUtensorMap* map, int block) {
          const uint32_t s = ring.take(par);
          if (!warp_wait(bar(sh.empty[s]), par ^ 1u, abort_flag, p.status)) return false;
          if (elect_one()) {
            tc::mbar_arrive_expect_tx(bar(sh.full[s]), (uint32_t)G::TILE_BYTES);
            for (int b = 0; b < G::BOXES; ++b)
              tma_load_3d(slot(s) + (uint32_t)(b * BOX), map, b * 64, h, w.k0 + block * BK, bar(sh.full[s]));
          }
          __syncwarp();
          ring.give(s);
          return true;
        };
        const int steps = T.halves ? T.n0 : T.n1;
        for (int j = 0; ok && j < steps; ++j) {
          ok = load(&tm.k, j) && load(&tm.v, j);
          if (ok && T.halves && j < T.n1) ok = load(&tm.k, T.n0 + j) && load(&tm.v, T.n0 + j);
        }
        for (int t = 0; t < T.own(); ++t) ring.give(own[t]);
      }
      if (!ok) {                       // give our copies time to land before the CTA winds down
        const uint64_t t0 = tc::global_timer_ns();
        while (tc::global_timer_ns() - t0 < 2000000ull) {
        }
      }
    } else if (warp == 1) {
      // ---------------- MMA issuer ----------------
      const bool lead = elect_one();
      const int ksteps = (p.head_dim + 15) / 16;
      const uint32_t id_s = tc::idesc_f16(TILE, BK, BF16), id_o = tc::idesc_f16(TILE, ksteps * 16, BF16) | B_BY_ROWS;
      Ring ring(SLOTS);
      uint32_t done0 = 0, done1 = 0;               // steps of the tiles so far
      bool ok = true, any = false;
      for (Units U(p.work, total); ok && U.here(); U.next()) {
        const Item& w = U.w;
        const Tiles T(w, p);
        if (T.blocks == 0) continue;
        uint32_t par0, par1 = 0;
        const uint32_t q0 = ring.take(par0), q1 = T.halves ? q0 : ring.take(par1);
        const int len = ring.len, stride = T.halves ? 4 : 2;
        Cursor k0 = {0}, k1 = {T.halves ? 2 : 0}, v0 = {1}, v1 = {T.halves ? 3 : 1};
        const auto product_s = [&](int t, int j, Cursor& c) {
          const uint32_t s = ring.at(c.i);
          if (!warp_wait(bar(sh.full[s]), ring.parity(s) ^ c.wrapped, abort_flag, p.status)) return false;
          c.move(stride, len);
          tc::tc_fence_after();
          mma_cols<DP / 16, true>(lead, tmem + t * BK, slot(t ? q1 : q0), slot(s), id_s, ksteps);
          commit(lead, bar(sh.s_full[t]));
          if (T.halves || t == 1) commit(lead, bar(sh.empty[s]));          // else the second tile still reads it
          any = true;
          return true;
        };
        const auto product_o = [&](int t, int j, Cursor& c, uint32_t& done) {
          const uint32_t s = ring.at(c.i);
          if (!warp_wait(bar(sh.full[s]), ring.parity(s) ^ c.wrapped, abort_flag, p.status)) return false;
          c.move(stride, len);
          const int block = T.block(t, j), keys = keys_in(w, block);
          // (a tile may end before the block does: its shares are 0 there)
          const int mine = min(keys, T.halves ? BK : visible(w, p.causal, T.pos0(t) + T.npos(t) - 1) - block * BK);
          if (keys % 16 != 0 && (T.halves || t == 0 || j >= T.n0))     // once, before the first product by these rows
            zero_rows(slot(s), G::BOXES, keys, (keys + 15) / 16 * 16, lane);
          // the shares of the first 64 keys come before the others': their products run meanwhile
          if (!warp_wait(bar(sh.p_half[t]), done & 1, abort_flag, p.status)) return false;
          tc::tc_fence_after();
          mma_rows<32, true, 0, 4>(lead, tmem + (2 + t) * BK, tmem + t * BK, slot(s), id_o, (mine + 15) / 16, j != 0);
          if (!warp_wait(bar(sh.p_full[t]), done & 1, abort_flag, p.status)) return false;
          ++done;
          tc::tc_fence_after();
          mma_rows<32, true, 4, 8>(lead, tmem + (2 + t) * BK, tmem + t * BK, slot(s), id_o, (mine + 15) / 16, j != 0);
          commit(lead, bar(sh.pv_done[t]));
          if (T.halves || t == 1) commit(lead, bar(sh.empty[s]));
          return true;
        };
        // the own tiles are free once the last product by them is done
        const auto free_own = [&](uint32_t s) {
          commit(lead, bar(sh.empty[s]));
        };
        ok = warp_wait(bar(sh.full[q0]), par0, abort_flag, p.status) &&
             (T.halves || warp_wait(bar(sh.full[q1]), par1, abort_flag, p.status));
        if (ok && T.n0 > 0) ok = product_s(0, 0, k0);
        if (ok && T.n1 > 0) ok = product_s(1, 0, k1);
        const int most = max(T.n0, T.n1);
        if (ok && most == 1) {
          free_own(q0);
          if (!T.halves) free_own(q1);
        }
        for (int j = 0; ok && j < most; ++j) {
          if (j < T.n0) ok = product_o(0, j, v0, done0);
          if (ok && j + 1 < T.n0) ok = product_s(0, j + 1, k0);
          if (ok && j < T.n1) ok = product_o(1, j, v1, done1);
          if (ok && j + 1 < T.n1) ok = product_s(1, j + 1, k1);
          if (ok && j + 2 == most) {
            free_own(q0);
            if (!T.halves) free_own(q1);
          }
        }
        ring.pass(T.loads());
        ring.give(q0);
        if (!T.halves) ring.give(q1);
      }
      if (any) {
        if (elect_one()) tc::mma_commit(bar(sh.drain));
        __syncwarp();
        tc::mbar_wait_drain(bar(sh.drain), 0, 100000000ull);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_ROWS));
    // ---------------- a thread a row: P, and O at the end ----------------
    const int t = (warp - 4) >> 2, quad = warp & 3, row = quad * 32 + lane;
    const uint32_t lanes = (uint32_t)(quad * 32) << 16;
    const uint32_t ts = tmem + lanes + (uint32_t)(t * BK), to = tmem + lanes + (uint32_t)((2 + t) * BK);
    const int D = p.head_dim, pos = row / p.rep, in_group = row - pos * p.rep;
    const uint64_t scale2 = pair(p.scale_log2, p.scale_log2);
    constexpr float SHIFT = BF16 ? 0.f : 7.f;
    uint32_t steps = 0, merges = 0, joins = 0;
    bool ok = true;
    Units U(p.work, total);
    while (ok && U.here()) {
      const Item w = U.w;
      const int h = U.h;
      const Tiles T(w, p);
      const int rows = T.npos(t) * p.rep;
      const bool active = quad * 32 < rows, valid = row < rows;
      const int ipos = T.pos0(t) + pos;                                   // in the item
      const int see = valid ? visible(w, p.causal, ipos) : 0, all_see = visible(w, p.causal, T.pos0(t));
      float m = -INFINITY, l = 0.f;                                       // m: what the shares were made with
      for (int j = 0; j < T.n(t); ++j) {
        ok = warp_wait(bar(sh.s_full[t]), steps & 1, abort_flag, p.status);
        if (!ok) break;
        ++steps;
        if (active) {
          tc::tc_fence_after();
          uint32_t x[4][32];
#pragma unroll
          for (int c = 0; c < 4; ++c) ld32(ts + c * 32, x[c]);
          ld_wait();
#pragma unroll
          for (int c = 0; c < 4; ++c) ld_use(x[c]);
          const int first = T.block(t, j) * BK;
          if (all_see < first + BK) {
            const int lim = see - first;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const uint32_t seen = first_bits(lim - c * 32);
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (!(seen & 1u << i)) x[c][i] = 0xff800000u;             // -inf
            }
            __syncwarp();
          }
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int i = 0; i < 32; i += 2)
#pragma unroll
            for (int c = 0; c < 4; ++c) mx[c] = max3(mx[c], __uint_as_float(x[c][i]), __uint_as_float(x[c][i + 1]));
          const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * p.scale_log2;
          if (__any_sync(0xffffffffu, top > m + RAISE || (m == -INFINITY && top > m))) {
            const float now = fmaxf(m, top);
            if (j > 0) {
              // O holds the steps before: it is complete once the last one's product is
              const float f = m == now ? 1.f : ex2(m - now);
              ok = warp_wait(bar(sh.pv_done[t]), steps & 1, abort_flag, p.status);
              if (!ok) break;
              tc::tc_fence_after();
#pragma unroll 1
              for (int c = 0; c < D; c += 32) {
                uint32_t o[32];
                ld32(to + c, o);
                ld_wait();
                ld_use(o);
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                st32(to + c, o);
              }
              l *= f;
            }
            m = now;
          }
          const float from = (m == -INFINITY ? 0.f : m) - SHIFT;
          const uint64_t from2 = pair(-from, -from);
          uint64_t s[4] = {0, 0, 0, 0};
#pragma unroll
          for (int c = 0; c < 4; c += 2) {
            uint32_t y[32];
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
              for (int i = 0; i < 32; i += 2) {
                const uint64_t z = fma2(pair_bits(x[c + k][i], x[c + k][i + 1]), scale2, from2);
                const float a = ex2(lo(z)), b = ex2(hi(z));
                s[i / 2 & 3] = add2(s[i / 2 & 3], pair(a, b));
                y[k * 16 + i / 2] = pack2<BF16>(a, b);
              }
            st32(ts + c * 16, y);
            if (c == 0) {
              tc::tmem_wait_st();
              tc::tc_fence_before();
              __syncwarp();
              if (lane == 0) tc::mbar_arrive(bar(sh.p_half[t]));
            }
          }
          const uint64_t sum2 = add2(add2(s[0], s[1]), add2(s[2], s[3]));
          l += lo(sum2) + hi(sum2);
          tc::tmem_wait_st();
          tc::tc_fence_before();
        }
        __syncwarp();
        if (lane == 0) {
          if (!active) tc::mbar_arrive(bar(sh.p_half[t]));
          tc::mbar_arrive(bar(sh.p_full[t]));
        }
      }
      if (!ok) break;
      // ---- the unit's rows: what does not need O comes before the wait for it, the next unit's item too ----
      const float base2 = m == -INFINITY ? m : m - SHIFT;                 // log2 of the sums' unit
      const bool have = T.n(t) > 0, merging = T.halves && T.n(1) > 0, cut = w.nparts > 1;
      U.next();
      if (have && !merging && !cut) {
        const int64_t r = w.q0 + T.pos0(t) + pos;
        uint16_t* const out = static_cast<uint16_t*>(p.O) + r * p.ld_o + (int64_t)(h * p.rep + in_group) * D;
        const bool some = l != 0.f;                                       // (a row that saw nothing: 0, whatever its lane held)
        const uint32_t keep = some ? 0xffffffffu : 0u;
        const float inv = some ? 1.f / l : 0.f;
        const uint64_t inv2 = pair(inv, inv);
        if (valid && p.lse) p.lse[r * p.heads + h * p.rep + in_group] = some ? (base2 + log2f(l)) * 0.69314718f : -INFINITY;
        ok = warp_wait(bar(sh.pv_done[t]), (steps & 1) ^ 1u, abort_flag, p.status);
        if (!ok) break;
        if (active) {
          tc::tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < D; c += 64) {
            uint32_t o[2][32];
            __syncwarp();                                                 // (lanes without a row stored nothing)
            ld32(to + c, o[0]);
            ld32(to + c + 32, o[1]);
            ld_wait();
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              ld_use(o[k]);
              uint32_t y[16];
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const uint64_t z = mul2(pair_bits(o[k][2 * i], o[k][2 * i + 1]), inv2);
                y[i] = pack2<BF16>(lo(z), hi(z)) & keep;
              }
              if (valid) store_pairs(out + c + 32 * k, y, min(32, D - c - 32 * k), p.whole);
            }
          }
          tc::tc_fence_before();
        }
        continue;
      }
      if (have) {
        ok = warp_wait(bar(sh.pv_done[t]), (steps & 1) ^ 1u, abort_flag, p.status);
        if (!ok) break;
        tc::tc_fence_after();
      }
      const auto o_chunk = [&](int c, float* v) {                         // 32 columns of O (of all lanes)
        uint32_t o[32];
        __syncwarp();
        ld32(to + c, o);
        ld_wait();
        ld_use(o);
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(o[i]);
      };
      float* const mg = p.merge + ((size_t)blockIdx.x * TILE + row) * TC_DIM;
      float2* const mgs = p.merge_stat + (size_t)blockIdx.x * TILE + row;
      if (t == 1 && T.halves) {
        if (merging) {                                                    // this half goes to the first tile's warps
          ok = warp_wait(bar(sh.merge_empty), (merges & 1) ^ 1u, abort_flag, p.status);
          if (!ok) break;
          ++merges;
          if (active) {
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
              float v[32];
              o_chunk(c, v);
#pragma unroll
              for (int i = 0; i < 32; i += 4)
                if (valid && c + i < D) *reinterpret_cast<float4*>(mg + c + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
            }
            if (valid) *mgs = make_float2(base2, l);
          }
          tc::tc_fence_before();
          __threadfence_block();
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(bar(sh.merge_full));
        }
        continue;
      }
      float f0 = 1.f, f1 = 0.f, unit = base2, sum = l;                    // O = f0 mine + f1 other
      if (merging) {
        ok = warp_wait(bar(sh.merge_full), merges & 1, abort_flag, p.status);
        if (!ok) break;
        ++merges;
        if (valid) {
          const float2 other = *mgs;
          unit = fmaxf(base2, other.x);
          const float from = unit == -INFINITY ? 0.f : unit;
          f0 = ex2(base2 - from);
          f1 = ex2(other.x - from);
          sum = f0 * l + f1 * other.y;
        }
      }
      const int first_slot = w.slot + h * w.nparts, row0 = t * TILE;      // rows of a slot: the tiles' one after another
      const float inv = cut ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
      const auto out_at = [&](int r, int d) {                             // r: row of the tile
        const int ps = r / p.rep;
        return (int64_t)(w.q0 + T.pos0(t) + ps) * p.ld_o + (int64_t)(h * p.rep + r - ps * p.rep) * D + d;
      };
      const auto stat_at = [&](int r) {
        const int ps = r / p.rep;
        return (int64_t)(w.q0 + T.pos0(t) + ps) * p.heads + h * p.rep + r - ps * p.rep;
      };
      if (active) {
        uint16_t* const out = static_cast<uint16_t*>(p.O) + (valid ? out_at(row, 0) : 0);
        float* const part = slot_sums(p.slots, first_slot + w.part) + (size_t)(row0 + row) * D;
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          float v[32];
          if (have) {
            o_chunk(c, v);
          } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = 0.f;
          }
          if (merging && valid) {
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
              if (c + i < D) {
                const float4 o = *reinterpret_cast<const float4*>(mg + c + i);
                v[i] = f0 * v[i] + f1 * o.x; v[i + 1] = f0 * v[i + 1] + f1 * o.y;
                v[i + 2] = f0 * v[i + 2] + f1 * o.z; v[i + 3] = f0 * v[i + 3] + f1 * o.w;
              }
            }
          }
          if (!valid) continue;
          if (cut) {
#pragma unroll
            for (int i = 0; i < 32; i += 4)
              if (c + i < D) *reinterpret_cast<float4*>(part + c + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
          } else {
            // (a row that saw nothing: 0, whatever its lane held)
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = sum == 0.f ? 0.f : v[i] * inv;
            store_row<BF16>(out + c, v, min(32, D - c), p.whole);
          }
        }
        if (valid) {
          if (cut) slot_stat(p.slots, first_slot + w.part)[row0 + row] = make_float2(unit, sum);
          else if (p.lse) p.lse[stat_at(row)] = sum == 0.f ? -INFINITY : (unit + log2f(sum)) * 0.69314718f;
        }
      }
      tc::tc_fence_before();
      if (merging) {
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(bar(sh.merge_empty));
      }
      if (cut) {
        // the last of the row's parts adds them all up (as last_part, with bounded waits)
        unsigned* const ticket = p.slots.tickets + 4 * first_slot + t;
        __threadfence();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(bar(sh.join_in[t]));
        if (quad == 0) {
          ok = warp_wait(bar(sh.join_in[t]), joins & 1, abort_flag, p.status);
          if (!ok) break;
          if (lane == 0) {
            __threadfence();
            const bool last = atomicAdd(ticket, 1u) == (unsigned)(w.nparts - 1);
            if (last) *ticket = 0;
            __threadfence();
            sh.last[t] = last;
            tc::mbar_arrive(bar(sh.join_out[t]));
          }
        }
        ok = warp_wait(bar(sh.join_out[t]), joins & 1, abort_flag, p.status);
        if (!ok) break;
        ++joins;
        if (*(volatile int*)&sh.last[t]) {
          __threadfence();
          join_rows4(p.slots, first_slot, w.nparts, row0, rows, D, row, TILE,
                     [&](int r, int d, float4 x) {
                       *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.O) + out_at(r, d)) =
                           make_uint2(pack2<BF16>(x.x, x.y), pack2<BF16>(x.z, x.w));
                     },
                     [&](int r, float top, float s) {
                       if (p.lse) p.lse[stat_at(r)] = s == 0.f ? -INFINITY : (top + log2f(s)) * 0.69314718f;
                     });
        }
      }
    }
  }
  tc::tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    __syncwarp();
    tc::tc_fence_after();
    tc::tmem_dealloc(tmem, TMEM_COLS);
  }
}

template <int DP, bool BF16>
int run(Ctx* ctx, const Args& a) {
  Params p = {};
  const int st = slots(ctx, &p.slots);
  if (st) return st;
  p.work = work_of(a, LIST_FWD);
  p.merge = p.slots.merge;
  p.merge_stat = p.slots.merge_stat;
  p.status = ctx->d_status;
  p.rep = a.s.rep(); p.kv_heads = a.s.kv_heads; p.heads = a.s.heads; p.head_dim = a.s.head_dim; p.causal = a.s.causal;
  p.positions = tile_positions(p.rep);
  p.scale_log2 = a.scale * 1.44269504f;
  p.O = a.O; p.ld_o = a.ld_o; p.lse = a.lse;
  p.whole = ((uintptr_t)a.O & 31) == 0 && a.ld_o % 16 == 0 && a.s.head_dim % 16 == 0;
  Maps tm;
  int e = encode_rows(&tm.q, a.q, a.dtype, a.s, a.ld_q);
  if (!e) e = encode_keys(&tm.k, a.k, a.dtype, a.s, a.ld_k);
  if (!e) e = encode_keys(&tm.v, a.v, a.dtype, a.s, a.ld_v);
  if (e) return e;
  constexpr int SMEM = Cfg<DP>::SMEM;
  ZOACT_CUDA_TRY(cudaFuncSetAttribute(fwd_tc_kernel<DP, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM));
  const int64_t most = a.at.most[LIST_FWD] * a.s.kv_heads;
  ZOACT_CUDA_TRY(launch_pdl(ctx, fwd_tc_kernel<DP, BF16>, dim3((unsigned)(most < ctx->sm_count ? most : ctx->sm_count)), dim3(THREADS),
                            (size_t)SMEM, tm, p));
  ++ctx->n_launch;
  return ZOACT_OK;
}

}  // namespace

int launch_fwd_tc(Ctx* ctx, const Args& a) {
  const bool bf = a.dtype == ZOACT_DT_BF16;
  if (a.s.head_dim <= 64) return bf ? run<64, true>(ctx, a) : run<64, false>(ctx, a);
  return bf ? run<128, true>(ctx, a) : run<128, false>(ctx, a);
}

}  // namespace attn
}  // namespace zoact
