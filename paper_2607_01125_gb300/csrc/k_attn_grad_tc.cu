// The gradient of attention over packed sequences on the tensor cores (16-bit operands, heads of up to 128 columns), from the
// forward pass's log-sum-exps and delta = dO . O:
//     P = exp2(S scale log2 e - lse log2 e),  dP = dO V^T,  dS = P (dP - delta),
//     dq = scale dS K,  dk = scale dS^T Q,  dv = P^T dO.
// Two kernels make S and dP twice (7 products for 5), which leaves no sum to atomics: one has a tile of 128 rows (position, head of
// the group) and runs over the keys for dq, the other 128 keys and runs over the rows of all heads of the group for dk and dv.
// P and dS are rounded to the operands' type and stay in TMEM, over the sums that they were made of.
//
//   dq:      S twice (two steps), dP, dq in TMEM; while the row threads make dS of one step, the tensor core has dq of the step
//            before and S of the step after.
//   dk, dv:  S^T, dP^T, dk, dv in TMEM.  P^T of a step is made while dk of the step before and its dP^T run, dS^T while dv and the
//            next S^T do: the two halves of a step hide one another.
//
// 256 threads work on 128 rows (keys): two warpgroups with 64 columns each.  In fp16, P^T is made 2^10 larger, and dS by the power
// of two that brings its bound to 2^13 .. 2^15: |dS| = P |dP - sum P dP| <= 2 P (1 - P) B <= B / 2, where
// B = head_dim max|dO| max|v| of the sequence and the group of heads bounds |dP|.  Both keep small values out of the subnormal
// range and large ones finite, whatever other sequences hold, and the factors leave with the result.  Rows behind a sequence's end are zeroed in shared memory where a product would sum over them.
//
// Measured (GB300, bf16, 32 heads on 8 of 128): 4096 tokens dq 153 us (tensor pipe 58% busy), dk and dv 213 us (55%; their rows'
// statistics are read from shared memory beside the operands); 16 sequences of 256 36 and 37 us, bound by latencies.
#include "attn_join.cuh"
#include "attn_tc.cuh"

namespace zoact {
namespace attn {

namespace {

using namespace tcx;

constexpr int THREADS = 384, REGS_FEW = 104, REGS_ROWS = 200;      // 3 x 168 as launched
constexpr int TMEM_COLS = 512;

template <int DP> struct Cfg {
  static constexpr int BOXES = DP / 64, TILE_BYTES = BOXES * BOX;
  static constexpr int SLOTS = DP == 128 ? 7 : 12;
  static constexpr int TILES = SLOTS * TILE_BYTES;
  static constexpr int HALF = DP / 2;                             // columns of the results of a warpgroup
};

struct Params {
  Work work;
  Slots slots;
  int* status;
  int rep, kv_heads, heads, head_dim, causal, positions;
  float scale, scale_log2;
  const float *lse, *delta;
  const float2* largest;                                          // |dO| and |v| of each sequence and key head (fp16)
  void *dq, *dk, *dv;
  int64_t ld_dq, ld_dk, ld_dv;
  int whole_q, whole_k, whole_v;                                  // rows lie on 32 bytes
};

struct Maps { CUtensorMap q, g, k, v; };

struct Shared {
  uint64_t full[12], empty[12], s_full[2], p_full, dp_full, ds_full, acc_full, stat_full[2], stat_empty[2];
  uint64_t join_in, join_out, drain;
  uint32_t tmem_base;
  int abort_flag, last;
  uint8_t pos_of[TILE];                                           // position of a tile's row
  alignas(16) float lse[2][TILE];                                 // of a step's rows (dk, dv), read four at a time
  alignas(16) float delta[2][TILE];
};
constexpr int SHARED_BYTES = 2560 + 128;
static_assert(sizeof(Shared) <= SHARED_BYTES, "barriers and statistics");
static_assert(Cfg<128>::TILES + SHARED_BYTES <= 232448 && Cfg<64>::TILES + SHARED_BYTES <= 232448, "shared memory");

// The power of two that P^T is made larger by, as an exponent, and its inverse.
template <bool BF16> constexpr float P_SHIFT = BF16 ? 0.f : 10.f;
template <bool BF16> constexpr float P_INV = BF16 ? 1.f : 0x1p-10f;

// The largest |dO| and |v| of an item's sequence and key head.  (They lie in the plan behind its lists, where a plan that was refused
// may have no room for them: they are read for its units alone.)
template <bool BF16> __device__ __forceinline__ float2 largest_of(const Params& p, const Item& w, int h) {
  return BF16 ? make_float2(0.f, 0.f) : __ldcg(&p.largest[(int64_t)w.seq * p.kv_heads + h]);
}

// The power of two that dS is made larger by, and its inverse.
template <bool BF16> struct Factors {
  float up = 1.f, down = 1.f;
  __device__ explicit Factors(float2 largest) {
    if constexpr (!BF16) {
      // exponents of -24 to 15: B / 2 < 2^(6 + (eg + 1) + (ev + 1)), and e between -23 and 55
      const int eg = (int)(__float_as_uint(largest.x) >> 23) - 127, ev = (int)(__float_as_uint(largest.y) >> 23) - 127;
      const int e = largest.x > 0.f && largest.y > 0.f ? 7 - eg - ev : 0;
      up = __uint_as_float((uint32_t)(127 + e) << 23);
      down = __uint_as_float((uint32_t)(127 - e) << 23);
    }
  }
};

// The barriers, and each row's position.
template <int SLOTS>
__device__ __forceinline__ void init_shared(Shared* sh, int rep) {
  const auto bar = [](const uint64_t& b) { return tc::smem_u32(&b); };
  if (threadIdx.x == 0) {
    for (int s = 0; s < SLOTS; ++s) {
      tc::mbar_init(bar(sh->full[s]), 1);
      tc::mbar_init(bar(sh->empty[s]), 1);
    }
    for (int b = 0; b < 2; ++b) {
      tc::mbar_init(bar(sh->s_full[b]), 1);
      tc::mbar_init(bar(sh->stat_full[b]), 1);
      tc::mbar_init(bar(sh->stat_empty[b]), 8);
    }
    tc::mbar_init(bar(sh->p_full), 8);
    tc::mbar_init(bar(sh->dp_full), 1);
    tc::mbar_init(bar(sh->ds_full), 8);
    tc::mbar_init(bar(sh->acc_full), 1);
    tc::mbar_init(bar(sh->join_in), 8);
    tc::mbar_init(bar(sh->join_out), 1);
    tc::mbar_init(bar(sh->drain), 1);
    sh->abort_flag = 0;
    tc::fence_mbar_init();
  }
  if (threadIdx.x < TILE) sh->pos_of[threadIdx.x] = (uint8_t)(threadIdx.x / rep);
}

// Whether this row of work's last part is here: the row threads' part of last_part, with bounded waits.  ok: the waits held.
__device__ __forceinline__ bool last_of_parts(Shared* sh, unsigned* ticket, int nparts, uint32_t parity, int rwarp, int lane, int* status,
                                              bool& ok) {
  volatile int* abort_flag = &sh->abort_flag;
  __threadfence();
  __syncwarp();
  if (lane == 0) tc::mbar_arrive(tc::smem_u32(&sh->join_in));
  if (rwarp == 0) {
    ok = warp_wait(tc::smem_u32(&sh->join_in), parity, abort_flag, status);
    if (!ok) return false;
    if (lane == 0) {
      __threadfence();
      const bool last = atomicAdd(ticket, 1u) == (unsigned)(nparts - 1);
      if (last) *ticket = 0;
      __threadfence();
      sh->last = last;
      tc::mbar_arrive(tc::smem_u32(&sh->join_out));
    }
  }
  ok = warp_wait(tc::smem_u32(&sh->join_out), parity, abort_flag, status);
  if (!ok) return false;
  const bool last = *(volatile int*)&sh->last != 0;
  if (last) __threadfence();
  return last;
}

// 32 columns of a result from TMEM, times f.
__device__ __forceinline__ void acc_chunk(uint32_t taddr, float f, float* v) {
  uint32_t o[32];
  __syncwarp();                                                   // (lanes without a row stored nothing)
  ld32(taddr, o);
  ld_wait();
  ld_use(o);
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(o[i]) * f;
}
__device__ __forceinline__ void put_part(float* d, const float* v, int n) {
#pragma unroll
  for (int i = 0; i < 32; i += 4)
    if (i < n) *reinterpret_cast<float4*>(d + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
}

// A thread's half row of a result, times f, from TMEM to `out`; n: columns of it, which may be fewer than the half.
template <int HALF, bool BF16>
__device__ __forceinline__ void store_half(uint32_t taddr, float f, uint16_t* out, int n, bool valid, bool whole) {
  constexpr int PARTS = HALF / 32;
  uint32_t o[PARTS][32];
  const uint64_t f2 = pair(f, f);
  __syncwarp();
#pragma unroll
  for (int k = 0; k < PARTS; ++k) ld32(taddr + 32 * k, o[k]);
  ld_wait();
#pragma unroll
  for (int k = 0; k < PARTS; ++k) {
    ld_use(o[k]);
    uint32_t y[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint64_t z = mul2(pair_bits(o[k][2 * i], o[k][2 * i + 1]), f2);
      y[i] = pack2<BF16>(lo(z), hi(z));
    }
    if (valid) store_pairs(out + 32 * k, y, min(32, n - 32 * k), whole);
  }
}

template <int DP, bool BF16>
__global__ void __launch_bounds__(THREADS, 1) dq_tc_kernel(const __grid_constant__ Maps tm, const __grid_constant__ Params p) {
  using G = Cfg<DP>;
  constexpr int SLOTS = G::SLOTS;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  Shared* sh = reinterpret_cast<Shared*>(smem_raw + G::TILES);
  const uint32_t smem = tc::smem_u32(smem_raw);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  if (smem & 1023u) {                  // (swizzled tiles: dynamic shared memory begins there, as nothing static lies before it)
    if (threadIdx.x == 0 && blockIdx.x == 0) record_error(p.status, ZOACT_ERR_UNSUPPORTED);
    return;
  }
  volatile int* abort_flag = &sh->abort_flag;
  const auto bar = [](const uint64_t& b) { return tc::smem_u32(&b); };
  init_shared<SLOTS>(sh, p.rep);
  if (threadIdx.x == 32) {
    tc::prefetch_tmap(&tm.q);
    tc::prefetch_tmap(&tm.g);
    tc::prefetch_tmap(&tm.k);
    tc::prefetch_tmap(&tm.v);
  }
  __syncwarp();
  if (warp == 1) {
    tc::tmem_alloc(tc::smem_u32(&sh->tmem_base), TMEM_COLS);
    tc::tmem_relinquish();
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, sh->tmem_base, 0);
  const uint32_t t_s = tmem, t_dp = tmem + 2 * BK, t_dq = tmem + 3 * BK;        // S: two of BK columns
  pdl_wait();
  pdl_trigger();

  const int total = uniform(work_count(p.work, p.kv_heads, threadIdx.x == 0 && blockIdx.x == 0 ? p.status : nullptr));
  const auto slot = [&](uint32_t s) { return smem + s * (uint32_t)G::TILE_BYTES; };
  const int ksteps = (p.head_dim + 15) / 16;

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_FEW));
    if (warp == 0) {
      // ---------------- TMA producer ----------------
      Ring ring(SLOTS);
      bool ok = true;
      const uint32_t row_bytes = (uint32_t)(G::BOXES * p.positions * p.rep * 128);
      for (Units U(p.work, total); ok && U.here(); U.next()) {
        const Item& w = U.w;
        const int h = U.h, n = (w.nk + BK - 1) / BK;
        if (n == 0) continue;
        uint32_t par, own[2] = {0, 0};
        for (int t = 0; ok && t < 2; ++t) {
          const uint32_t s = own[t] = ring.take(par);
          ok = warp_wait(bar(sh->empty[s]), par ^ 1u, abort_flag, p.status);
          if (ok && elect_one()) {
            tc::mbar_arrive_expect_tx(bar(sh->full[s]), row_bytes);
            for (int b = 0; b < G::BOXES; ++b)
              tma_load_4d(slot(s) + (uint32_t)(b * BOX), t ? &tm.g : &tm.q, b * 64, 0, h, w.q0, bar(sh->full[s]));
          }
          __syncwarp();
        }
        for (int j = 0; ok && j < 2 * n; ++j) {
          const uint32_t s = ring.take(par);
          ok = warp_wait(bar(sh->empty[s]), par ^ 1u, abort_flag, p.status);
          if (!ok) break;
          if (elect_one()) {
            tc::mbar_arrive_expect_tx(bar(sh->full[s]), (uint32_t)G::TILE_BYTES);
            for (int b = 0; b < G::BOXES; ++b)
              tma_load_3d(slot(s) + (uint32_t)(b * BOX), j & 1 ? &tm.v : &tm.k, b * 64, h, w.k0 + j / 2 * BK, bar(sh->full[s]));
          }
          __syncwarp();
          ring.give(s);
        }
        ring.give(own[0]);
        ring.give(own[1]);
      }
      if (!ok) {                       // give our copies time to land before the CTA winds down
        const uint64_t t0 = tc::global_timer_ns();
        while (tc::global_timer_ns() - t0 < 2000000ull) {
        }
      }
    } else if (warp == 1) {
      // ---------------- MMA issuer ----------------
      const bool lead = elect_one();
      const uint32_t id_s = tc::idesc_f16(TILE, BK, BF16), id_q = tc::idesc_f16(TILE, ksteps * 16, BF16) | B_BY_ROWS;
      Ring ring(SLOTS);
      uint32_t step = 0;
      bool ok = true, any = false;
      for (Units U(p.work, total); ok && U.here(); U.next()) {
        const Item& w = U.w;
        const int n = (w.nk + BK - 1) / BK;
        if (n == 0) continue;
        uint32_t par_q, par_g;
        const uint32_t q_slot = ring.take(par_q), g_slot = ring.take(par_g);
        const int len = ring.len;
        Cursor ks = {0}, kq = {0}, vs = {1};         // K for S and for dq, V
        const auto product_s = [&](int j) {
          const uint32_t s = ring.at(ks.i);
          if (!warp_wait(bar(sh->full[s]), ring.parity(s) ^ ks.wrapped, abort_flag, p.status)) return false;
          ks.move(2, len);
          const int keys = min(BK, w.nk - j * BK);
          if (keys % 16 != 0) zero_rows(slot(s), G::BOXES, keys, (keys + 15) / 16 * 16, lane);
          tc::tc_fence_after();
          mma_cols<DP / 16, false>(lead, t_s + ((step + j) & 1) * BK, slot(q_slot), slot(s), id_s, ksteps);
          commit(lead, bar(sh->s_full[(step + j) & 1]));
          if (j == n - 1) commit(lead, bar(sh->empty[q_slot]));
          any = true;
          return true;
        };
        const auto product_dp = [&](int j) {
          const uint32_t s = ring.at(vs.i);
          if (!warp_wait(bar(sh->full[s]), ring.parity(s) ^ vs.wrapped, abort_flag, p.status)) return false;
          vs.move(2, len);
          tc::tc_fence_after();
          mma_cols<DP / 16, false>(lead, t_dp, slot(g_slot), slot(s), id_s, ksteps);
          commit(lead, bar(sh->dp_full));
          commit(lead, bar(sh->empty[s]));
          if (j == n - 1) commit(lead, bar(sh->empty[g_slot]));
          return true;
        };
        ok = warp_wait(bar(sh->full[q_slot]), par_q, abort_flag, p.status) && product_s(0) &&
             warp_wait(bar(sh->full[g_slot]), par_g, abort_flag, p.status) && product_dp(0) && (n < 2 || product_s(1));
        for (int j = 0; ok && j < n; ++j) {
          ok = warp_wait(bar(sh->ds_full), (step + j) & 1, abort_flag, p.status);
          if (!ok) break;
          if (j + 1 < n) ok = product_dp(j + 1);
          if (!ok) break;
          tc::tc_fence_after();
          const uint32_t s = ring.at(kq.i);
          kq.move(2, len);
          const int keys = min(BK, w.nk - j * BK);
          mma_rows<64, false>(lead, t_dq, t_s + ((step + j) & 1) * BK, slot(s), id_q, (keys + 15) / 16, j != 0);
          commit(lead, bar(sh->empty[s]));
          if (j == n - 1) commit(lead, bar(sh->acc_full));
          if (j + 2 < n) ok = product_s(j + 2);
        }
        ring.pass(2 * n);
        ring.give(q_slot);
        ring.give(g_slot);
        step += n;
      }
      if (any) {
        if (elect_one()) tc::mma_commit(bar(sh->drain));
        __syncwarp();
        tc::mbar_wait_drain(bar(sh->drain), 0, 100000000ull);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_ROWS));
    // ---------------- a thread half a row: dS, and dq at the end ----------------
    const int half = (warp - 4) >> 2, quad = warp & 3, row = quad * 32 + lane, rwarp = warp - 4;
    const uint32_t lanes = (uint32_t)(quad * 32) << 16;
    const int D = p.head_dim, pos = row / p.rep, in_group = row - pos * p.rep;
    const uint64_t scale2 = pair(p.scale_log2, p.scale_log2);
    uint32_t step = 0, units = 0, joins = 0;
    bool ok = true;
    // of this thread's row of an item: log-sum-exp and delta
    const auto stat_of = [&](const Item& w, int h, float& lse, float& delta) {
      lse = delta = 0.f;
      if (row >= w.npos * p.rep) return;
      const int64_t e = (int64_t)(w.q0 + pos) * p.heads + h * p.rep + in_group;
      lse = p.lse[e];
      delta = p.delta[e];
    };
    Units U(p.work, total);
    float lse_next = 0.f, delta_next = 0.f;
    float2 largest_next = make_float2(0.f, 0.f);
    if (U.here()) {
      stat_of(U.w, U.h, lse_next, delta_next);
      largest_next = largest_of<BF16>(p, U.w, U.h);
    }
    while (ok && U.here()) {
      const Item w = U.w;
      const int h = U.h, n = (w.nk + BK - 1) / BK, rows = w.npos * p.rep;
      const bool active = quad * 32 < rows, valid = row < rows;
      const int see = valid ? visible<int>(w, p.causal, pos) : 0, all_see = visible<int>(w, p.causal, 0);
      const float base = share_base(lse_next);
      const uint64_t base2 = pair(base, base), delta2 = pair(-delta_next, -delta_next);
      const Factors<BF16> f(largest_next);
      const uint64_t ds2 = pair(f.up, f.up);
      for (int j = 0; j < n; ++j, ++step) {
        ok = warp_wait(bar(sh->s_full[step & 1]), step >> 1 & 1, abort_flag, p.status);
        if (!ok) break;
        const uint32_t s0 = t_s + (step & 1) * BK + lanes + half * 64, d0 = t_dp + lanes + half * 64;
        const int lim = see - j * BK - half * 64;                         // columns of this half that are seen
        const bool masked = all_see < (j + 1) * BK;
        uint64_t pr[32];
        if (active) {
          // P while the tensor core has this step's dP
          tc::tc_fence_after();
          uint32_t x[2][32];
          ld32(s0, x[0]);
          ld32(s0 + 32, x[1]);
          ld_wait();
          ld_use(x[0]);
          ld_use(x[1]);
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              const uint64_t z = fma2(pair_bits(x[c][i], x[c][i + 1]), scale2, base2);
              pr[c * 16 + i / 2] = pair(ex2(lo(z)), ex2(hi(z)));
            }
        }
        ok = warp_wait(bar(sh->dp_full), step & 1, abort_flag, p.status);
        if (!ok) break;
        if (active) {
          tc::tc_fence_after();
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint32_t d[32], y[16];
            ld32(d0 + c * 32, d);
            ld_wait();
            ld_use(d);
            if (masked) {                                                 // 0, whatever the sums are
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const int col = c * 32 + 2 * i;
                if (col >= lim) { pr[c * 16 + i] = 0; d[2 * i] = 0; }
                if (col + 1 >= lim) { pr[c * 16 + i] &= 0xffffffffull; d[2 * i + 1] = 0; }
              }
              __syncwarp();
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              uint64_t v = mul2(pr[c * 16 + i], add2(pair_bits(d[2 * i], d[2 * i + 1]), delta2));
              if (!BF16) v = mul2(v, ds2);
              y[i] = pack2<BF16>(lo(v), hi(v));
            }
            st16(s0 + c * 16, y);
          }
          tc::tmem_wait_st();
          tc::tc_fence_before();
        }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(bar(sh->ds_full));
      }
      if (!ok) break;
      // (the next unit's item and statistics are on their way before the wait for dq)
      U.next();
      if (U.here()) {
        stat_of(U.w, U.h, lse_next, delta_next);
        largest_next = largest_of<BF16>(p, U.w, U.h);
      }
      const float out_f = p.scale * f.down;
      const bool cut = w.nparts > 1;
      uint16_t* const dq = static_cast<uint16_t*>(p.dq);
      uint16_t* const out = dq + (int64_t)(w.q0 + pos) * p.ld_dq + (int64_t)(h * p.rep + in_group) * D;
      if (n > 0) {
        ok = warp_wait(bar(sh->acc_full), units & 1, abort_flag, p.status);
        if (!ok) break;
        ++units;
        tc::tc_fence_after();
        if (!cut) {
          const int c = half * G::HALF;
          if (active) store_half<G::HALF, BF16>(t_dq + lanes + c, out_f, out + c, D - c, valid, p.whole_q);
          tc::tc_fence_before();
          continue;
        }
      }
      const int first = w.slot + h * w.nparts;
      if (active) {
#pragma unroll 1
        for (int c = half * G::HALF; c < min(D, (half + 1) * G::HALF); c += 32) {
          float v[32];
          if (n > 0) {
            acc_chunk(t_dq + lanes + c, out_f, v);
          } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = 0.f;
          }
          if (!valid) continue;
          if (cut) put_part(slot_sums(p.slots, first + w.part) + (size_t)row * D + c, v, D - c);
          else store_row<BF16>(out + c, v, min(32, D - c), p.whole_q);
        }
      }
      tc::tc_fence_before();
      if (cut) {
        const bool last = last_of_parts(sh, p.slots.tickets + 4 * first, w.nparts, joins & 1, rwarp, lane, p.status, ok);
        if (!ok) break;
        ++joins;
        if (last) {
          join_sums4(p.slots, first, w.nparts, 0, rows * D / 4, rwarp * 32 + lane, 256, [&](int e, float4 v) {
            const int rr = e * 4 / D, ps = rr / p.rep;
            *reinterpret_cast<uint2*>(dq + (int64_t)(w.q0 + ps) * p.ld_dq + (int64_t)(h * p.rep + rr - ps * p.rep) * D + (e * 4 - rr * D)) =
                make_uint2(pack2<BF16>(v.x, v.y), pack2<BF16>(v.z, v.w));
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
__global__ void __launch_bounds__(THREADS, 1) dkv_tc_kernel(const __grid_constant__ Maps tm, const __grid_constant__ Params p) {
  using G = Cfg<DP>;
  constexpr int SLOTS = G::SLOTS;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  Shared* sh = reinterpret_cast<Shared*>(smem_raw + G::TILES);
  const uint32_t smem = tc::smem_u32(smem_raw);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  if (smem & 1023u) {                  // (swizzled tiles: dynamic shared memory begins there, as nothing static lies before it)
    if (threadIdx.x == 0 && blockIdx.x == 0) record_error(p.status, ZOACT_ERR_UNSUPPORTED);
    return;
  }
  volatile int* abort_flag = &sh->abort_flag;
  const auto bar = [](const uint64_t& b) { return tc::smem_u32(&b); };
  init_shared<SLOTS>(sh, p.rep);
  if (threadIdx.x == 32) {
    tc::prefetch_tmap(&tm.q);
    tc::prefetch_tmap(&tm.g);
    tc::prefetch_tmap(&tm.k);
    tc::prefetch_tmap(&tm.v);
  }
  __syncwarp();
  if (warp == 1) {
    tc::tmem_alloc(tc::smem_u32(&sh->tmem_base), TMEM_COLS);
    tc::tmem_relinquish();
  }
  tc::tc_fence_before();
  __syncthreads();
  tc::tc_fence_after();
  const uint32_t tmem = __shfl_sync(0xffffffffu, sh->tmem_base, 0);
  const uint32_t t_s = tmem, t_dp = tmem + BK, t_dv = tmem + 2 * BK, t_dk = tmem + 3 * BK;
  pdl_wait();
  pdl_trigger();

  const int total = uniform(work_count(p.work, p.kv_heads, threadIdx.x == 0 && blockIdx.x == 0 ? p.status : nullptr));
  const auto slot = [&](uint32_t s) { return smem + s * (uint32_t)G::TILE_BYTES; };
  const int P = p.positions;
  const int ksteps = (p.head_dim + 15) / 16;

  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_FEW));
    if (warp == 0) {
      // ---------------- TMA producer ----------------
      Ring ring(SLOTS);
      bool ok = true;
      const uint32_t row_bytes = (uint32_t)(G::BOXES * P * p.rep * 128);
      for (Units U(p.work, total); ok && U.here(); U.next()) {
        const Item& w = U.w;
        const int h = U.h, n = (w.npos + P - 1) / P;
        if (n == 0) continue;
        uint32_t par, own[2] = {0, 0};
        for (int t = 0; ok && t < 2; ++t) {
          const uint32_t s = own[t] = ring.take(par);
          ok = warp_wait(bar(sh->empty[s]), par ^ 1u, abort_flag, p.status);
          if (ok && elect_one()) {
            tc::mbar_arrive_expect_tx(bar(sh->full[s]), (uint32_t)G::TILE_BYTES);
            for (int b = 0; b < G::BOXES; ++b)
              tma_load_3d(slot(s) + (uint32_t)(b * BOX), t ? &tm.v : &tm.k, b * 64, h, w.k0, bar(sh->full[s]));
          }
          __syncwarp();
        }
        for (int j = 0; ok && j < 2 * n; ++j) {
          const uint32_t s = ring.take(par);
          ok = warp_wait(bar(sh->empty[s]), par ^ 1u, abort_flag, p.status);
          if (!ok) break;
          if (elect_one()) {
            tc::mbar_arrive_expect_tx(bar(sh->full[s]), row_bytes);
            for (int b = 0; b < G::BOXES; ++b)
              tma_load_4d(slot(s) + (uint32_t)(b * BOX), j & 1 ? &tm.g : &tm.q, b * 64, 0, h, w.q0 + j / 2 * P, bar(sh->full[s]));
          }
          __syncwarp();
          ring.give(s);
        }
        ring.give(own[0]);
        ring.give(own[1]);
      }
      if (!ok) {                       // give our copies time to land before the CTA winds down
        const uint64_t t0 = tc::global_timer_ns();
        while (tc::global_timer_ns() - t0 < 2000000ull) {
        }
      }
    } else if (warp == 1) {
      // ---------------- MMA issuer ----------------
      const bool lead = elect_one();
      const uint32_t id_d = tc::idesc_f16(BK, ksteps * 16, BF16) | B_BY_ROWS;
      Ring ring(SLOTS);
      uint32_t step = 0;
      bool ok = true, any = false;
      for (Units U(p.work, total); ok && U.here(); U.next()) {
        const Item& w = U.w;
        const int n = (w.npos + P - 1) / P;
        if (n == 0) continue;
        uint32_t par_k, par_v;
        const uint32_t k_slot = ring.take(par_k), v_slot = ring.take(par_v);
        const int len = ring.len;
        Cursor c1[2] = {{0}, {1}}, c2[2] = {{0}, {1}};       // Q and dO: for the products over columns, and over rows
        const auto rows_of = [&](int i) { return min(P, w.npos - i * P) * p.rep; };
        // S^T (G = 0: K by Q) or dP^T (1: V by dO) of step i, as wide as the step has rows
        const auto product = [&](int g, int i, Cursor& c) {
          const uint32_t s = ring.at(c.i);
          if (!warp_wait(bar(sh->full[s]), ring.parity(s) ^ c.wrapped, abort_flag, p.status)) return false;
          c.move(2, len);
          const int rows = rows_of(i), up = (rows + 15) / 16 * 16;
          if (rows != up) zero_rows(slot(s), G::BOXES, rows, up, lane);
          tc::tc_fence_after();
          const uint32_t own = g ? v_slot : k_slot;
          mma_cols<DP / 16, false>(lead, g ? t_dp : t_s, slot(own), slot(s), tc::idesc_f16(BK, up, BF16), ksteps);
          commit(lead, g ? bar(sh->dp_full) : bar(sh->s_full[0]));
          if (i == n - 1) commit(lead, bar(sh->empty[own]));
          any = true;
          return true;
        };
        // dv += P^T dO (g = 1) or dk += dS^T Q (0)
        const auto sum = [&](int g, int i, Cursor& c) {
          const uint32_t s = ring.at(c.i);
          c.move(2, len);
          tc::tc_fence_after();
          mma_rows<64, false>(lead, g ? t_dv : t_dk, g ? t_s : t_dp, slot(s), id_d, (rows_of(i) + 15) / 16, i != 0);
          commit(lead, bar(sh->empty[s]));
          if (!g && i == n - 1) commit(lead, bar(sh->acc_full));
        };
        ok = warp_wait(bar(sh->full[k_slot]), par_k, abort_flag, p.status) && product(0, 0, c1[0]) &&
             warp_wait(bar(sh->full[v_slot]), par_v, abort_flag, p.status) && product(1, 0, c1[1]);
        for (int i = 0; ok && i < n; ++i) {
          ok = warp_wait(bar(sh->p_full), (step + i) & 1, abort_flag, p.status);
          if (!ok) break;
          sum(1, i, c2[1]);
          if (i + 1 < n) ok = product(0, i + 1, c1[0]);
          if (!ok) break;
          ok = warp_wait(bar(sh->ds_full), (step + i) & 1, abort_flag, p.status);
          if (!ok) break;
          sum(0, i, c2[0]);
          if (i + 1 < n) ok = product(1, i + 1, c1[1]);
        }
        ring.pass(2 * n);
        ring.give(k_slot);
        ring.give(v_slot);
        step += n;
      }
      if (any) {
        if (elect_one()) tc::mma_commit(bar(sh->drain));
        __syncwarp();
        tc::mbar_wait_drain(bar(sh->drain), 0, 100000000ull);
      }
    } else if (warp == 2) {
      // ---------------- the rows' statistics, two steps ahead ----------------
      uint32_t step = 0;
      bool ok = true;
      for (Units U(p.work, total); ok && U.here(); U.next()) {
        const Item& w = U.w;
        const int h = U.h, n = (w.npos + P - 1) / P;
        for (int i = 0; i < n; ++i, ++step) {
          const int b = step & 1, rows = min(P, w.npos - i * P) * p.rep;
          float lse[4], delta[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int row = lane + 32 * k, pos = sh->pos_of[row];
            const int64_t e = (int64_t)(w.q0 + i * P + pos) * p.heads + h * p.rep + row - pos * p.rep;
            // (rows behind the last: no share)
            lse[k] = row < rows ? P_SHIFT<BF16> + share_base(p.lse[e]) : -INFINITY;
            delta[k] = row < rows ? -p.delta[e] : 0.f;
          }
          ok = warp_wait(bar(sh->stat_empty[b]), (step >> 1 & 1) ^ 1u, abort_flag, p.status);
          if (!ok) break;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            sh->lse[b][lane + 32 * k] = lse[k];
            sh->delta[b][lane + 32 * k] = delta[k];
          }
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(bar(sh->stat_full[b]));
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_ROWS));
    // ---------------- a thread half of a key's rows: P^T and dS^T, dk and dv at the end ----------------
    const int half = (warp - 4) >> 2, quad = warp & 3, key = quad * 32 + lane, rwarp = warp - 4;
    const uint32_t lanes = (uint32_t)(quad * 32) << 16;
    const int D = p.head_dim;
    const uint64_t scale2 = pair(p.scale_log2, p.scale_log2);
    uint32_t step = 0, units = 0, joins = 0;
    bool ok = true;
    Units U(p.work, total);
    float2 largest_next = U.here() ? largest_of<BF16>(p, U.w, U.h) : make_float2(0.f, 0.f);
    while (ok && U.here()) {
      const Item w = U.w;
      const int h = U.h, n = (w.npos + P - 1) / P;
      const Factors<BF16> f(largest_next);
      const float up = f.up * P_INV<BF16>;                        // of dS from P^T as made
      const uint64_t ds2 = pair(up, up);
      const bool active = quad * 32 < w.nk, valid = key < w.nk;
      for (int i = 0; i < n; ++i, ++step) {
        const int b = step & 1;
        ok = warp_wait(bar(sh->stat_full[b]), step >> 1 & 1, abort_flag, p.status);
        if (!ok) break;
        uint64_t pr[32], st[32];
        const uint32_t s0 = t_s + lanes + half * 64, d0 = t_dp + lanes + half * 64;
        // the rows' statistics (negative, in pairs) come before the sums that they go with: a read of shared memory waits behind
        // the operands of the tensor core
        const ulonglong2* const lse = reinterpret_cast<const ulonglong2*>(&sh->lse[b][half * 64]);
        const ulonglong2* const delta = reinterpret_cast<const ulonglong2*>(&sh->delta[b][half * 64]);
#pragma unroll
        for (int q = 0; q < 16; ++q) {
          const ulonglong2 l = lse[q];
          st[2 * q] = l.x;
          st[2 * q + 1] = l.y;
        }
        ok = warp_wait(bar(sh->s_full[0]), step & 1, abort_flag, p.status);
        if (!ok) break;
        const bool masked = visible<int>(w, p.causal, i * P) < w.nk;
        if (active) {
          tc::tc_fence_after();
          uint32_t x[2][32];
          ld32(s0, x[0]);
          ld32(s0 + 32, x[1]);
          ld_wait();
          ld_use(x[0]);
          ld_use(x[1]);
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint32_t y[16];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              const uint64_t z0 = fma2(pair_bits(x[c][4 * q], x[c][4 * q + 1]), scale2, st[c * 16 + 2 * q]);
              const uint64_t z1 = fma2(pair_bits(x[c][4 * q + 2], x[c][4 * q + 3]), scale2, st[c * 16 + 2 * q + 1]);
              pr[c * 16 + 2 * q] = pair(ex2(lo(z0)), ex2(hi(z0)));
              pr[c * 16 + 2 * q + 1] = pair(ex2(lo(z1)), ex2(hi(z1)));
            }
            if (masked) {
              // a row at position x of the step sees this key from x = `from` on
              const int from = key + 1 - w.diag - i * P;
#pragma unroll
              for (int k = 0; k < 16; ++k) {
                const int col = half * 64 + c * 32 + 2 * k;
                if ((int)sh->pos_of[col] < from) pr[c * 16 + k] &= ~0xffffffffull;
                if ((int)sh->pos_of[col + 1] < from) pr[c * 16 + k] &= 0xffffffffull;
              }
              __syncwarp();
            }
#pragma unroll
            for (int k = 0; k < 16; ++k) y[k] = pack2<BF16>(lo(pr[c * 16 + k]), hi(pr[c * 16 + k]));
            st16(s0 + c * 16, y);
          }
          tc::tmem_wait_st();
          tc::tc_fence_before();
        }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(bar(sh->p_full));
#pragma unroll
        for (int q = 0; q < 16; ++q) {
          const ulonglong2 d = delta[q];
          st[2 * q] = d.x;
          st[2 * q + 1] = d.y;
        }
        ok = warp_wait(bar(sh->dp_full), step & 1, abort_flag, p.status);
        if (!ok) break;
        if (active) {
          tc::tc_fence_after();
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint32_t x[32], y[16];
            ld32(d0 + c * 32, x);
            ld_wait();
            ld_use(x);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              uint64_t v0 = mul2(pr[c * 16 + 2 * q], add2(pair_bits(x[4 * q], x[4 * q + 1]), st[c * 16 + 2 * q]));
              uint64_t v1 = mul2(pr[c * 16 + 2 * q + 1], add2(pair_bits(x[4 * q + 2], x[4 * q + 3]), st[c * 16 + 2 * q + 1]));
              if (!BF16) {
                v0 = mul2(v0, ds2);
                v1 = mul2(v1, ds2);
              }
              y[2 * q] = pack2<BF16>(lo(v0), hi(v0));
              y[2 * q + 1] = pack2<BF16>(lo(v1), hi(v1));
            }
            st16(d0 + c * 16, y);
          }
          tc::tmem_wait_st();
          tc::tc_fence_before();
        }
        __syncwarp();
        if (lane == 0) {
          tc::mbar_arrive(bar(sh->ds_full));
          tc::mbar_arrive(bar(sh->stat_empty[b]));
        }
      }
      if (!ok) break;
      U.next();
      if (U.here()) largest_next = largest_of<BF16>(p, U.w, U.h);
      const float fk = p.scale * f.down, fv = P_INV<BF16>;
      const bool cut = w.nparts > 1;
      uint16_t* const dk = static_cast<uint16_t*>(p.dk) + (int64_t)w.k0 * p.ld_dk + (int64_t)h * D;
      uint16_t* const dv = static_cast<uint16_t*>(p.dv) + (int64_t)w.k0 * p.ld_dv + (int64_t)h * D;
      if (n > 0) {
        const int c = half * G::HALF;
        uint16_t *const to_k = dk + (int64_t)key * p.ld_dk + c, *const to_v = dv + (int64_t)key * p.ld_dv + c;
        ok = warp_wait(bar(sh->acc_full), units & 1, abort_flag, p.status);
        if (!ok) break;
        ++units;
        tc::tc_fence_after();
        if (!cut) {
          if (active) {
            store_half<G::HALF, BF16>(t_dv + lanes + c, fv, to_v, D - c, valid, p.whole_v);
            store_half<G::HALF, BF16>(t_dk + lanes + c, fk, to_k, D - c, valid, p.whole_k);
          }
          tc::tc_fence_before();
          continue;
        }
      }
      const int first = w.slot + h * w.nparts;
      if (active) {
#pragma unroll 1
        for (int c = half * G::HALF; c < min(D, (half + 1) * G::HALF); c += 32) {
          float v[32];
#pragma unroll
          for (int which = 0; which < 2; ++which) {
            if (n > 0) {
              acc_chunk((which ? t_dv : t_dk) + lanes + c, which ? fv : fk, v);
            } else {
#pragma unroll
              for (int i = 0; i < 32; ++i) v[i] = 0.f;
            }
            if (!valid) continue;
            if (cut) put_part(slot_sums(p.slots, first + w.part) + (size_t)(which * BK + key) * D + c, v, D - c);
            else if (which) store_row<BF16>(dv + (int64_t)key * p.ld_dv + c, v, min(32, D - c), p.whole_v);
            else store_row<BF16>(dk + (int64_t)key * p.ld_dk + c, v, min(32, D - c), p.whole_k);
          }
        }
      }
      tc::tc_fence_before();
      if (cut) {
        const bool last = last_of_parts(sh, p.slots.tickets + 4 * first, w.nparts, joins & 1, rwarp, lane, p.status, ok);
        if (!ok) break;
        ++joins;
        if (last) {
          for (int which = 0; which < 2; ++which)
            join_sums4(p.slots, first, w.nparts, (size_t)(which * BK) * D, w.nk * D / 4, rwarp * 32 + lane, 256, [&](int e, float4 v) {
              const int kk = e * 4 / D, d = e * 4 - kk * D;
              *reinterpret_cast<uint2*>(which ? dv + (int64_t)kk * p.ld_dv + d : dk + (int64_t)kk * p.ld_dk + d) =
                  make_uint2(pack2<BF16>(v.x, v.y), pack2<BF16>(v.z, v.w));
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
  p.status = ctx->d_status;
  p.rep = a.s.rep(); p.kv_heads = a.s.kv_heads; p.heads = a.s.heads; p.head_dim = a.s.head_dim; p.causal = a.s.causal;
  p.positions = tile_positions(p.rep);
  p.scale = a.scale; p.scale_log2 = a.scale * 1.44269504f;
  p.lse = a.lse; p.delta = a.delta; p.largest = a.largest;
  p.dq = a.dq; p.dk = a.dk; p.dv = a.dv; p.ld_dq = a.ld_dq; p.ld_dk = a.ld_dk; p.ld_dv = a.ld_dv;
  const auto whole = [&](const void* q, int64_t ld) { return ((uintptr_t)q & 31) == 0 && ld % 16 == 0 && a.s.head_dim % 16 == 0; };
  p.whole_q = whole(a.dq, a.ld_dq); p.whole_k = whole(a.dk, a.ld_dk); p.whole_v = whole(a.dv, a.ld_dv);
  Maps tm;
  int e = encode_rows(&tm.q, a.q, a.dtype, a.s, a.ld_q);
  if (!e) e = encode_rows(&tm.g, a.dO, a.dtype, a.s, a.ld_do);
  if (!e) e = encode_keys(&tm.k, a.k, a.dtype, a.s, a.ld_k);
  if (!e) e = encode_keys(&tm.v, a.v, a.dtype, a.s, a.ld_v);
  if (e) return e;
  constexpr int SMEM = Cfg<DP>::TILES + SHARED_BYTES;
  for (int list : {LIST_DQ, LIST_DKV}) {
    auto kern = list == LIST_DQ ? dq_tc_kernel<DP, BF16> : dkv_tc_kernel<DP, BF16>;
    p.work = work_of(a, list);
    ZOACT_CUDA_TRY(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM));
    const int64_t most = a.at.most[list] * a.s.kv_heads;
    ZOACT_CUDA_TRY(launch_pdl(ctx, kern, dim3((unsigned)(most < ctx->sm_count ? most : ctx->sm_count)), dim3(THREADS), (size_t)SMEM,
                              tm, p));
    ++ctx->n_launch;
  }
  return ZOACT_OK;
}

}  // namespace

int launch_grad_tc(Ctx* ctx, const Args& a) {
  const bool bf = a.dtype == ZOACT_DT_BF16;
  if (a.s.head_dim <= 64) return bf ? run<64, true>(ctx, a) : run<64, false>(ctx, a);
  return bf ? run<128, true>(ctx, a) : run<128, false>(ctx, a);
}

}  // namespace attn
}  // namespace zoact
