// Blackwell building blocks of the attention kernels, beside tc_common.cuh: tiles of rows of (position, head of the group) pairs
// and of keys, MMAs with the left operand in TMEM, and TMEM transfers of 32 columns that are waited for together.
//
// A tile has 128 rows of 64-column boxes (128 bytes, 128-byte swizzle), DP / 64 boxes of BOX bytes.  As a left or right operand
// of a product over the head's columns it is K-major; as the right operand of a product over its rows (P V, dS K, ...) it is read
// N-major where it lies: boxes BOX apart along N, 1024 bytes for 8 rows of K.
#pragma once
#include "attn.h"
#include "tc_common.cuh"

namespace zoact {
namespace attn {
namespace tcx {

constexpr int BOX = TILE * 128;         // bytes of 128 rows x 64 columns of 16-bit elements

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
      : "memory");
}

// Descriptors of a tile at `start` (shared memory): over its columns (K-major), over its rows (N-major).
constexpr uint32_t DESC_HI = (1024u >> 4) | 1u << 14 | 2u << 29;
__device__ __forceinline__ uint64_t desc_cols(uint32_t start) { return (uint64_t)DESC_HI << 32 | (start >> 4) | 1u << 16; }
__device__ __forceinline__ uint64_t desc_rows(uint32_t start) {
  return (uint64_t)DESC_HI << 32 | (start >> 4) | (uint32_t)(BOX >> 4) << 16;
}
constexpr uint32_t B_BY_ROWS = 1u << 16;          // instruction descriptor: the right operand is N-major

// D[tmem] (+)= A * B[smem], issued by the warp's elected lane (`lead`: a predicate, so that the warp stays together and the
// operands in uniform registers).  A in shared memory, or in TMEM: 128 lanes x 16-bit pairs, two K to a column.
__device__ __forceinline__ void mma_ss(bool lead, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"((uint32_t)lead)
      : "memory");
}
__device__ __forceinline__ void mma_ts(bool lead, uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"((uint32_t)lead)
      : "memory");
}
// Arrive on `bar` once what the elected lane issued so far has completed.
__device__ __forceinline__ void commit(bool lead, uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\t"
      "setp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar),
      "r"((uint32_t)lead)
      : "memory");
}

// A warp's own value, which the instructions of the tensor core take from uniform registers: a loop whose addresses the compiler
// did not know to be one for the whole warp took 100 cycles an MMA to issue, more than the MMA itself.
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __shfl_sync(0xffffffffu, x, 0); }

// Products of `steps` times 16 in K, at most STEPS (all arguments the warp's own).  How a call of fewer steps leaves the others out
// shows in every call's time.  EACH: every MMA by its own predicate (8192 tokens forward 363 us, the gradient of 4096 400);
// otherwise all steps in a row without a test, or a branch at each (378 to 389, 388; branches alone 377, 393).
template <bool EACH, int FIRST, int LAST, typename Step>
__device__ __forceinline__ void run_steps(bool lead, int steps, const Step& step) {
  if (!EACH && steps >= LAST) {
#pragma unroll
    for (int k = FIRST; k < LAST; ++k) step(lead, k);
  } else {
#pragma unroll
    for (int k = FIRST; k < LAST; ++k) {
      if (EACH) step(lead && k < steps, k);
      else if (k < steps) step(lead, k);
    }
  }
}
// Over columns: A and B tiles in shared memory.
template <int STEPS, bool EACH>
__device__ __forceinline__ void mma_cols(bool lead, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, int steps) {
  run_steps<EACH, 0, STEPS>(lead, steps, [&](bool go, int k) {
    const uint32_t at = (uint32_t)(k >> 2) * BOX + (uint32_t)(k & 3) * 32u;
    mma_ss(go, d, desc_cols(a + at), desc_cols(b + at), idesc, k != 0);
  });
}
// Over the rows of B (steps FIRST to LAST of them): A in TMEM, the columns of 64 K of it SECOND apart.
template <int SECOND, bool EACH, int FIRST = 0, int LAST = TILE / 16>
__device__ __forceinline__ void mma_rows(bool lead, uint32_t d, uint32_t a_tmem, uint32_t b, uint32_t idesc, int steps, uint32_t accumulate) {
  run_steps<EACH, FIRST, LAST>(lead, steps, [&](bool go, int k) {
    mma_ts(go, d, a_tmem + (uint32_t)(k >> 2) * SECOND + (uint32_t)(k & 3) * 8u, desc_rows(b + (uint32_t)k * 2048u), idesc,
           k != 0 ? 1u : accumulate);
  });
}

// The lowest n bits (n of any size): which of 32 columns are seen, tested a bit each with the instruction's own predicates.
__device__ __forceinline__ uint32_t first_bits(int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; }

__device__ __forceinline__ bool elect_one() {
  uint32_t is;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
  return is != 0;
}
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* status) {
  return __all_sync(0xffffffffu, tc::mbar_wait(bar, parity, abort_flag, status));
}

// TMEM transfers are instructions of the whole warp: where lanes had branches of their own before one, a __syncwarp() brings them
// together.  32 columns of this thread's lane; nothing reads them before ld_wait().
__device__ __forceinline__ void ld32(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// Registers of an ld32 as values from here on (after ld_wait, which this statement cannot pass).
__device__ __forceinline__ void ld_use(uint32_t* r) {
  asm volatile("" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                    "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]));
  asm volatile("" : "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]),
                    "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31]));
}
__device__ __forceinline__ void st32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
      "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
      "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
      "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void st16(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <bool BF16> __device__ __forceinline__ uint32_t pack2(float a, float b) {
  if constexpr (BF16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  } else {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
}

// Pairs of fp32 in one instruction, each half rounded as by itself.
__device__ __forceinline__ uint64_t pair(float a, float b) { return (uint64_t)__float_as_uint(b) << 32 | __float_as_uint(a); }
__device__ __forceinline__ uint64_t pair_bits(uint32_t a, uint32_t b) { return (uint64_t)b << 32 | a; }
__device__ __forceinline__ float lo(uint64_t x) { return __uint_as_float((uint32_t)x); }
__device__ __forceinline__ float hi(uint64_t x) { return __uint_as_float((uint32_t)(x >> 32)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// Slots of shared memory in the order in which they are filled next, as the producer and the issuer both count them.  A unit's own
// tiles (those that stay for all of its steps) take slots off the front and give them back behind its last load; its other
// loads go round the slots in between.  So the next unit's tiles arrive while this one's last steps run.
struct Ring {
  uint64_t order;                         // slot numbers, 4 bits each, the next one lowest
  uint32_t phase = 0;                     // bit s: parity of slot s's next filling
  int len;
  __device__ explicit Ring(int n) : order(0xba9876543210ull), len(n) {}
  __device__ __forceinline__ uint32_t at(int i) const { return (uint32_t)(order >> (4 * i)) & 15u; }
  __device__ __forceinline__ uint32_t parity(uint32_t s) const { return phase >> s & 1u; }
  // The next slot and the parity of its filling.
  __device__ __forceinline__ uint32_t take(uint32_t& par) {
    const uint32_t s = at(0);
    par = parity(s);
    phase ^= 1u << s;
    order >>= 4;
    --len;
    return s;
  }
  __device__ __forceinline__ void give(uint32_t s) {
    order = (order & ((1ull << (4 * len)) - 1)) | (uint64_t)s << (4 * len);
    ++len;
  }
  // n slots taken and given back, one after another.
  __device__ __forceinline__ void pass(int n) {
    const int rounds = n / len;
    const int rest = n - rounds * len;
    for (int i = 0; i < len; ++i)
      if ((rounds + (i < rest ? 1 : 0)) & 1) phase ^= 1u << at(i);
    const uint64_t all = (1ull << (4 * len)) - 1, o = order & all;
    order = (o >> (4 * rest) | o << (4 * (len - rest))) & all;
  }
};
// A place among a unit's loads, moved on by less than a round at a time.
struct Cursor {
  int i;
  uint32_t wrapped = 0;
  __device__ __forceinline__ void move(int n, int len) {
    i += n;
    if (i >= len) { i -= len; wrapped ^= 1u; }
  }
};

// The units of a list that a CTA runs, with the next one's item on its way.
struct Units {
  const Work* work;
  int total, round = 0, u, next_u = -1, h = 0, next_h = 0;
  Item w, next_w;
  __device__ __forceinline__ Units(const Work& wk, int n);
  __device__ __forceinline__ int unit(int r) const {
    const int x = unit_of(r, (int)blockIdx.x, (int)gridDim.x);
    return x < total ? x : -1;          // (totals are below 2^31 by more than two rounds)
  }
  __device__ __forceinline__ bool here() const { return u >= 0; }
  __device__ __forceinline__ void next();
  __device__ __forceinline__ void fetch();
};

__device__ __forceinline__ Item load_item(const Item* p) {
  const int4 a = reinterpret_cast<const int4*>(p)[0], b = reinterpret_cast<const int4*>(p)[1];
  return {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w, p->seq};
}

__device__ __forceinline__ Item uniform_item(const Item& w) {
  return {uniform(w.q0), uniform(w.npos), uniform(w.k0), uniform(w.nk), uniform(w.diag), uniform(w.part), uniform(w.nparts), uniform(w.slot),
          w.seq};
}
__device__ __forceinline__ void Units::next() {
  u = next_u;
  h = uniform(next_h);
  if (u >= 0) w = uniform_item(next_w);
  ++round;
  fetch();
}
__device__ __forceinline__ void Units::fetch() {
  next_u = u >= 0 ? unit(round + 1) : -1;
  if (next_u >= 0) next_w = load_item(work->items + work->item(next_u, next_h));
}
__device__ __forceinline__ Units::Units(const Work& wk, int n) : work(&wk), total(n) {
  u = unit(0);
  if (u >= 0) w = uniform_item(load_item(work->items + work->item(u, h)));
  h = uniform(h);
  fetch();
}

// Zero rows [from, to) of a tile of `boxes` boxes, by one warp, before the tensor core reads them.
__device__ __forceinline__ void zero_rows(uint32_t tile, int boxes, int from, int to, int lane) {
  for (int b = 0; b < boxes; ++b)
    for (int i = from * 8 + lane; i < to * 8; i += 32) tc::st_shared_v4(tile + (uint32_t)(b * BOX + i * 16), make_uint4(0, 0, 0, 0));
  tc::fence_proxy_async_smem();
  __syncwarp();
}

// Columns [0, n) of a thread's row of a 16-bit output, n a multiple of 8 up to 32; `whole`: rows lie on 32 bytes.
__device__ __forceinline__ void store_pairs(void* row, const uint32_t* y, int n, bool whole) {
#pragma unroll
  for (int j = 0; j < 16; j += 8) {
    if (2 * j >= n) break;
    char* p = static_cast<char*>(row) + 4 * j;
    const uint32_t* w = y + j;
    if (whole && 2 * j + 16 <= n) {
      asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                   "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                   : "memory");
    } else {
      *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
      if (2 * j + 16 <= n) *reinterpret_cast<uint4*>(p + 16) = make_uint4(w[4], w[5], w[6], w[7]);
    }
  }
}
template <bool BF16>
__device__ __forceinline__ void store_row(void* row, const float* x, int n, bool whole) {
  uint32_t y[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) y[i] = pack2<BF16>(x[2 * i], x[2 * i + 1]);
  store_pairs(row, y, n, whole);
}

}  // namespace tcx

// Host: the boxes of a tile: `positions` rows of 64 columns of every head of a group, and 128 rows of 64 columns of a key head.
inline int encode_rows(CUtensorMap* map, const void* base, int dtype, const Shape& s, int64_t ld) {
  return encode_tmap_heads_16bit(map, base, dtype, s.rows_q, s.heads, s.rep(), s.head_dim, ld, tile_positions(s.rep()));
}
inline int encode_keys(CUtensorMap* map, const void* base, int dtype, const Shape& s, int64_t ld) {
  return encode_tmap_heads_16bit(map, base, dtype, s.rows_k, s.kv_heads, 0, s.head_dim, ld, BK);
}

}  // namespace attn
}  // namespace zoact
