// Attention over packed sequences: what its kernels share.
#pragma once
#include "internal.h"

namespace zoact {
namespace attn {

constexpr int BK = 128;                 // keys of a block of work
constexpr int TILE = 128;               // rows of a tile: (position, head of the group) pairs, the group fastest
constexpr int MAX_REP = 128;            // query heads of a group at most
constexpr int MAX_DIM = 256, TC_DIM = 128;
constexpr int SPLIT_OVER = 2;           // pieces of work an SM that long rows of work are cut for, at most

// A rectangle of work: positions [q0, q0 + npos) against keys [k0, k0 + nk); position i sees the first visible(i) of them.
// A row of work (positions of a forward or dq tile, keys of a dk / dv tile) that is cut into nparts leaves each part's sums in
// a slot: part p of key head h in slot + h nparts + p.
struct alignas(16) Item {
  int32_t q0, npos, k0, nk, diag, part, nparts, slot;
  int32_t seq;                          // the sequence that the work is of
};
// (With part and nparts as two 16-bit fields, in 32 bytes, the kernel for dq joined its parts to zeros; no reason for it was found in
// the source.)
static_assert(sizeof(Item) == 48, "items are read as two 16-byte words, and the sequence where it is needed");

// (rows are below 2^31 - 2^16, and 32 bits suffice; the long prompt of the forward kernel took 389 us with them for 363, the
// gradient's short sequences 89.0 for 91.2)
template <typename Wide = int64_t>
__device__ __forceinline__ int visible(const Item& w, int causal, int i) {
  if (!causal) return w.nk;
  const Wide v = (Wide)w.diag + i;
  return v < 0 ? 0 : v > w.nk ? w.nk : (int)v;
}

// What the gradient adds to a row's scores (times log2 e) for its shares: the log-sum-exp, negative.  A row without any share, whose
// scores may all be -infinity, has none here either.
__device__ __forceinline__ float share_base(float lse) { return lse == -INFINITY ? -INFINITY : -lse * 1.44269504f; }

// Positions of a tile.
__host__ __device__ inline int tile_positions(int rep) { return TILE / rep; }

enum List { LIST_FWD = 0, LIST_DQ, LIST_DKV, LISTS };

constexpr int HAS_FWD = 1, HAS_GRAD = 2;

// The head of a plan; the lists of items follow.
struct Head {
  uint64_t tag;                         // the shape and the number of SMs that the plan is for
  int32_t count[LISTS];
  int32_t has;                          // HAS_FWD, HAS_GRAD; 0: the spans were refused
};

struct Shape {
  int64_t rows_q, rows_k;
  int n_seq, heads, kv_heads, head_dim, causal;
  int rep() const { return heads / kv_heads; }
};

// Where the parts of a plan lie (bytes).
struct Layout {
  size_t seqs, prefix, items[LISTS], delta, largest, total;
  int64_t most[LISTS];                  // items a list can have
};
Layout plan_layout(const Shape& s, int sm_count, int grad);
uint64_t plan_tag(const Shape& s, int sm_count);
inline int slot_count(int sm_count) { return 2 * SPLIT_OVER * sm_count; }

// Scratch of rows of work that are cut: fixed sizes, so that no later call moves what a captured graph uses.
struct Slots {
  float* sums;                          // [slots][2 TILE][TC_DIM]
  float2* stat;                         // [slots][2 TILE]: maximum (times scale log2 e) and sum of exponentials
  unsigned* tickets;                    // [slots][4], zero between launches
  float* merge;                         // [SMs][TILE][TC_DIM]: a tile's half of the keys (forward)
  float2* merge_stat;                   // [SMs][TILE]
};
int slots(Ctx* ctx, Slots* s);

struct Args {
  Shape s;
  const uint8_t* plan;
  Layout at;
  uint64_t tag;
  const void *q, *k, *v;
  int64_t ld_q, ld_k, ld_v;
  int dtype;
  float scale;
  void* O;
  int64_t ld_o;
  float* lse;                           // [rows_q, heads] or nullptr
  // gradient
  const void* dO;
  int64_t ld_do;
  void *dq, *dk, *dv;
  int64_t ld_dq, ld_dk, ld_dv;
  float* delta;                         // [rows_q, heads], in the plan
  float2* largest;                      // [n_seq, kv_heads]: |dO| of a group's heads and |v| (fp16), in the plan
};

// What a kernel needs of a list.
struct Work {
  const Head* head;
  const Item* items;
  uint64_t tag;
  int list, kv_heads;
  // Unit u is item u / kv_heads of key head u % kv_heads.  (With the quotient from a product the forward kernel's long prompt took
  // 401 us for 387.)
  __device__ __forceinline__ int item(int u, int& head_of) const {
    head_of = u % kv_heads;
    return u / kv_heads;
  }
};
inline Work work_of(const Args& a, int list) {
  return {reinterpret_cast<const Head*>(a.plan), reinterpret_cast<const Item*>(a.plan + a.at.items[list]), a.tag, list, a.s.kv_heads};
}
// Items times key heads, or 0 (and the status word) where the plan is not one for this call.
__device__ __forceinline__ int work_count(const Work& w, int kv_heads, int* status) {
  const Head* h = w.head;
  const int need = w.list == LIST_FWD ? HAS_FWD : HAS_GRAD;
  if (h->tag != w.tag || !(h->has & need)) {
    if (h->tag != w.tag || h->has != 0) record_error(status, ZOACT_ERR_INVALID_ARG);
    return 0;
  }
  return h->count[w.list] * kv_heads;
}
// Unit u of block c of n: every other round runs backwards, so that a block's shares of a list sorted by size even out.
__device__ __forceinline__ int unit_of(int round, int c, int n) { return round * n + (round & 1 ? n - 1 - c : c); }

bool tc_supported(const Args& a, bool grad);
int launch_fwd_simt(Ctx* ctx, const Args& a);
int launch_grad_simt(Ctx* ctx, const Args& a);
int launch_fwd_tc(Ctx* ctx, const Args& a);
int launch_grad_tc(Ctx* ctx, const Args& a);
int launch_delta(Ctx* ctx, const Args& a);
int launch_plan(Ctx* ctx, const Shape& s, const void* spans, int id64, uint8_t* plan, int grad);

}  // namespace attn
}  // namespace zoact
