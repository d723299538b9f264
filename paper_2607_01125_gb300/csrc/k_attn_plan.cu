// The plan of attention over packed sequences: from the sequences' spans (rows of queries, rows of keys) the lists of work that
// the kernels run through, largest first.  It is made once for a batch and read by every layer, forward and gradient.
//
// One block: it checks the spans, counts every sequence's rows of work, adds up their sizes, and writes the items in order of
// size (a counting sort).  A row of work larger than its share of the GPU (split_over) is cut along its long
// axis; the parts' sums are joined by the last of them to finish, in the order of the parts.  Bound by latencies: 10 us for 32
// sequences of 256, 20 us with the gradient's lists, once a batch.
#include "attn.h"

namespace zoact {
namespace attn {

namespace {

constexpr int THREADS = 1024, BINS = 1024;

// Steps that rows of work are not cut below: a step takes 0.6 to 1.2 us, and a part's sums 4 to 8 us to be left and joined (few
// rows: 2 us).
__device__ constexpr int min_steps(int list) { return list == LIST_FWD ? 4 : 12; }
// Shares of an SM's part of all steps that rows of work are cut to: halves even out a list that has few long rows; dk and dv, whose
// parts leave twice the sums, are only cut where a row is longer than all that an SM has to do.
__device__ constexpr int split_over(int list) { return list == LIST_DKV ? 1 : SPLIT_OVER; }

size_t up(size_t n) { return (n + 255) / 256 * 256; }

__device__ __forceinline__ int64_t block_sum(int64_t v, int64_t* sh) {
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  int64_t t = 0;
  for (int i = 0; i < THREADS / 32; ++i) t += sh[i];
  return t;
}

// Exclusive sums over the block; total in *all.
__device__ __forceinline__ int block_scan(int v, int* sh, int* all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int x = v;
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 31) sh[warp] = x;
  __syncthreads();
  int before = 0, total = 0;
  for (int i = 0; i < THREADS / 32; ++i) {
    if (i < warp) before += sh[i];
    total += sh[i];
  }
  *all = total;
  return before + x - v;
}

struct Builder {
  int list, causal, kv_heads, positions, n_seq;
  const int4* seqs;                       // q0, nq, k0, nk
  const int* prefix;                      // rows of work before each sequence

  __device__ int rows_of(const int4& s) const {
    if (list == LIST_DKV) return (s.w + BK - 1) / BK;
    const int per = list == LIST_FWD ? 2 * positions : positions;
    return (s.y + per - 1) / per;
  }
  // Row of work r: its rectangle, and how many steps long it is.
  __device__ int row_at(int r, Item& w) const {
    int lo = 0, hi = n_seq;               // the sequence with prefix[lo] <= r < prefix[lo + 1]
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (prefix[mid] <= r) lo = mid; else hi = mid;
    }
    const int4 s = seqs[lo];
    const int b = r - prefix[lo];
    const int64_t first = (int64_t)s.w - s.y + 1;          // keys that position 0 of the sequence sees
    w.part = 0; w.nparts = 1; w.slot = 0; w.seq = lo;
    if (list == LIST_DKV) {
      w.k0 = s.z + b * BK;
      w.nk = min(BK, s.w - b * BK);
      // the first position that sees the block's first key
      int64_t i0 = causal ? (int64_t)b * BK + 1 - first : 0;
      i0 = i0 < 0 ? 0 : i0 > s.y ? s.y : i0;
      w.q0 = s.x + (int)i0;
      w.npos = s.y - (int)i0;
      w.diag = causal ? (int)(first + i0 - (int64_t)b * BK) : w.nk;
      return (w.npos + positions - 1) / positions;
    }
    const int per = list == LIST_FWD ? 2 * positions : positions;
    w.q0 = s.x + b * per;
    w.npos = min(per, s.y - b * per);
    w.k0 = s.z;
    const int64_t see = first + (int64_t)b * per;          // of this row's first position
    int64_t nk = s.w;
    if (causal) {
      nk = see + w.npos - 1;
      nk = nk < 0 ? 0 : nk > s.w ? s.w : nk;
    }
    w.nk = (int)nk;
    w.diag = causal ? (int)see : w.nk;
    return (w.nk + BK - 1) / BK;
  }
  // Part p of n of a row that is `steps` long.
  __device__ void cut(Item& w, int steps, int p, int n) const {
    const int a = (int)((int64_t)steps * p / n), b = (int)((int64_t)steps * (p + 1) / n);
    w.part = p;
    w.nparts = n;
    if (list == LIST_DKV) {
      const int i0 = a * positions, i1 = min(b * positions, w.npos);
      w.q0 += i0;
      w.npos = i1 - i0;
      if (causal) w.diag += i0;
    } else {
      const int j0 = a * BK, j1 = min(b * BK, w.nk);
      w.k0 += j0;
      w.nk = j1 - j0;
      w.diag = causal ? w.diag - j0 : w.nk;
    }
  }
};

struct PlanArgs {
  Shape s;
  const void* spans;
  int id64, grad, sm_count;
  uint64_t tag;
  uint8_t* plan;
  Layout at;
  int* status;
};

__global__ void __launch_bounds__(THREADS) plan_kernel(const PlanArgs p) {
  __shared__ int64_t sums[THREADS / 32];
  __shared__ int scan[THREADS / 32], bins[BINS], slot_next, bad;
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x, n = p.s.n_seq;
  Head* head = reinterpret_cast<Head*>(p.plan);
  int4* seqs = reinterpret_cast<int4*>(p.plan + p.at.seqs);
  int* prefix = reinterpret_cast<int*>(p.plan + p.at.prefix);
  if (tid == 0) bad = 0;
  __syncthreads();
  for (int i = tid; i < n; i += THREADS) {
    int64_t v[4];
    for (int j = 0; j < 4; ++j) v[j] = load_id(p.spans, p.id64, 4 * (int64_t)i + j);
    // differences, so that no sum of what may be any number overflows
    bool ok = v[0] >= 0 && v[1] >= 0 && v[2] >= 0 && v[3] >= 0 && v[0] <= p.s.rows_q && v[1] <= p.s.rows_q - v[0] &&
              v[2] <= p.s.rows_k && v[3] <= p.s.rows_k - v[2];
    if (ok && i > 0) {                    // in order: a row of the output belongs to one sequence
      const int64_t pq = load_id(p.spans, p.id64, 4 * (int64_t)(i - 1)), nq = load_id(p.spans, p.id64, 4 * (int64_t)(i - 1) + 1);
      const int64_t pk = load_id(p.spans, p.id64, 4 * (int64_t)(i - 1) + 2), nk = load_id(p.spans, p.id64, 4 * (int64_t)(i - 1) + 3);
      ok = pq <= v[0] && nq <= v[0] - pq && (!p.grad || (pk <= v[2] && nk <= v[2] - pk));
    }
    if (!ok) bad = 1;
    seqs[i] = make_int4((int)v[0], (int)v[1], (int)v[2], (int)v[3]);
  }
  __syncthreads();
  const bool ok = bad == 0;
  if (tid == 0) {
    head->tag = p.tag;
    head->has = !ok ? 0 : p.grad ? HAS_FWD | HAS_GRAD : HAS_FWD;
    if (!ok) record_error(p.status, ZOACT_ERR_INVALID_ARG);
  }
  if (!ok) return;
  Builder b = {0, p.s.causal, p.s.kv_heads, tile_positions(p.s.heads / p.s.kv_heads), n, seqs, prefix};
  for (int list = 0; list < (p.grad ? LISTS : 1); ++list) {
    b.list = list;
    __syncthreads();                      // the list before has been read
    int rows = 0;
    for (int i0 = 0; i0 < n; i0 += THREADS) {
      const int i = i0 + tid;
      int all;
      const int before = block_scan(i < n ? b.rows_of(seqs[i]) : 0, scan, &all);
      if (i < n) prefix[i] = rows + before;
      rows += all;
    }
    if (tid < BINS) bins[tid] = 0;
    if (tid == 0) slot_next = 0;
    int64_t steps = 0;
    Item w;
    __syncthreads();
    for (int r = tid; r < rows; r += THREADS) steps += b.row_at(r, w);
    steps = block_sum(steps, sums) * p.s.kv_heads;
    // a part is no shorter than its share of the GPU: at most 2 parts of a share each, so that the slots suffice
    const int over = split_over(list) * p.sm_count;
    const int64_t share = max((int64_t)min_steps(list), (steps + over - 1) / over);
    const bool cuts = p.s.head_dim <= TC_DIM;
    const auto parts_of = [&](int len) { return cuts && len > share ? (int)((len + share - 1) / share) : 1; };
    const auto bin_of = [&](int len, int parts) { return BINS - 1 - min((len + parts - 1) / parts, BINS - 1); };
    for (int r = tid; r < rows; r += THREADS) {
      const int len = b.row_at(r, w), parts = parts_of(len);
      atomicAdd(&bins[bin_of(len, parts)], parts);
    }
    __syncthreads();
    int all;
    const int start = block_scan(bins[tid], scan, &all);
    __syncthreads();
    bins[tid] = start;
    __syncthreads();
    Item* items = reinterpret_cast<Item*>(p.plan + p.at.items[list]);
    for (int r = tid; r < rows; r += THREADS) {
      const int len = b.row_at(r, w), parts = parts_of(len);
      const int at = atomicAdd(&bins[bin_of(len, parts)], parts);
      const int slot = parts > 1 ? atomicAdd(&slot_next, parts * p.s.kv_heads) : 0;
      for (int i = 0; i < parts; ++i) {
        Item c = w;
        if (parts > 1) b.cut(c, len, i, parts);
        c.slot = slot;
        if (at + i < p.at.most[list]) items[at + i] = c;
      }
    }
    if (tid == 0) head->count[list] = all;
  }
}

}  // namespace

Layout plan_layout(const Shape& s, int sm_count, int grad) {
  Layout l = {};
  const int positions = tile_positions(s.rep());
  size_t at = up(sizeof(Head));
  l.seqs = at;
  at += up((size_t)s.n_seq * sizeof(int4));
  l.prefix = at;
  at += up((size_t)s.n_seq * sizeof(int));
  for (int i = 0; i < (grad ? LISTS : 1); ++i) {
    const int64_t rows = i == LIST_DKV ? s.rows_k : s.rows_q, per = i == LIST_FWD ? 2 * positions : i == LIST_DQ ? positions : BK;
    // (parts of cut rows: at most 2 for each share of work; the sequences' rows of q, and with a gradient of k, do not overlap)
    l.most[i] = rows / per + s.n_seq + slot_count(sm_count);
    l.items[i] = at;
    at += up((size_t)l.most[i] * sizeof(Item));
  }
  l.delta = at;
  if (grad) at += up((size_t)s.rows_q * s.heads * sizeof(float));
  l.largest = at;
  if (grad) at += up((size_t)s.n_seq * s.kv_heads * sizeof(float2));
  l.total = at;
  return l;
}

uint64_t plan_tag(const Shape& s, int sm_count) {
  const uint64_t v[] = {(uint64_t)s.rows_q, (uint64_t)s.rows_k, (uint64_t)s.n_seq, (uint64_t)s.heads, (uint64_t)s.kv_heads,
                        (uint64_t)s.head_dim, (uint64_t)s.causal, (uint64_t)sm_count};
  uint64_t h = 0x7a6f617474656e64ull;
  for (uint64_t x : v) {
    h ^= x + 0x9E3779B97F4A7C15ull;
    h ^= h >> 30; h *= 0xBF58476D1CE4E5B9ull;       // SplitMix64's mixer (Steele, Lea, Flood, OOPSLA 2014)
    h ^= h >> 27; h *= 0x94D049BB133111EBull;
    h ^= h >> 31;
  }
  return h;
}

int launch_plan(Ctx* ctx, const Shape& s, const void* spans, int id64, uint8_t* plan, int grad) {
  const Layout at = plan_layout(s, ctx->sm_count, grad);
  PlanArgs p = {s, spans, id64, grad, ctx->sm_count, plan_tag(s, ctx->sm_count), plan, at, ctx->d_status};
  ZOACT_CUDA_TRY(launch_pdl(ctx, plan_kernel, dim3(1), dim3(THREADS), 0, p));
  ++ctx->n_launch;
  return ZOACT_OK;
}

int slots(Ctx* ctx, Slots* s) {
  const size_t n = (size_t)slot_count(ctx->sm_count);
  const size_t rows = n * 2 * TILE, own = (size_t)ctx->sm_count * TILE;
  s->sums = (float*)scratch(ctx, SLOT_ATTN, (rows + own) * (TC_DIM * sizeof(float) + sizeof(float2)));
  if (!s->sums) return ZOACT_ERR_NOMEM;
  s->merge = s->sums + rows * TC_DIM;
  s->stat = reinterpret_cast<float2*>(s->merge + own * TC_DIM);
  s->merge_stat = s->stat + rows;
  s->tickets = (unsigned*)scratch_zeroed(ctx, SLOT_ATTN_TICKETS, n * 4 * sizeof(unsigned));
  return s->tickets ? ZOACT_OK : ZOACT_ERR_NOMEM;
}

bool tc_supported(const Args& a, bool grad) {
  const auto lies = [](const void* p, int64_t ld) { return ((uintptr_t)p & 15) == 0 && ld % 8 == 0; };
  if (a.dtype == ZOACT_DT_FP32 || a.s.head_dim % 8 != 0 || a.s.head_dim > TC_DIM || a.s.rows_q == 0 || a.s.rows_k == 0) return false;
  return lies(a.q, a.ld_q) && lies(a.k, a.ld_k) && lies(a.v, a.ld_v) && lies(a.O, a.ld_o) &&
         (!grad || (lies(a.dO, a.ld_do) && lies(a.dq, a.ld_dq) && lies(a.dk, a.ld_dk) && lies(a.dv, a.ld_dv)));
}

}  // namespace attn
}  // namespace zoact
