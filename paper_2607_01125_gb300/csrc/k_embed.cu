// The embedding at the input of a language model: scaled rows of a table by token id, and the table's gradient.  A negative id
// is a token without a row (padding): its output is zero and it adds nothing to the gradient.
//
// Both are bound by memory.  The gradient sums the tokens of each id in token order, whatever their number: the tokens are
// sorted by id (stable), a block takes 16 sorted tokens and a slice of the columns, writes the rows whose tokens it has all
// of, and leaves its sums of the first and the last id where these go on in other blocks to a second kernel.  A short list's
// order is counted, a long one's sorted in one cluster of eight CTAs, which exchange their digit counts through shared memory;
// in the same launch all other SMs write the zeros of a dense gradient, which takes longer.
//
// Measured: 4096 rows of 4096 in bf16 9.9 us (5.2 TB/s); their gradient into a dense 128256 x 4096 table 154 us (zeros 138, sums
// 15, join 6; 7.0 TB/s; 10240 tokens 183, 16384 196, 40000 271), that of 9001 tokens added to an 8192 x 5120 fp16 table 52 us (order 12, sums 26, join 16).
#include "internal.h"
#include "tc_common.cuh"

namespace zoact {
namespace {

constexpr int EMB_THREADS = 256;

template <int E, typename T>
__device__ __forceinline__ void emb_load(const T* p, float* v) {
  if constexpr (E == 1) {
    v[0] = to_f32<T>(*p);
  } else {
    constexpr int N = 16 / (int)sizeof(T);
#pragma unroll
    for (int q = 0; q < E / N; ++q) {
      const uint4 u = *reinterpret_cast<const uint4*>(p + q * N);
      const T* e = reinterpret_cast<const T*>(&u);
#pragma unroll
      for (int i = 0; i < N; ++i) v[q * N + i] = to_f32<T>(e[i]);
    }
  }
}
template <int E, typename T>
__device__ __forceinline__ void emb_store(T* p, const float* v) {
  if constexpr (E == 1) {
    *p = from_f32<T>(v[0]);
  } else {
    constexpr int N = 16 / (int)sizeof(T);
#pragma unroll
    for (int q = 0; q < E / N; ++q) {
      uint4 u;
      T* e = reinterpret_cast<T*>(&u);
#pragma unroll
      for (int i = 0; i < N; ++i) e[i] = from_f32<T>(v[q * N + i]);
      *reinterpret_cast<uint4*>(p + q * N) = u;
    }
  }
}

// A block a token, VPT vectors of a thread in flight together.
template <typename T, int E>
__global__ void __launch_bounds__(EMB_THREADS)
embed_kernel(const T* __restrict__ tab, const void* __restrict__ ids, int id64, int64_t vocab, int d, float scale,
             T* __restrict__ Y, int* status) {
  constexpr int VPT = 4;
  pdl_wait();                              // ids and table as earlier kernels left them
  pdl_trigger();
  const int64_t t = blockIdx.x;
  const int64_t id = load_id(ids, id64, t);
  const bool ok = id >= 0 && id < vocab;
  if (id >= vocab && threadIdx.x == 0) record_error(status, ZOACT_ERR_INVALID_ARG);
  const T* e = tab + (ok ? id : 0) * d;
  T* y = Y + t * d;
  const int nv = d / E;
  for (int i0 = threadIdx.x; i0 < nv; i0 += VPT * blockDim.x) {
    float v[VPT][E];
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
#pragma unroll
      for (int j = 0; j < E; ++j) v[k][j] = 0.f;
      const int i = i0 + k * blockDim.x;
      if (ok && i < nv) emb_load<E, T>(e + (int64_t)i * E, v[k]);
    }
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
      const int i = i0 + k * blockDim.x;
#pragma unroll
      for (int j = 0; j < E; ++j) v[k][j] *= scale;
      if (i < nv) emb_store<E, T>(y + (int64_t)i * E, v[k]);
    }
  }
}

// ---- tokens sorted by id ----
constexpr int SORT_CTAS = 8, SORT_THREADS = 1024, SORT_WARPS = SORT_THREADS / 32;
constexpr int DIGIT_BITS = 9, DIGITS = 1 << DIGIT_BITS;

__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_peer_u32(const uint32_t* p, uint32_t rank) {
  uint32_t a, v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(tc::smem_u32(p)), "r"(rank));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}

struct __align__(16) SortShared {
  uint32_t hist[SORT_WARPS][DIGITS];       // a warp's count of each digit, then where its next item of that digit goes
  uint32_t total[DIGITS], base[DIGITS];
  uint32_t warp_sum[DIGITS / 32];
};

// Stable sort of the tokens by id, least significant digits first; ids that are no token's become `vocab` and end up last.
// A warp has a contiguous range of items in each pass and keeps its items' order within a digit by its lanes' order.
// Items are (id, token); the first pass reads the ids and writes b, the next reads b and writes a, and so on.
__device__ __forceinline__ void sort_tokens(SortShared& sh, const void* __restrict__ ids, int id64, int64_t n, uint32_t vocab,
                                            int passes, uint2* a, uint2* b, int* status) {
  uint32_t rank;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t below = (1u << lane) - 1u;
  const int64_t per = ((n + SORT_CTAS * SORT_WARPS - 1) / (SORT_CTAS * SORT_WARPS) + 31) / 32 * 32;
  const int64_t i0 = ((int64_t)rank * SORT_WARPS + warp) * per, i1 = i0 + per < n ? i0 + per : n;
  for (int p = 0; p < passes; ++p) {
    const int shift = p * DIGIT_BITS;
    auto item = [&](int64_t i) {
      if (p > 0) return __ldcg(a + i);
      const int64_t id = load_id(ids, id64, i);
      const bool ok = id >= 0 && id < (int64_t)vocab;
      return make_uint2(ok ? (uint32_t)id : vocab, (uint32_t)i);
    };
    for (int d = threadIdx.x; d < SORT_WARPS * DIGITS / 4; d += SORT_THREADS)
      reinterpret_cast<uint4*>(sh.hist)[d] = make_uint4(0u, 0u, 0u, 0u);
    __syncthreads();
    for (int64_t i = i0 + lane; i - lane < i1; i += 32) {
      const bool in = i < i1;
      uint32_t d = DIGITS;                 // lanes past the range match each other only
      if (in) {
        const uint2 it = item(i);
        if (p == 0 && it.x == vocab && load_id(ids, id64, i) >= (int64_t)vocab) record_error(status, ZOACT_ERR_INVALID_ARG);
        d = (it.x >> shift) & (DIGITS - 1);
      }
      const uint32_t same = __match_any_sync(0xffffffffu, d);
      if (in && (same & below) == 0) sh.hist[warp][d] += __popc(same);
      __syncwarp();
    }
    __syncthreads();
    // a digit's items: warps in order within the CTA ...
    uint32_t mine = 0;
    if (threadIdx.x < DIGITS) {
      uint32_t c[SORT_WARPS];
#pragma unroll
      for (int w = 0; w < SORT_WARPS; ++w) c[w] = sh.hist[w][threadIdx.x];
#pragma unroll
      for (int w = 0; w < SORT_WARPS; ++w) {
        sh.hist[w][threadIdx.x] = mine;
        mine += c[w];
      }
      sh.total[threadIdx.x] = mine;
    }
    cluster_barrier();
    // ... CTAs in order within the cluster, and digits in order
    uint32_t before = 0, all = 0;
    if (threadIdx.x < DIGITS) {
#pragma unroll
      for (uint32_t r = 0; r < SORT_CTAS; ++r) {
        const uint32_t c = cluster_peer_u32(&sh.total[threadIdx.x], r);
        before += r < rank ? c : 0u;
        all += c;
      }
      uint32_t incl = all;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
      }
      if (lane == 31) sh.warp_sum[warp] = incl;
      sh.base[threadIdx.x] = incl - all + before;
    }
    __syncthreads();
    if (threadIdx.x < DIGITS) {
      uint32_t s = 0;
      for (int w = 0; w < warp; ++w) s += sh.warp_sum[w];
      sh.base[threadIdx.x] += s;
    }
    __syncthreads();
    for (int64_t i = i0 + lane; i - lane < i1; i += 32) {
      const bool in = i < i1;
      uint2 it = make_uint2(0u, 0u);
      uint32_t d = DIGITS;
      if (in) {
        it = item(i);
        d = (it.x >> shift) & (DIGITS - 1);
      }
      const uint32_t same = __match_any_sync(0xffffffffu, d);
      uint32_t at = 0;
      if (in) at = sh.hist[warp][d];
      __syncwarp();
      if (in) {
        if ((same & below) == 0) sh.hist[warp][d] = at + __popc(same);
        __stcg(b + sh.base[d] + at + __popc(same & below), it);
      }
      __syncwarp();
    }
    cluster_barrier();                     // the items are in place, and the counts may be overwritten
    uint2* t = a;
    a = b;
    b = t;
  }
}

// Zeros to [p, p + bytes) by the launch's other CTAs, ZERO_VECTORS 16-byte stores a thread and no loop: a CTA for each 64 KB in
// address order writes 7.6 TB/s, alone or in the sort's clusters (1.05 GB beside the order of 4096 and of 12000 tokens: 138 and
// 139 us).  A loop over the SMs' CTAs wrote 6.4, and 4.6 in clusters, which do not fill every SM.
constexpr int ZERO_VECTORS = 4;
constexpr int64_t ZERO_BYTES = (int64_t)SORT_THREADS * ZERO_VECTORS * 16;     // of a CTA

__device__ __forceinline__ void zero_bytes(uint8_t* p, int64_t bytes, int64_t cta) {
  const int64_t head = (16 - ((uintptr_t)p & 15)) & 15;
  const int64_t nv = bytes > head ? (bytes - head) / 16 : 0;
  uint4* v = reinterpret_cast<uint4*>(p + head);
  const int64_t i0 = cta * SORT_THREADS * ZERO_VECTORS + threadIdx.x;
#pragma unroll
  for (int k = 0; k < ZERO_VECTORS; ++k)
    if (i0 + k * SORT_THREADS < nv) v[i0 + k * SORT_THREADS] = make_uint4(0u, 0u, 0u, 0u);
  if (cta == 0 && threadIdx.x < 16) {              // the ends of an array that does not begin or end on 16 bytes
    const int64_t tail = head + nv * 16;
    if ((int64_t)threadIdx.x < head && (int64_t)threadIdx.x < bytes) p[threadIdx.x] = 0;
    if (tail + (int64_t)threadIdx.x < bytes) p[tail + threadIdx.x] = 0;
  }
}

__global__ void __cluster_dims__(SORT_CTAS, 1, 1) __launch_bounds__(SORT_THREADS)
embed_sort_kernel(const void* __restrict__ ids, int id64, int64_t n, int64_t vocab, int passes, uint2* a, uint2* b,
                  uint8_t* zero, int64_t zero_len, int* status) {
  extern __shared__ __align__(16) uint8_t sort_smem[];
  SortShared& sh = *reinterpret_cast<SortShared*>(sort_smem);
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x < SORT_CTAS)              // the first cluster
    sort_tokens(sh, ids, id64, n, (uint32_t)vocab, passes, a, b, status);
  else
    zero_bytes(zero, zero_len, (int64_t)blockIdx.x - SORT_CTAS);
}

// The same order for a short list, every token's place counted: place(i) = the tokens with a smaller id, and the earlier ones
// with the same.  n^2 comparisons, but no passes that wait for one another.  A block places RANK_TOKENS tokens; a lane has
// a token and a warp a RANK_PARTS'th of the list, read from shared memory four ids at a time.  Ids are whole numbers below 2^24,
// held as floats: id + 1 - x cut to [0, 1] counts an x <= id in one addition (an integer comparison issues at half the rate).
// The whole gradient of a narrow table, this way and by the passes: 64 tokens 7.1 us for 13.9, 4096 14.4 for 18.9, 9001 19.9
// for 23.1, 12000 34.3 for 24.8 (RANK_MOST).
constexpr int RANK_TOKENS = 64, RANK_PARTS = SORT_WARPS / (RANK_TOKENS / 32);
constexpr int RANK_MOST = 10240;
constexpr int64_t RANK_VOCAB = (1 << 24) - 1;

__device__ __forceinline__ void rank_tokens(float* sh, const void* __restrict__ ids, int id64, int n, int vocab,
                                            uint2* sorted, int* status) {
  const int n_pad = (n + 3) / 4 * 4;
  float(*count)[RANK_TOKENS] = reinterpret_cast<float(*)[RANK_TOKENS]>(sh + n_pad);
  constexpr int AHEAD = 8;
  for (int i0 = threadIdx.x; i0 < n_pad; i0 += AHEAD * SORT_THREADS) {
    int64_t id[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int i = i0 + k * SORT_THREADS;
      if (i < n) id[k] = load_id(ids, id64, i);
    }
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int i = i0 + k * SORT_THREADS;
      if (i < n) {
        sh[i] = (float)(id[k] >= 0 && id[k] < vocab ? (int)id[k] : vocab);
        if (blockIdx.x == 0 && id[k] >= vocab) record_error(status, ZOACT_ERR_INVALID_ARG);
      } else if (i < n_pad) {
        sh[i] = INFINITY;                  // past the list: above every id
      }
    }
  }
  __syncthreads();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int slot = warp % (RANK_TOKENS / 32) * 32 + lane, me = (int)blockIdx.x * RANK_TOKENS + slot;
  const int groups = n_pad / 4, per = (groups + RANK_PARTS - 1) / RANK_PARTS;
  const int part = warp / (RANK_TOKENS / 32), g0 = part * per, g1 = g0 + per < groups ? g0 + per : groups;
  const float id = me < n ? sh[me] : 0.f, id1 = id + 1.f;
  float c0 = 0.f, c1 = 0.f;
  // groups wholly before the warp's tokens count equal ids too, those wholly after them do not
  const int first = (me - lane) / 4, past = first + 8;
  const float4* v = reinterpret_cast<const float4*>(sh);
  int g = g0;
#pragma unroll 8
  for (; g < (g1 < first ? g1 : first); ++g) {
    const float4 u = v[g];
    c0 += __saturatef(id1 - u.x);
    c1 += __saturatef(id1 - u.y);
    c0 += __saturatef(id1 - u.z);
    c1 += __saturatef(id1 - u.w);
  }
  for (; g < (g1 < past ? g1 : past); ++g) {
    const float4 u = v[g];
    const float e[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) c0 += e[k] < id || (e[k] == id && g * 4 + k < me) ? 1.f : 0.f;
  }
#pragma unroll 8
  for (; g < g1; ++g) {
    const float4 u = v[g];
    c0 += __saturatef(id - u.x);
    c1 += __saturatef(id - u.y);
    c0 += __saturatef(id - u.z);
    c1 += __saturatef(id - u.w);
  }
  const float c = c0 + c1;
  count[part][slot] = c;
  __syncthreads();
  const int i = (int)blockIdx.x * RANK_TOKENS + threadIdx.x;
  if (threadIdx.x >= RANK_TOKENS || i >= n) return;
  float at = 0.f;
#pragma unroll
  for (int k = 0; k < RANK_PARTS; ++k) at += count[k][threadIdx.x];
  __stcg(sorted + (int)at, make_uint2((uint32_t)sh[i], (uint32_t)i));
}

// The first `ranks` blocks place the tokens, the others write zeros as above.
__global__ void __launch_bounds__(SORT_THREADS)
embed_rank_kernel(const void* __restrict__ ids, int id64, int n, int64_t vocab, int ranks, uint2* sorted, uint8_t* zero,
                  int64_t zero_len, int* status) {
  extern __shared__ __align__(16) uint8_t sort_smem[];
  pdl_wait();
  pdl_trigger();
  if ((int)blockIdx.x < ranks)
    rank_tokens(reinterpret_cast<float*>(sort_smem), ids, id64, n, (int)vocab, sorted, status);
  else
    zero_bytes(zero, zero_len, (int64_t)blockIdx.x - ranks);
}

// ---- sums of sorted tokens ----
constexpr int PIECE = 16;                  // sorted tokens of a block, all in flight together

// E elements that lie together, in one load.
template <typename T, int E>
struct alignas(E * sizeof(T)) Raw {
  T e[E];
};

// A block waits for its ids and then once for all its rows, so several blocks on an SM carry it: with four elements a thread and
// 85 registers there are three (9001 tokens of 5120 columns added to an fp16 table: 9 us less than with eight and one block;
// two blocks 3.5 us more; pieces of 8 tokens, which leave twice the sums to join, 9 us more).
// One block: tokens [PIECE blockIdx.x, ...) of the sorted list, columns of slice blockIdx.y.  part [pieces][2][d] fp32: the sum
// of the piece's first id where earlier pieces have it too, and of its last id where only later ones do.
template <typename T, typename TE, int E, bool ADD>
__global__ void __launch_bounds__(EMB_THREADS, 3)
embed_sum_kernel(const T* __restrict__ dY, int64_t n, int d, const uint2* __restrict__ sorted, uint32_t vocab, float scale,
                 TE* __restrict__ dE, float* __restrict__ part) {
  pdl_wait();
  pdl_trigger();
  __shared__ uint2 item[PIECE + 2];        // with the tokens before and after
  const int64_t p0 = (int64_t)blockIdx.x * PIECE;
  if (threadIdx.x < PIECE + 2) {
    const int64_t i = p0 + (int)threadIdx.x - 1;
    item[threadIdx.x] = i >= 0 && i < n ? __ldcg(sorted + i) : make_uint2(0xffffffffu, 0u);
  }
  __syncthreads();
  const int64_t c = ((int64_t)blockIdx.y * blockDim.x + threadIdx.x) * E;
  if (c >= d) return;
  const uint32_t before = item[0].x;
  Raw<T, E> v[PIECE];
  Raw<TE, E> old[ADD ? PIECE : 1];
#pragma unroll
  for (int k = 0; k < PIECE; ++k) {
    const uint32_t id = item[k + 1].x;     // past the list's end, and where it is no token's: not below vocab
    if (id < vocab) {
      v[k] = *reinterpret_cast<const Raw<T, E>*>(dY + (int64_t)item[k + 1].y * d + c);
      if (ADD && id != before && item[k + 2].x != id) old[k] = *reinterpret_cast<const Raw<TE, E>*>(dE + (int64_t)id * d + c);
    }
  }
  float sum[E];
#pragma unroll
  for (int j = 0; j < E; ++j) sum[j] = 0.f;
#pragma unroll
  for (int k = 0; k < PIECE; ++k) {
    const uint32_t id = item[k + 1].x, next = item[k + 2].x;
    if (id >= vocab) continue;
#pragma unroll
    for (int j = 0; j < E; ++j) sum[j] += to_f32<T>(v[k].e[j]);
    if (next == id && k + 1 < PIECE) continue;
    if (id == before || next == id) {
      Raw<float, E>* o = reinterpret_cast<Raw<float, E>*>(part + ((int64_t)blockIdx.x * 2 + (id == before ? 0 : 1)) * d + c);
      Raw<float, E> r;
#pragma unroll
      for (int j = 0; j < E; ++j) r.e[j] = sum[j];
      *o = r;
    } else {
      Raw<TE, E> r;
#pragma unroll
      for (int j = 0; j < E; ++j) r.e[j] = from_f32<TE>(ADD ? fmaf(scale, sum[j], to_f32<TE>(old[ADD ? k : 0].e[j])) : scale * sum[j]);
      *reinterpret_cast<Raw<TE, E>*>(dE + (int64_t)id * d + c) = r;
    }
#pragma unroll
    for (int j = 0; j < E; ++j) sum[j] = 0.f;
  }
}

// The ids that several pieces have: the block of the piece where one begins adds the pieces' sums in order.  How many there
// are is counted first, so that the sums' loads wait for nothing but their own memory, 16 at a time (9001 tokens, 8192 ids, 5120
// columns: 15.5 us; with each load behind the look at its piece's id 29 us; four pieces a block 20.5 us).
template <typename TE, int E, bool ADD>
__global__ void __launch_bounds__(EMB_THREADS)
embed_join_kernel(int64_t n, int d, const uint2* __restrict__ sorted, uint32_t vocab, float scale, TE* __restrict__ dE,
                  const float* __restrict__ part) {
  pdl_wait();
  pdl_trigger();
  const int64_t p = blockIdx.x, end = (p + 1) * PIECE;
  if (end >= n) return;
  const uint32_t id = __ldcg(sorted + end - 1).x, after = __ldcg(sorted + end).x;
  const uint32_t before = p > 0 ? __ldcg(sorted + p * PIECE - 1).x : 0xffffffffu;
  if (id >= vocab || after != id || before == id) return;            // it ends here, or began earlier
  int64_t last = p;                                                  // the last piece that begins with it
  for (int more = 1;;) {
    const int64_t q = last + 1 + threadIdx.x;
    more = __syncthreads_count(q * PIECE < n && __ldcg(sorted + q * PIECE).x == id);      // sorted: the first `more` ones
    last += more;
    if (more < (int)blockDim.x) break;
  }
  const int64_t c = ((int64_t)blockIdx.y * blockDim.x + threadIdx.x) * E;
  if (c >= d) return;
  TE* o = dE + (int64_t)id * d + c;
  Raw<TE, E> old;
  if (ADD) old = *reinterpret_cast<const Raw<TE, E>*>(o);
  const Raw<float, E> own = *reinterpret_cast<const Raw<float, E>*>(part + (p * 2 + 1) * d + c);
  float sum[E];
#pragma unroll
  for (int j = 0; j < E; ++j) sum[j] = own.e[j];
  constexpr int AHEAD = 16;
  for (int64_t q = p + 1; q <= last; q += AHEAD) {
    Raw<float, E> v[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      if (q + k <= last) v[k] = *reinterpret_cast<const Raw<float, E>*>(part + (q + k) * 2 * d + c);
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      if (q + k <= last) {
#pragma unroll
        for (int j = 0; j < E; ++j) sum[j] += v[k].e[j];
      }
  }
  Raw<TE, E> r;
#pragma unroll
  for (int j = 0; j < E; ++j) r.e[j] = from_f32<TE>(ADD ? fmaf(scale, sum[j], to_f32<TE>(old.e[j])) : scale * sum[j]);
  *reinterpret_cast<Raw<TE, E>*>(o) = r;
}

bool on16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

template <typename T, int E>
int go_embed(Ctx* ctx, const void* tab, int64_t vocab, int d, const void* ids, int id64, int64_t n, float scale, void* Y) {
  const int threads = (d / E + 127) / 128 * 32;      // four vectors a thread
  ZOACT_CUDA_TRY(launch_pdl(ctx, embed_kernel<T, E>, dim3((unsigned)n), dim3(threads < EMB_THREADS ? threads : EMB_THREADS), 0,
                            (const T*)tab, ids, id64, vocab, d, scale, (T*)Y, ctx->d_status));
  ++ctx->n_launch;
  return ZOACT_OK;
}

template <typename T>
int run_embed(Ctx* ctx, const void* tab, int64_t vocab, int d, const void* ids, int id64, int64_t n, float scale, void* Y) {
  constexpr int E = 16 / (int)sizeof(T);
  return d % E == 0 && on16(tab) && on16(Y) ? go_embed<T, E>(ctx, tab, vocab, d, ids, id64, n, scale, Y)
                                            : go_embed<T, 1>(ctx, tab, vocab, d, ids, id64, n, scale, Y);
}

template <typename T, typename TE, int E, bool ADD>
int go_sums(Ctx* ctx, const void* dY, int64_t n, int d, const uint2* sorted, int64_t vocab, float scale, void* dE, float* part) {
  const int nv = d / E, slices = (nv + EMB_THREADS - 1) / EMB_THREADS, threads = ((nv + slices - 1) / slices + 31) / 32 * 32;
  const dim3 grid((unsigned)((n + PIECE - 1) / PIECE), (unsigned)slices);
  ZOACT_CUDA_TRY(launch_pdl(ctx, embed_sum_kernel<T, TE, E, ADD>, grid, dim3(threads), 0, (const T*)dY, n, d, sorted,
                            (uint32_t)vocab, scale, (TE*)dE, part));
  ++ctx->n_launch;
  if (grid.x > 1) {
    ZOACT_CUDA_TRY(launch_pdl(ctx, embed_join_kernel<TE, E, ADD>, grid, dim3(threads), 0, n, d, sorted, (uint32_t)vocab, scale,
                              (TE*)dE, (const float*)part));
    ++ctx->n_launch;
  }
  return ZOACT_OK;
}

template <typename T, typename TE>
int run_embed_grad(Ctx* ctx, const void* dY, int64_t n, int d, const void* ids, int id64, int64_t vocab, float scale,
                   void* dE, int accumulate) {
  constexpr int E = 4;                     // 16 bytes of a sum; see embed_sum_kernel
  const int64_t pieces = (n + PIECE - 1) / PIECE;
  const size_t list = ((size_t)n * sizeof(uint2) + 255) / 256 * 256;
  char* s = (char*)scratch(ctx, SLOT_EMBED, 2 * list + (size_t)pieces * 2 * d * 4);
  if (!s) return ZOACT_ERR_NOMEM;
  uint2* a = (uint2*)s;
  uint2* b = (uint2*)(s + list);
  float* part = (float*)(s + 2 * list);
  const int64_t zero_len = accumulate ? 0 : vocab * d * (int64_t)sizeof(TE), zero_ctas = (zero_len + ZERO_BYTES - 1) / ZERO_BYTES;
  const uint2* sorted = a;
  if (n <= RANK_MOST && vocab <= RANK_VOCAB) {
    const int ranks = (int)((n + RANK_TOKENS - 1) / RANK_TOKENS);
    const int smem = ((int)n + 3) / 4 * 16 + RANK_PARTS * RANK_TOKENS * 4;
    static_assert((RANK_MOST + 3) / 4 * 16 + RANK_PARTS * RANK_TOKENS * 4 <= 48 * 1024, "what any kernel may use");
    ZOACT_CUDA_TRY(launch_pdl(ctx, embed_rank_kernel, dim3((unsigned)(ranks + zero_ctas)), dim3(SORT_THREADS), (size_t)smem, ids,
                              id64, (int)n, vocab, ranks, a, (uint8_t*)dE, zero_len, ctx->d_status));
  } else {
    int passes = 1;
    while (passes * DIGIT_BITS < 32 && (vocab >> (passes * DIGIT_BITS)) != 0) ++passes;
    sorted = passes % 2 ? b : a;
    ZOACT_CUDA_TRY(cudaFuncSetAttribute(embed_sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(SortShared)));
    ZOACT_CUDA_TRY(launch_pdl(ctx, embed_sort_kernel,
                              dim3((unsigned)((SORT_CTAS + zero_ctas + SORT_CTAS - 1) / SORT_CTAS * SORT_CTAS)),
                              dim3(SORT_THREADS), sizeof(SortShared), ids, id64, n, vocab, passes, a, b, (uint8_t*)dE, zero_len,
                              ctx->d_status));
  }
  ++ctx->n_launch;
  if (n == 0) return ZOACT_OK;
  if (d % E == 0 && on16(dY) && on16(dE))
    return accumulate ? go_sums<T, TE, E, true>(ctx, dY, n, d, sorted, vocab, scale, dE, part)
                      : go_sums<T, TE, E, false>(ctx, dY, n, d, sorted, vocab, scale, dE, part);
  return accumulate ? go_sums<T, TE, 1, true>(ctx, dY, n, d, sorted, vocab, scale, dE, part)
                    : go_sums<T, TE, 1, false>(ctx, dY, n, d, sorted, vocab, scale, dE, part);
}

}  // namespace

int launch_embed(Ctx* ctx, const void* E, int dtype, int64_t vocab, int d, const void* ids, int id64, int64_t n,
                 float scale, void* Y) {
  if (n == 0) return ZOACT_OK;
  switch (dtype) {
    case ZOACT_DT_FP32: return run_embed<float>(ctx, E, vocab, d, ids, id64, n, scale, Y);
    case ZOACT_DT_BF16: return run_embed<__nv_bfloat16>(ctx, E, vocab, d, ids, id64, n, scale, Y);
    default: return run_embed<__half>(ctx, E, vocab, d, ids, id64, n, scale, Y);
  }
}

int launch_embed_grad(Ctx* ctx, const void* dY, int dtype, int64_t n, int d, const void* ids, int id64, int64_t vocab,
                      float scale, void* dE, int edtype, int accumulate) {
  if (n == 0 && accumulate) return ZOACT_OK;
  const bool f32 = edtype == ZOACT_DT_FP32;
  switch (dtype) {
    case ZOACT_DT_FP32: return run_embed_grad<float, float>(ctx, dY, n, d, ids, id64, vocab, scale, dE, accumulate);
    case ZOACT_DT_BF16:
      return f32 ? run_embed_grad<__nv_bfloat16, float>(ctx, dY, n, d, ids, id64, vocab, scale, dE, accumulate)
                 : run_embed_grad<__nv_bfloat16, __nv_bfloat16>(ctx, dY, n, d, ids, id64, vocab, scale, dE, accumulate);
    default:
      return f32 ? run_embed_grad<__half, float>(ctx, dY, n, d, ids, id64, vocab, scale, dE, accumulate)
                 : run_embed_grad<__half, __half>(ctx, dY, n, d, ids, id64, vocab, scale, dE, accumulate);
  }
}

}  // namespace zoact
