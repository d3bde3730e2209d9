// Attention over a cache in 4 bits for few query rows per KV head
// (include/mpt_kv.h, mpt_kv4_attend): single new tokens and drafts.  (It is right
// for any number of rows.)
//
// The running form, the items and the split of the work are those of
// k_attend_few.cu; rows are taken 8 or 16 to an item.  Scores are made the other
// way round, S^T = K Q^T and O^T = V^T P^T: keys, then elements, are a product's
// 16 rows, and 8 query rows its columns, so that the usual group of 8 heads or
// fewer wastes nothing, and a lane holds 8 accumulators for 32 elements of a row.
// Both operands that come from codes are the A of m16n8k16, and the cache's
// layout is that operand's: a lane's words of a key hold the pairs (e, e + 4) of
// elements of its own, in an order that the query's fragments follow, and its
// words of values pairs of tokens.  P^T comes from S^T by a transposition of
// 8 x 8 matrices across lanes.  It is f16, as the product asks for beside exact
// values: 11 bits of each probability, which is the only rounding besides the
// output's (against 64 bits 2.9e-4 of f16 outputs, where 32-bit probabilities
// leave 2.1e-4; of bf16 ones 1.67e-3 and 1.66e-3).
//
// Bound: 36 bytes a key and group of 32 elements, read once; and, before that,
// issue slots: 11 operations for 8 codes, three of them to align a piece's codes,
// about 350 a warp for 16 keys of 128 elements with all that is not codes.  So a
// warp takes 32 keys at once (waits, maxima and votes are shared by them: three
// requests of 100,001 to 131,072 keys 100 -> 90 us; 28 of heads of 256 68 -> 63), the
// maximum of a row is looked for only when a score is above its reference by more
// than 2^kLag, and one warp of five copies (a page's part of a stage is contiguous,
// so a copy is up to 36 KB).
//
// Measured (GB300, 8 KV heads of 128; from the fastest GPU to the slowest): the
// three requests 80 to 88 us, 5.0 TB/s on the fastest, of which 11 us are start, end
// and join (0.87 of the copy rate between them); 28 of 2,000 to 6,000 36 to 40 us; 150
// of 300 to 5,000, 16 heads of 64, up to 4 tokens, 136 us; one of 777 9.0 to 9.5 us,
// launches and a chain of dependent reads.
//
// Tried and slower: a ring for each warp, filled by itself, four blocks of four
// warps an SM (the three requests 97 us against 88: a fifth more operations), two
// blocks an SM (95), an item's queries read before the item before is joined (80 ->
// 88: registers).  No different: fewer or more stages, three blocks of heads of
// 64 instead of four, values' codes read before the exponentials, left shifts as
// products on the other pipe.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "kv4.cuh"

namespace mpt {
namespace {

__device__ uint32_t g_few4_counts[kKvCounts];

constexpr int kWarps = 4;  // of products; one more copies
constexpr int kThreads = 32 * (kWarps + 1);
constexpr int kLag = 4;    // scores may exceed a row's reference by 2^kLag
using L = Lift<true, kLag>;

// N: groups of 32 elements; kR: query rows of an item, in eights.
template <int N, int kR>
struct Few4Cfg {
  static constexpr int kRows = 8 * kR, kCols = 32 * N;
  static constexpr int kPerSm = kR == 1 ? (N <= 2 ? 4 : N <= 4 ? 3 : 2) : N <= 2 ? 3 : 2;
  static constexpr int kGroups = 2;  // of 16 keys, a warp takes of a stage
  static constexpr int kKeys = 16 * kGroups * kWarps;
  static constexpr int kStage = kKeys / kCodeTokens * kv4_tile(N);
  static constexpr int kStages = N <= 3 ? 4 : N == 4 ? 3 : 2;
  static constexpr int kPad = kCols + 4;  // row of the joining buffer, in floats
  static constexpr int kBuf = kWarps * kRows * kPad * 4;
  static constexpr int kMl = kWarps * 2 * kRows * 4;
  static constexpr int kSmem = 128 + kStages * kStage + kBuf + kMl + kStages * 24 + 320;
  static constexpr int kSlot = kRows * kCols + 2 * kRows;  // floats of a partial result
  // What an item costs beside its key tiles (queries, first copies, the join of
  // the warps: 3 us), in their time.  It is counted before them, as units of the
  // line without work, or the blocks with the short requests would be the last
  // (150 requests of 300 to 5,000 keys, 16 heads of 64: 154 us without, 146, 139,
  // 137 and 138 with 1 to 4; 8 heads of 128, 32 query heads: 181, 165 and 162 with 1, 3 and 4).
  static constexpr int kItem = 3;
};

__device__ __forceinline__ void mma(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The same from zero.
__device__ __forceinline__ void mma_first(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t pack_out(bool f16, float lo, float hi) {
  uint32_t r;
  if (f16) return pack_f16(lo, hi);
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ void bar_consumers() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

template <int N>
__device__ __forceinline__ void load_words(uint32_t* w, uint32_t at) {
  if constexpr (N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 4)
      asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[i]), "=r"(w[i + 1]), "=r"(w[i + 2]), "=r"(w[i + 3]) : "r"(at + 4 * i));
  } else if constexpr (N % 2 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 2) asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(w[i]), "=r"(w[i + 1]) : "r"(at + 4 * i));
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[i]) : "r"(at + 4 * i));
  }
}
__device__ __forceinline__ uint32_t load_u16(uint32_t at) {
  uint16_t r;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(r) : "r"(at));
  return r;
}
__device__ __forceinline__ uint32_t load_u32(uint32_t at) {
  uint32_t r;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(r) : "r"(at));
  return r;
}

// Bounded wait of a whole warp: false once the block has given up, or after four
// seconds (which it then counts).  The lanes vote at each look: where they leave
// the loop one by one, as in wait_bar, the three long requests take 88 us, not 80.
__device__ __forceinline__ bool look(unsigned long long* bar, uint32_t parity) { return __all_sync(~0u, mbar_try_wait(bar, parity)); }
__device__ __noinline__ bool wait_longer(unsigned long long* bar, uint32_t parity, int* gave_up) {
  const unsigned long long start = now_ns();
  for (;;) {
    if (look(bar, parity)) return true;
    bool over = *(volatile int*)gave_up != 0;
    if (!over && now_ns() - start > 4000000000ull) {
      over = true;
      *(volatile int*)gave_up = 1;
      if ((threadIdx.x & 31) == 0) atomicAdd(&g_few4_counts[kKvGaveUp], 1u);
    }
    if (__any_sync(~0u, over)) return false;
  }
}
__device__ __forceinline__ bool wait_warp(unsigned long long* bar, uint32_t parity, int* gave_up) {
  return look(bar, parity) || wait_longer(bar, parity, gave_up);
}

// One item: rows of one KV head of one request.
struct Few4Item {
  int req, head, row0, rows;  // rows: valid ones
  AttnReq r;
  int tiles;  // key tiles that any of its rows sees
};
template <int kRows>
__device__ __forceinline__ int row_tiles(const AttnParams& p, const AttnReq& r) {
  return (int)(((int64_t)r.ql * p.group + kRows - 1) / kRows);
}
template <int kKeys>
__device__ __forceinline__ int tiles_of(int n) {
  return n < 1 ? 0 : (n - 1) / kKeys + 1;
}
template <int kKeys>
__device__ __forceinline__ int key_tiles(const AttnReq& r) {
  const int n = tiles_of<kKeys>(r.kvl);
  return n < 1 ? 1 : n;
}
template <int kRows, int kKeys>
__device__ __forceinline__ Few4Item few_item(const AttnParams& p, const AttnReq& r, int req, int64_t item, int rt) {
  Few4Item it;
  it.req = req;
  it.head = (int)(item / rt);
  it.row0 = (int)(item % rt) * kRows;
  const int64_t left = (int64_t)r.ql * p.group - it.row0;
  it.rows = left < kRows ? (int)left : kRows;
  it.r = r;
  it.tiles = tiles_of<kKeys>(attn_limit(p, r, (it.row0 + it.rows - 1) / p.group));
  return it;
}
[[maybe_unused]] __device__ __forceinline__ bool few_inside(const AttnParams& p, const Few4Item& x, int row) {
  return attn_inside(p, x.req, x.head, x.r.q0, x.r.ql, x.r.kvl) && row >= 0 && row / p.group < x.r.ql;
}

// A query row's part of a lane as f16, the type of the other operand (bf16 would
// round what codes stand for), and (bf16) the power of two 2^e that was taken out
// of it, the row's largest element being below 2^(e + 1): nothing overflows.  Of
// bf16's 8 bits f16 holds all down to 2^-17 of 2^e, and what is below to 2^-25 of it.
template <int N>
__device__ __forceinline__ float query_words(const uint4* raw, bool f16, uint32_t (*qf)[2]) {
  float back = 1.f, by = 1.f;
  if (!f16) {
    uint32_t top = 0;
#pragma unroll
    for (int w = 0; w < N; ++w) {
      const uint32_t v[4] = {raw[w].x, raw[w].y, raw[w].z, raw[w].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) top = max(top, max(v[i] << 16 & 0x7FFFFFFFu, v[i] & 0x7FFF0000u));
    }
    top = max(top, __shfl_xor_sync(~0u, top, 1));
    top = max(top, __shfl_xor_sync(~0u, top, 2));
    int e = (int)(top >> 23) - 127;
    e = top == 0 ? 0 : e < -126 ? -126 : e > 126 ? 126 : e;
    by = __uint_as_float((uint32_t)(127 - e) << 23);
    back = __uint_as_float((uint32_t)(127 + e) << 23);
  }
#pragma unroll
  for (int w = 0; w < N; ++w) {
    uint32_t v[4] = {raw[w].x, raw[w].y, raw[w].z, raw[w].w};
    if (!f16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = pack_f16(__uint_as_float(v[i] << 16) * by, __uint_as_float(v[i] & 0xFFFF0000u) * by);
    }
    qf[2 * w][0] = __byte_perm(v[0], v[2], 0x5410);
    qf[2 * w][1] = __byte_perm(v[0], v[2], 0x7632);
    qf[2 * w + 1][0] = __byte_perm(v[1], v[3], 0x5410);
    qf[2 * w + 1][1] = __byte_perm(v[1], v[3], 0x7632);
  }
  return back;
}

template <int N, int kR>
__global__ void __launch_bounds__(kThreads, Few4Cfg<N, kR>::kPerSm) k_attend4_few(const __grid_constant__ AttnParams p) {
  using C = Few4Cfg<N, kR>;
  constexpr int kRows = C::kRows, kKeys = C::kKeys, kGroups = C::kGroups;
  extern __shared__ char raw[];
  char* ring = (char*)(((uintptr_t)raw + 127) & ~(uintptr_t)127);
  float* bufs = (float*)(ring + C::kStages * C::kStage);
  float* ml = (float*)((char*)bufs + C::kBuf);  // [kWarps][2][kRows]
  unsigned long long* full = (unsigned long long*)((char*)ml + C::kMl);
  unsigned long long* empty = full + C::kStages;
  uint32_t* there = (uint32_t*)(empty + C::kStages);  // per stage: which copies the cache holds
  int64_t* scratch = (int64_t*)((char*)full + C::kStages * 24);
  __shared__ int gave_up;

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], kWarps);
    }
    gave_up = 0;
    mbar_init_fence();
  }
  launch_dependents();
  const AttnRange range = attn_range<kThreads>(p.batch, blockIdx.x, gridDim.x, scratch, [&](int i) -> int64_t {
    if (attn_falls(p, i)) return -1;
    const AttnReq r = attn_req(p, i);
    return (int64_t)p.kv_heads * row_tiles<kRows>(p, r) * (key_tiles<kKeys>(r) + C::kItem);
  });
  if (tid == 0) p.desc[blockIdx.x] = make_int4(0, 0, 0, 0);
  if (range.begin >= range.end) return;
  __syncthreads();

  int req = range.req;
  AttnReq r = attn_req(p, req);
  int rt = row_tiles<kRows>(p, r);
  int cost = key_tiles<kKeys>(r) + C::kItem;
  int64_t item = range.off / cost;
  int u0 = (int)(range.off % cost);  // the item's first unit here
  int64_t left = range.end - range.begin;
  auto first_tile = [](int u) { return u > C::kItem ? u - C::kItem : 0; };
  auto next_item = [&](int seg) -> bool {
    left -= seg;
    u0 = 0;
    if (++item == (int64_t)p.kv_heads * rt) {
      item = 0;
      do {
        if (++req >= p.batch) return false;
        r = attn_req(p, req);
        rt = row_tiles<kRows>(p, r);
        cost = key_tiles<kKeys>(r) + C::kItem;
      } while (rt == 0);
    }
    return left > 0;
  };

  if (warp == kWarps) {
    // ---- copies: a page's part of a stage is contiguous ----
    const int box = p.box < kKeys ? p.box : kKeys, per = kKeys / box;  // keys of a copy; copies of a stage
    const uint32_t bytes = (uint32_t)(box / kCodeTokens * kv4_tile(N));
    const unsigned all = per == 32 ? ~0u : (1u << per) - 1;
    bool ok = true;
    uint32_t done = 0, s = 0, phase = 0;  // stages filled; the next one, and how often the ring has been
    do {
      const Few4Item x = few_item<kRows, kKeys>(p, r, req, item, rt);
      const int seg = (int)(left < cost - u0 ? left : cost - u0);
      const int t0 = first_tile(u0), end = first_tile(u0 + seg), last = end < x.tiles ? end : x.tiles;
      const int32_t* row = p.table + (int64_t)req * p.table_stride;
      auto page_of = [&](int t) -> int {  // lane b: the page of the b-th copy
        const int64_t key = (int64_t)t * kKeys + lane * box;
        if (t >= last || lane >= per || key >= r.kvl) return -1;
        const int id = row[key >> p.page_log2];
        return id < 0 || id >= p.n_pages ? -1 : id;
      };
      int next = page_of(t0);
      for (int t = t0; t < last; ++t, ++done) {
        const int id = next;
        next = page_of(t + 1);
        if (done >= C::kStages) {
          ok = wait_warp(&empty[s], phase ^ 1, &gave_up) && *(volatile int*)&gave_up == 0;
          ok = __all_sync(~0u, ok);
          if (!ok) break;
        }
        const int slot = (t * kKeys) & ((1 << p.page_log2) - 1);  // of pages larger than a stage
        const bool bad = KV_BAD(g_few4_counts, id < 0 || (id < p.n_pages && x.head < p.kv_heads && slot + box <= 1 << p.page_log2 && lane < per));
        const unsigned held = __ballot_sync(~0u, id >= 0 && !bad);
        if (lane == 0) {
          there[s] = held == all ? ~0u : held;  // a bit per copy, all of them where none is missing
          mbar_arrive_expect_tx(&full[s], bytes * __popc(held));
        }
        __syncwarp();
        if (held >> lane & 1u)
          asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                           smem_u32(ring + s * C::kStage) + lane * bytes),
                       "l"(p.k + (int64_t)id * p.k_page + (int64_t)x.head * p.k_head + (slot / kCodeTokens) * kv4_tile(N)), "r"(bytes),
                       "r"(smem_u32(&full[s]))
                       : "memory");
        __syncwarp();
        if (++s == C::kStages) {
          s = 0;
          phase ^= 1;
        }
      }
      if (!ok || !next_item(seg)) break;
    } while (true);
    // The block ends after the copies have landed, also where the warps that take them have given up.
    for (uint32_t k = done > C::kStages ? done - C::kStages : 0; k < done; ++k) wait_landed(&full[k % C::kStages], (k / C::kStages) & 1);
    return;
  }

  // ---- products ----
  const int g = lane >> 2, q = lane & 3;
  const uint32_t ring_at = smem_u32(ring) + warp * 2 * kGroups * kv4_tile(N);  // this warp's tiles of a stage
  const uint32_t k_at = kv4_key(N, g) + q * 4 * N, v_at = kv4_value(N, q) + g * 4 * N;
  uint32_t s = 0, phase = 0;  // the stage at hand
  for (;;) {
    const Few4Item x = few_item<kRows, kKeys>(p, r, req, item, rt);
    const int seg = (int)(left < cost - u0 ? left : cost - u0);
    if (u0 + seg <= C::kItem) {  // the block ends before the item's key tiles begin
      if (!next_item(seg)) break;
      continue;
    }
    const int t0 = first_tile(u0), end = first_tile(u0 + seg), last = end < x.tiles ? end : x.tiles;
    const bool starts = t0 == 0, ends = u0 + seg == cost;

    // query row 8 i + g of this lane's fragments; rows 8 i + 2 q + e of its scores
    uint32_t qf[kR][2 * N][2];
    float by[kR][2];
    int lim[kR][2];
#pragma unroll
    for (int i = 0; i < kR; ++i) {
      const int row = x.row0 + 8 * i + g;
      const bool valid = 8 * i + g < x.rows && !KV_BAD(g_few4_counts, few_inside(p, x, row));
      const char* at = p.q + 2 * ((int64_t)(r.q0 + row / p.group) * p.q_tok + ((int64_t)x.head * p.group + row % p.group) * p.q_head);
      uint4 u[N];
#pragma unroll
      for (int w = 0; w < N; ++w) {
        const int col = 8 * (q * N + w);
        u[w] = valid && col < p.dim ? *(const uint4*)(at + 2 * col) : make_uint4(0, 0, 0, 0);
      }
      const float back = kv4_scale(p.scale_log2, query_words<N>(u, p.f16, qf[i]));
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int mine = 8 * i + 2 * q + e;
        by[i][e] = __shfl_sync(~0u, back, (2 * q + e) * 4);
        lim[i][e] = mine < x.rows ? attn_limit(p, r, (x.row0 + mine) / p.group) : 0;
      }
    }
    // what every valid row sees, and what any does
    const int lim_lo = attn_limit(p, r, x.row0 / p.group), lim_hi = attn_limit(p, r, (x.row0 + x.rows - 1) / p.group);

    // Of each row: the running maximum (a reference that lags behind it), the sum,
    // what a score's exponent is less by, and the score above which the reference grows.
    float o[kR][2 * N][4], m[kR][2], l[kR][2], off[kR][2], most[kR][2];
#pragma unroll
    for (int i = 0; i < kR; ++i) {
#pragma unroll
      for (int n = 0; n < 2 * N; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][n][e] = 0.f;
      m[i][0] = m[i][1] = -INFINITY;
      l[i][0] = l[i][1] = 0.f;
      off[i][0] = off[i][1] = L::kLift;
      most[i][0] = most[i][1] = -INFINITY;
    }

    for (int t = t0; t < last; ++t) {
      // having given up, the block still ends in order
      (void)wait_warp(&full[s], phase, &gave_up);
      const uint32_t at = ring_at + s * C::kStage;
      const int key0 = t * kKeys + 16 * kGroups * warp;
      if (key0 < lim_hi) {
        // S^T = K Q^T, 16 keys at a time: rows g (a tile of 8) and g + 8 (the next)
        float sc[kGroups][kR][4];
#pragma unroll
        for (int u = 0; u < kGroups; ++u) {
          const uint32_t a_at = at + 2 * u * kv4_tile(N), b_at = a_at + kv4_tile(N);
          float half[kR][4];  // every second product, so that a chain is half as long
          uint32_t wa[N], wb[N], sa, oa, sb, ob;
          load_words<N>(wa, a_at + k_at);
          load_words<N>(wb, b_at + k_at);
#pragma unroll
          for (int w = 0; w < N; ++w) {
            // the group of word q N + w: the same for all of a lane's words where N is 1, 2 or 4
            if (w == 0 || (N == 8 && w == 4) || (N & (N - 1)) != 0) {
              const uint32_t mk = kv4_key_marks(N, g) + 2 * ((q * N + w) >> 2);
              kv4_key_steps(load_u16(a_at + mk), load_u16(b_at + mk), sa, oa, sb, ob);
            }
            uint32_t a[4], b[4];
            kv4_word(wa[w], sa, oa, a);
            kv4_word(wb[w], sb, ob, b);
#pragma unroll
            for (int i = 0; i < kR; ++i) {
              if (w == 0) {
                mma_first(sc[u][i], a[0], b[0], a[1], b[1], qf[i][2 * w][0], qf[i][2 * w][1]);
                mma_first(half[i], a[2], b[2], a[3], b[3], qf[i][2 * w + 1][0], qf[i][2 * w + 1][1]);
              } else {
                mma(sc[u][i], a[0], b[0], a[1], b[1], qf[i][2 * w][0], qf[i][2 * w][1]);
                mma(half[i], a[2], b[2], a[3], b[3], qf[i][2 * w + 1][0], qf[i][2 * w + 1][1]);
              }
            }
          }
#pragma unroll
          for (int i = 0; i < kR; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[u][i][e] += half[i][e];
        }
        const uint32_t held = there[s];
        if (lim_lo - key0 < 16 * kGroups || held != ~0u) {
          const int shift = __ffs(p.box < kKeys ? p.box : kKeys) - 1;  // keys of a copy, a power of two
#pragma unroll
          for (int u = 0; u < kGroups; ++u)
#pragma unroll
            for (int i = 0; i < kR; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (key0 + 16 * u + g + 8 * (e >> 1) >= lim[i][e & 1] ||
                    !(held >> ((16 * kGroups * warp + 16 * u + 8 * (e >> 1)) >> shift) & 1u))
                  sc[u][i][e] = -INFINITY;
        }
        bool grows = false;
#pragma unroll
        for (int u = 0; u < kGroups; ++u)
#pragma unroll
          for (int i = 0; i < kR; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) grows |= sc[u][i][e] > most[i][e & 1];
        if (__any_sync(~0u, grows)) {
#pragma unroll
          for (int i = 0; i < kR; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float mx = fmaxf(sc[0][i][e], sc[0][i][2 + e]);
#pragma unroll
              for (int u = 1; u < kGroups; ++u) mx = fmaxf(mx, fmaxf(sc[u][i][e], sc[u][i][2 + e]));
              mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 4));
              mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 8));
              mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 16));
              const float mn = L::reference(fmaxf(m[i][e], mx * by[i][e])), safe = mn == -INFINITY ? 0.f : mn;
              const float alpha = ex2(m[i][e] - safe);
              m[i][e] = mn;
              off[i][e] = L::kLift - safe;
              most[i][e] = (mn + kLag) / by[i][e];
              l[i][e] *= alpha;
#pragma unroll
              for (int n = 0; n < 2 * N; ++n) {
                o[i][n][e] *= alpha;
                o[i][n][2 + e] *= alpha;
              }
            }
        }
        uint32_t pb[kGroups][kR][2];
#pragma unroll
        for (int u = 0; u < kGroups; ++u)
#pragma unroll
          for (int i = 0; i < kR; ++i) {
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = ex2(fmaf(sc[u][i][e], by[i][e & 1], off[i][e & 1]));
            l[i][0] += v[0] + v[2];
            l[i][1] += v[1] + v[3];
            pb[u][i][0] = transpose8(pack_f16(v[0], v[1]));
            pb[u][i][1] = transpose8(pack_f16(v[2], v[3]));
          }

        // O^T += V^T P^T: rows are elements, 4 (N g + w) on from the word's
#pragma unroll
        for (int u = 0; u < kGroups; ++u) {
          const uint32_t a_at = at + 2 * u * kv4_tile(N), b_at = a_at + kv4_tile(N);
          uint32_t wa[N], wb[N], sa, oa, sb, ob;
          load_words<N>(wa, a_at + v_at);
          load_words<N>(wb, b_at + v_at);
#pragma unroll
          for (int w = 0; w < N; ++w) {
            if (w == 0 || (N & (N - 1)) != 0) {
              const uint32_t mk = kv4_value_marks(N, q) + 4 * ((N * g + w) >> 3);
              kv4_value_step(load_u32(a_at + mk), sa, oa);
              kv4_value_step(load_u32(b_at + mk), sb, ob);
            }
            uint32_t a[4], b[4];
            kv4_word(wa[w], sa, oa, a);
            kv4_word(wb[w], sb, ob, b);
#pragma unroll
            for (int i = 0; i < kR; ++i) {
              mma(o[i][2 * w], a[0], a[1], b[0], b[1], pb[u][i][0], pb[u][i][1]);
              mma(o[i][2 * w + 1], a[2], a[3], b[2], b[3], pb[u][i][0], pb[u][i][1]);
            }
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&empty[s]);
      if (++s == C::kStages) {
        s = 0;
        phase ^= 1;
      }
    }

    // ---- join the warps ----
#pragma unroll
    for (int i = 0; i < kR; ++i)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        l[i][e] += __shfl_xor_sync(~0u, l[i][e], 4);
        l[i][e] += __shfl_xor_sync(~0u, l[i][e], 8);
        l[i][e] += __shfl_xor_sync(~0u, l[i][e], 16);
        if (g == 0) {
          ml[(warp * 2 + 0) * kRows + 8 * i + 2 * q + e] = m[i][e];
          ml[(warp * 2 + 1) * kRows + 8 * i + 2 * q + e] = l[i][e];
        }
      }
    // Each warp's outputs beside one another, against its own maxima; a warp
    // without a key in a row has 0 there.
#pragma unroll
    for (int w = 0; w < N; ++w)
#pragma unroll
      for (int i = 0; i < kR; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          *(float4*)(bufs + (warp * kRows + 8 * i + 2 * q + e) * C::kPad + 4 * (N * g + w)) =
              make_float4(o[i][2 * w][e], o[i][2 * w][2 + e], o[i][2 * w + 1][e], o[i][2 * w + 1][2 + e]);
    bar_consumers();
    const bool whole = starts && ends;
    const int slot = blockIdx.x * 2 + (starts ? 1 : 0);
    const bool outside = KV_BAD(g_few4_counts, x.rows >= 1 && x.rows <= kRows && few_inside(p, x, x.row0) && few_inside(p, x, x.row0 + x.rows - 1) &&
                                                   slot < 2 * (int)gridDim.x);
    float* part = p.part + (int64_t)slot * C::kSlot;
    for (int e = tid; e < kRows * (C::kCols / 8); e += kWarps * 32) {
      const int row = e / (C::kCols / 8), col = e % (C::kCols / 8) * 8;
      if (row >= x.rows || outside) continue;
      float top = -INFINITY, sum = 0.f, v[8];
#pragma unroll
      for (int w = 0; w < kWarps; ++w) top = fmaxf(top, ml[w * 2 * kRows + row]);
      const float safe = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float f = ex2(ml[w * 2 * kRows + row] - safe);
        sum = fmaf(ml[(w * 2 + 1) * kRows + row], f, sum);
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
          const float4 z = *(const float4*)(bufs + (w * kRows + row) * C::kPad + col + i);
          v[i] = fmaf(f, z.x, v[i]), v[i + 1] = fmaf(f, z.y, v[i + 1]), v[i + 2] = fmaf(f, z.z, v[i + 2]), v[i + 3] = fmaf(f, z.w, v[i + 3]);
        }
      }
      if (whole) {
        const int abs = x.row0 + row;
        const int64_t tok = r.q0 + abs / p.group, head = (int64_t)x.head * p.group + abs % p.group;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        if (col < p.dim) {
          uint4 w;
          w.x = pack_out(p.f16, v[0] * inv, v[1] * inv);
          w.y = pack_out(p.f16, v[2] * inv, v[3] * inv);
          w.z = pack_out(p.f16, v[4] * inv, v[5] * inv);
          w.w = pack_out(p.f16, v[6] * inv, v[7] * inv);
          *(uint4*)(p.out + 2 * (tok * p.out_tok + head * p.out_head + col)) = w;
        }
        if (p.lse && col == 0) p.lse[tok * p.heads + head] = L::lse(top, sum);
      } else {
        float4* to = (float4*)(part + row * C::kCols + col);
        to[0] = make_float4(v[0], v[1], v[2], v[3]);
        to[1] = make_float4(v[4], v[5], v[6], v[7]);
        if (col == 0) {
          part[kRows * C::kCols + row] = top;
          part[kRows * C::kCols + kRows + row] = sum;
        }
      }
    }
    if (starts && !ends && tid == 0) {
      const int64_t first = range.end - seg - u0;  // the item's first unit
      p.desc[blockIdx.x] = make_int4(r.q0, x.row0, x.head | x.rows << 16, attn_block_of(range, first + cost - 1) - (int)blockIdx.x + 1);
    }
    bar_consumers();
    if (!next_item(seg)) break;
  }
}

// Joins the parts of the item that block c began and did not end: one block per
// (c, row), its four warps a quarter of the parts each.
template <int N, int kR>
__global__ void __launch_bounds__(128) k_attend4_few_join(const __grid_constant__ AttnParams p) {
  using C = Few4Cfg<N, kR>;
  constexpr int kRows = C::kRows, kCols = C::kCols;
  __shared__ float acc[4][kCols], sums[4];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  wait_for_primary();
  const int4 d = p.desc[blockIdx.x];
  const int rows = d.z >> 16, head0 = d.z & 0xFFFF;
  const int parts = KV_BAD(g_few4_counts, d.w >= 0 && d.w <= (int)(gridDim.x - blockIdx.x) && rows <= kRows && head0 < p.kv_heads &&
                                              d.x + (d.y + rows - (d.w > 0)) / p.group < p.tokens)
                        ? 0
                        : d.w;
  // part k: block c's last segment, then the first segments of the following blocks
  const float* const base = p.part + (int64_t)blockIdx.x * 2 * C::kSlot;
  auto slot = [&](int k) { return base + (int64_t)(k == 0 ? 1 : 2 * k) * C::kSlot; };
  for (int row = blockIdx.y; parts != 0 && row < rows; row += gridDim.y) {
    float top = -INFINITY;
    for (int k = lane; k < parts; k += 32) top = fmaxf(top, slot(k)[kRows * kCols + row]);
#pragma unroll
    for (int i = 16; i; i >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, i));
    const float safe = top == -INFINITY ? 0.f : top;
    float v[N], s = 0.f;
#pragma unroll
    for (int c = 0; c < N; ++c) v[c] = 0.f;
#pragma unroll 4
    for (int k = warp; k < parts; k += 4) {
      const float* at = slot(k);
      const float f = ex2(at[kRows * kCols + row] - safe);
      s = fmaf(f, at[kRows * kCols + kRows + row], s);
#pragma unroll
      for (int c = 0; c < N; ++c) v[c] = fmaf(f, at[row * kCols + c * 32 + lane], v[c]);
    }
#pragma unroll
    for (int c = 0; c < N; ++c) acc[warp][c * 32 + lane] = v[c];
    if (lane == 0) sums[warp] = s;
    __syncthreads();
    s = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    const int abs = d.y + row;
    const int64_t tok = d.x + abs / p.group, head = (int64_t)head0 * p.group + abs % p.group;
    const int col = threadIdx.x * 2;
    if (col < p.dim) {
      const float inv = s == 0.f ? 0.f : 1.f / s;
      const float a = (acc[0][col] + acc[1][col]) + (acc[2][col] + acc[3][col]);
      const float b = (acc[0][col + 1] + acc[1][col + 1]) + (acc[2][col + 1] + acc[3][col + 1]);
      *(uint32_t*)(p.out + 2 * (tok * p.out_tok + head * p.out_head + col)) = pack_out(p.f16, a * inv, b * inv);
    }
    if (p.lse && threadIdx.x == 0) p.lse[tok * p.heads + head] = L::lse(top, s);
    __syncthreads();
  }
}

template <int N, int kR>
cudaError_t launch(const AttnParams& p, int rows_hint, int sms, int device, cudaStream_t stream) {
  using C = Few4Cfg<N, kR>;
  static std::atomic<uint64_t> allowed;
  cudaError_t e = kv_allow_smem(k_attend4_few<N, kR>, C::kSmem, device, allowed);
  if (e != cudaSuccess) return e;
  const int blocks = sms * C::kPerSm;
  k_attend4_few<N, kR><<<blocks, kThreads, C::kSmem, stream>>>(p);
  if ((e = cudaGetLastError()) != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(blocks, rows_hint < 1 || rows_hint > C::kRows ? C::kRows : rows_hint);
  cfg.blockDim = dim3(128);
  cfg.stream = stream;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_attend4_few_join<N, kR>, p);
}

template <int N, int kR>
constexpr size_t room() {  // floats of partial results, of an SM's blocks
  return (size_t)Few4Cfg<N, kR>::kPerSm * 2 * Few4Cfg<N, kR>::kSlot;
}

}  // namespace

size_t attend4_few_workspace(int sms) {
  size_t most = room<4, 1>();
  most = most > room<4, 2>() ? most : room<4, 2>();
  most = most > room<8, 1>() ? most : room<8, 1>();
  most = most > room<2, 2>() ? most : room<2, 2>();
  return attn4_part_offset(sms) + (size_t)sms * most * sizeof(float);
}

// Items of 8 rows where no call has more, or where 16 would not leave room for
// the accumulators (more than 4 groups of elements).
cudaError_t launch_attend4_few(const AttnParams& p, int rows_hint, int sms, int device, cudaStream_t stream) {
  const bool two = rows_hint > 8;
  switch (kv4_groups(p.dim)) {
    case 1: return two ? launch<1, 2>(p, rows_hint, sms, device, stream) : launch<1, 1>(p, rows_hint, sms, device, stream);
    case 2: return two ? launch<2, 2>(p, rows_hint, sms, device, stream) : launch<2, 1>(p, rows_hint, sms, device, stream);
    case 3: return two ? launch<3, 2>(p, rows_hint, sms, device, stream) : launch<3, 1>(p, rows_hint, sms, device, stream);
    case 4: return two ? launch<4, 2>(p, rows_hint, sms, device, stream) : launch<4, 1>(p, rows_hint, sms, device, stream);
    case 5: return launch<5, 1>(p, rows_hint, sms, device, stream);
    case 6: return launch<6, 1>(p, rows_hint, sms, device, stream);
    case 7: return launch<7, 1>(p, rows_hint, sms, device, stream);
    default: return launch<8, 1>(p, rows_hint, sms, device, stream);
  }
}

cudaError_t attend4_few_counts(cudaStream_t stream, uint32_t* counts) {
  void* at = nullptr;
  const cudaError_t e = cudaGetSymbolAddress(&at, g_few4_counts);
  return e != cudaSuccess ? e : cudaMemcpyAsync(counts, at, sizeof(g_few4_counts), cudaMemcpyDeviceToHost, stream);
}

}  // namespace mpt
