// Pages of a key/value cache (include/mpt_kv.h): merge of attention parts,
// writes into pages, page bookkeeping and page copies.  All of them move bytes
// and are bound by the memory, or by latency where there is little to move.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "kv_pages.cuh"

namespace cg = cooperative_groups;

namespace mpt {
namespace {

__device__ uint32_t g_pages_counts[kKvCounts];

// ---------------------------------------------------------------------------
// Merge: out = sum_p exp(lse_p - lse) out_p
// ---------------------------------------------------------------------------

// One thread per 16 bytes of the result; the parts' loads are issued together.
// Four parts of 8,192 x 32 rows of 128 bf16: 54 us, 6.3 TB/s (0.93 of the copy
// rate); two of 28 x 32 rows: 2.3 us, a launch.  Above four parts at most four
// parts' loads are in flight and the sums are read twice: 5, 8 and 16 parts of
// 4,096 x 32 rows 45, 58 and 101 us, 0.68, 0.78 and 0.85 of the copy rate.  The
// weights are recomputed by each of a row's threads (n_parts reads that hit L1,
// n_parts exponentials): cheaper than handing them round.
template <int kType>
struct Vec;  // 16 bytes as 32-bit floats and back
template <>
struct Vec<MPT_KV_F32> {
  static constexpr int kN = 4;
  static __device__ __forceinline__ void load(const uint4& u, float* f) {
    f[0] = __uint_as_float(u.x), f[1] = __uint_as_float(u.y), f[2] = __uint_as_float(u.z), f[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ uint4 store(const float* f) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
};
template <>
struct Vec<MPT_KV_BF16> {
  static constexpr int kN = 8;
  static __device__ __forceinline__ void load(const uint4& u, float* f) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) f[2 * i] = __uint_as_float(w[i] << 16), f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
  static __device__ __forceinline__ uint4 store(const float* f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(f[2 * i + 1]), "f"(f[2 * i]));
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <>
struct Vec<MPT_KV_F16> {
  static constexpr int kN = 8;
  static __device__ __forceinline__ void load(const uint4& u, float* f) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __half2float(__ushort_as_half((unsigned short)w[i]));
      f[2 * i + 1] = __half2float(__ushort_as_half((unsigned short)(w[i] >> 16)));
    }
  }
  static __device__ __forceinline__ uint4 store(const float* f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(f[2 * i + 1]), "f"(f[2 * i]));
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

template <int kType, int kParts>
__global__ void __launch_bounds__(256) k_kv_merge(const __grid_constant__ MergeParams p) {
  using V = Vec<kType>;
  const int n = kParts ? kParts : p.n;
  const int64_t all = p.rows * p.vecs;
  for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < all; at += (int64_t)gridDim.x * 256) {
    const int64_t row = all < (1ll << 32) ? (int64_t)((uint32_t)at / (uint32_t)p.vecs) : at / p.vecs;
    if (KV_BAD(g_pages_counts, row >= 0 && row < p.rows && at - row * p.vecs >= 0 && at - row * p.vecs < p.vecs)) continue;
    uint4 u[kParts ? kParts : 1];
    float s[kParts ? kParts : 1];
    float top = -INFINITY, sum = 0.f, acc[V::kN];
#pragma unroll
    for (int i = 0; i < V::kN; ++i) acc[i] = 0.f;
    if constexpr (kParts > 0) {
#pragma unroll
      for (int k = 0; k < kParts; ++k) u[k] = ((const uint4*)p.outs[k])[at];
#pragma unroll
      for (int k = 0; k < kParts; ++k) s[k] = p.lses[k][row];
#pragma unroll
      for (int k = 0; k < kParts; ++k) top = fmaxf(top, s[k]);
    } else {
      for (int k = 0; k < n; ++k) top = fmaxf(top, p.lses[k][row]);
    }
    const float safe = top == -INFINITY ? 0.f : top;
#pragma unroll(kParts ? kParts : 4)
    for (int k = 0; k < n; ++k) {
      const float lse = kParts ? s[kParts ? k : 0] : p.lses[k][row];
      const float f = expf(lse - safe);
      float x[V::kN];
      V::load(kParts ? u[kParts ? k : 0] : ((const uint4*)p.outs[k])[at], x);
      sum += f;
      if (lse != -INFINITY) {  // an empty part's out has no say, whatever it holds
#pragma unroll
        for (int i = 0; i < V::kN; ++i) acc[i] = fmaf(f, x[i], acc[i]);
      }
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int i = 0; i < V::kN; ++i) acc[i] *= inv;
    ((uint4*)p.out)[at] = V::store(acc);
    if (p.lse && at == row * p.vecs) p.lse[row] = top + logf(sum);
  }
}

template <int kType>
cudaError_t merge_of(const MergeParams& p, cudaStream_t stream) {
  const int64_t blocks = (p.rows * p.vecs + 255) / 256;
  const unsigned grid = (unsigned)(blocks < (1 << 30) ? blocks : 1 << 30);
  switch (p.n) {
    case 2: k_kv_merge<kType, 2><<<grid, 256, 0, stream>>>(p); break;
    case 3: k_kv_merge<kType, 3><<<grid, 256, 0, stream>>>(p); break;
    case 4: k_kv_merge<kType, 4><<<grid, 256, 0, stream>>>(p); break;
    default: k_kv_merge<kType, 0><<<grid, 256, 0, stream>>>(p);
  }
  return cudaGetLastError();
}

// ---------------------------------------------------------------------------
// Write: a warp per new token and tensor (keys or values).  31,000 tokens of 8
// heads of 128 into pages of 16: 44 us, 5.8 TB/s; 28 tokens: 3.1 us, a launch and
// three dependent reads (request, page, new values).
// ---------------------------------------------------------------------------

__global__ void __launch_bounds__(128) k_kv_write(const __grid_constant__ WriteParams p) {
  const int lane = threadIdx.x & 31;
  const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (t >= p.tokens) return;
  // the request: how many of q_offsets[1..batch] are at most t, 32 probes at a time
  int lo = 0, hi = p.batch;
  while (lo < hi) {
    const int step = (hi - lo + 31) / 32, j = lo + (lane + 1) * step;
    const int n = __popc(__ballot_sync(~0u, j <= hi && p.q_offsets[j] <= t));
    hi = min(hi, lo + (n + 1) * step - 1);
    lo += n * step;
  }
  if (lo >= p.batch) return;
  const int64_t q0 = p.q_offsets[lo], q1 = p.q_offsets[lo + 1];
  if (t < q0 || t >= q1) return;  // the latter only where offsets decrease
  const int64_t pos = (int64_t)p.kv_lens[lo] - (q1 - q0) + (t - q0);
  if (pos < 0 || pos >> p.page_log2 >= p.width) return;
  const int page = p.table[(int64_t)lo * p.table_stride + (pos >> p.page_log2)];
  if (page < 0 || page >= p.n_pages) return;
  const int64_t slot = pos & ((1 << p.page_log2) - 1);
  if (KV_BAD(g_pages_counts, t < p.tokens && pos >= 0 && pos < (int64_t)p.width << p.page_log2 && slot >> p.page_log2 == 0)) return;
  const uint4* from;
  uint4* to;
  int64_t from_head, to_head;
  if (blockIdx.y == 0) {
    from = (const uint4*)p.k_new + t * p.k_new_tok, from_head = p.k_new_head;
    to = (uint4*)p.k + page * p.k_page + slot * p.k_slot, to_head = p.k_head;
  } else {
    from = (const uint4*)p.v_new + t * p.v_new_tok, from_head = p.v_new_head;
    to = (uint4*)p.v + page * p.v_page + slot * p.v_slot, to_head = p.v_head;
  }
  const int n = p.kv_heads * p.vecs;
#pragma unroll 4
  for (int c = lane; c < n; c += 32) {
    const int head = c / p.vecs, v = c - head * p.vecs;
    to[head * to_head + v] = from[head * from_head + v];
  }
}

// ---------------------------------------------------------------------------
// Page copies: units of up to 16 KB of one page and plane, dealt out to the
// blocks in turn; a block looks up 256 of its units at once and drops those
// without a pair, so that a list that is mostly -1 costs little.  Moving 11,000
// pages of 16 KB in 4 planes: 227 us, 81 % of the DRAM's peak (0.95 of the copy
// rate)
// ---------------------------------------------------------------------------

__global__ void __launch_bounds__(kCopyThreads) k_kv_copy_pages(const __grid_constant__ CopyParams p) {
  __shared__ int64_t from[kCopyThreads], to[kCopyThreads];
  __shared__ int left[kCopyThreads], count;
  const int tid = threadIdx.x;
  const int64_t segs = copy_segments(p.page_bytes), units = (int64_t)p.n * p.planes * segs;
  for (int64_t first = blockIdx.x; first < units; first += (int64_t)gridDim.x * kCopyThreads) {
    if (tid == 0) count = 0;
    __syncthreads();
    const int64_t unit = first + (int64_t)tid * gridDim.x;
    if (unit < units) {
      const int64_t seg = unit % segs, pp = unit / segs;
      const int plane = (int)(pp % p.planes), j = (int)(pp / p.planes);
      const int s = p.src[j], d = p.dst[j];
      if (s >= 0 && s < p.n_pages && d >= 0 && d < p.n_pages && s != d && !KV_BAD(g_pages_counts, j < p.n && plane < p.planes && seg * kCopySeg < p.page_bytes)) {
        const int at = atomicAdd(&count, 1);  // any order: each unit has bytes of its own
        const int64_t base = plane * p.plane_stride + seg * kCopySeg, rest = p.page_bytes - seg * kCopySeg;
        from[at] = base + s * p.page_stride;
        to[at] = base + d * p.page_stride;
        left[at] = rest < kCopySeg ? (int)rest : kCopySeg;
      }
    }
    __syncthreads();
    const int n = count;
    for (int k = 0; k < n; ++k) {
      uint4 v[kCopyVecs];
#pragma unroll
      for (int i = 0; i < kCopyVecs; ++i) {
        const int o = (i * kCopyThreads + tid) * 16;
        if (o < left[k]) v[i] = *(const uint4*)(p.pool + from[k] + o);
      }
#pragma unroll
      for (int i = 0; i < kCopyVecs; ++i) {
        const int o = (i * kCopyThreads + tid) * 16;
        if (o < left[k]) *(uint4*)(p.pool + to[k] + o) = v[i];
      }
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------
// Bookkeeping: one cluster of eight blocks per call, so that counting the free
// pages, ranking them and handing them out are one launch with cluster
// barriers in between.  A warp owns a run of page ids; ranks are its count
// before it (a prefix over the cluster's warps, read from the other blocks'
// shared memory) plus its own ballots.  The counts are whole, so the ranks and
// everything that follows do not depend on the order of anything.
// Bound: launch, cluster barriers and dependent reads; 7 to 10 us with 4,096
// pages, 13 to 24 us with 200,000.  One, two or four blocks are no faster with
// 4,096 pages and take 35, 24 and 18 us for a fork with 65,536 (eight: 13).
// ---------------------------------------------------------------------------

constexpr int kCluster = 8, kBookThreads = 1024, kBookWarps = kBookThreads / 32;
constexpr int kScanWarps = kCluster * kBookWarps;

struct Scan {
  int lo, hi;  // page ids of this warp
};

__device__ __forceinline__ Scan my_run(int n_pages, int warp_of_all, int* per_out = nullptr) {
  const int per = (int)((((int64_t)n_pages + kScanWarps - 1) / kScanWarps + 31) / 32 * 32);
  if (per_out) *per_out = per;
  const int64_t lo = (int64_t)warp_of_all * per;
  Scan s;
  s.lo = lo < n_pages ? (int)lo : n_pages;
  s.hi = lo + per < n_pages ? (int)(lo + per) : n_pages;
  return s;
}

// Whole-block exclusive prefix of one value per thread; *total gets the sum.
__device__ int64_t block_prefix(int64_t v, int64_t* scratch, int64_t* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t inc = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t o = __shfl_up_sync(~0u, inc, d);
    if (lane >= d) inc += o;
  }
  __syncthreads();
  if (lane == 31) scratch[warp] = inc;
  __syncthreads();
  int64_t before = 0, all = 0;
  for (int w = 0; w < kBookWarps; ++w) {
    if (w < warp) before += scratch[w];
    all += scratch[w];
  }
  *total = all;
  return before + inc - v;
}

// Prefix over all warps of the cluster of one count per warp.  `mine` and `all`
// are shared; every thread of the cluster calls it.
__device__ int cluster_prefix(cg::cluster_group& cl, int count, int* mine, int* all, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (lane == 0) mine[warp] = count;
  cl.sync();
  if (threadIdx.x < kScanWarps) all[threadIdx.x] = cl.map_shared_rank(mine, threadIdx.x / kBookWarps)[threadIdx.x % kBookWarps];
  __syncthreads();
  const int me = (int)cl.block_rank() * kBookWarps + warp;
  int before = 0, sum = 0;
  for (int i = lane; i < kScanWarps; i += 32) {
    const int v = all[i];
    sum += v;
    if (i < me) before += v;
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) {
    before += __shfl_xor_sync(~0u, before, d);
    sum += __shfl_xor_sync(~0u, sum, d);
  }
  *total = sum;
  return before;
}

struct BookShared {
  int64_t scratch[kBookWarps];
  int mine[kBookWarps], all[kScanWarps];
  int flags;
  int64_t need;
  int partial;
};

// Whether row r was marked before (marks are bits in the block's shared memory).
__device__ __forceinline__ bool mark(uint32_t* marks, int r) { return atomicOr(&marks[r >> 5], 1u << (r & 31)) >> (r & 31) & 1u; }

template <int OP>
__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kBookThreads) k_kv_book(const __grid_constant__ BookParams p) {
  extern __shared__ uint32_t marks[];  // a bit per row, then the first fresh page of each entry
  __shared__ BookShared sh;
  cg::cluster_group cl = cg::this_cluster();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = (int)cl.block_rank(), gw = rank * kBookWarps + warp;
  const mpt_kv_book& b = p.b;
  const int mask = (1 << p.page_log2) - 1;
  int* const ranks = (int*)(marks + (b.rows + 31) / 32);
  const Scan run = my_run(b.n_pages, gw);
  auto is_page = [&](int id) { return id >= 0 && id < b.n_pages; };
  const int64_t room = (int64_t)b.width << p.page_log2;  // tokens of a full row

  // Free pages of this warp's run.
  int free_here = 0;
  if (OP != kBookFree) {
#pragma unroll 8
    for (int at = run.lo; at < run.hi; at += 32) free_here += __popc(__ballot_sync(~0u, at + lane < run.hi && b.refs[at + lane] <= 0));
  }

  // The first block looks the list over: what each entry needs, and what is wrong.
  if (rank == 0) {
    if (tid == 0) sh.flags = 0;
    for (int i = tid; i < (b.rows + 31) / 32; i += kBookThreads) marks[i] = 0;
    __syncthreads();
    int64_t need_before = 0;
    int flags = 0;
    for (int base = 0; base < p.n; base += kBookThreads) {
      const int j = base + tid;
      int64_t need = 0;
      if (j < p.n) {
        if (OP == kBookFork) {
          const int src = p.l0[j], dst = p.l1[j], keep = p.l2[j];
          if (src < 0 || src >= b.rows || dst < 0 || dst >= b.rows || mark(marks, dst) || b.lens[dst] != 0 || keep < 0 ||
              keep > b.lens[src] || keep > room)
            flags |= MPT_KV_BAD_ROW;
          else
            need = (keep & mask) != 0 && is_page(b.table[(int64_t)src * b.table_stride + (keep >> p.page_log2)]);
        } else {
          const int row = p.l0[j];
          if (row < 0 || row >= b.rows || mark(marks, row)) {
            flags |= MPT_KV_BAD_ROW;
          } else {
            const int64_t len = b.lens[row], more = OP == kBookExtend ? p.l1[j] : 0;
            if (len < 0 || len > room || more < 0)
              flags |= MPT_KV_BAD_ROW;
            else if (len + more > room)
              flags |= MPT_KV_ROW_FULL;
            else
              need = ((len + more + mask) >> p.page_log2) - ((len + mask) >> p.page_log2);
          }
        }
      }
      if (OP != kBookFree) {
        int64_t all;
        const int64_t at = need_before + block_prefix(need, sh.scratch, &all);
        if (j < p.n) ranks[j] = (int)(at < b.n_pages ? at : b.n_pages);
        need_before += all;
      }
    }
    if (flags) atomicOr(&sh.flags, flags);
    if (tid == 0) sh.need = need_before;
  }
  int free_all = 0;
  const int before = cluster_prefix(cl, free_here, sh.mine, sh.all, &free_all);  // a cluster barrier: sh is written
  const BookShared* lead = cl.map_shared_rank(&sh, 0);
  const int64_t need = lead->need;
  int flags = lead->flags;
  if (need > free_all) flags |= MPT_KV_NO_PAGES;
  if (OP == kBookFree) flags &= ~MPT_KV_NO_PAGES;
  // A warp hands its free pages out: the r-th belongs to the last entry whose
  // pages begin at or before r.  Eight pages a lane at a time: the warps of the
  // lowest ids do it all, one after another's reads (a fork of 300 rows with
  // 65,536 pages 19 us one by one).
  if (flags == 0 && OP != kBookFree && __syncthreads_or(before < need)) {
    if (rank != 0) {
      const int* theirs = cl.map_shared_rank(ranks, 0);
      for (int i = tid; i < p.n; i += kBookThreads) ranks[i] = theirs[i];
      __syncthreads();
    }
    int at = before;
    for (int id0 = run.lo; id0 < run.hi && at < need; id0 += 256) {
      int r[8], j[8], x[8], y[8];  // rank (-1: not to give), entry
#pragma unroll
      for (int u = 0; u < 8; ++u) x[u] = id0 + 32 * u + lane < run.hi ? b.refs[id0 + 32 * u + lane] : 1;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const unsigned f = __ballot_sync(~0u, x[u] <= 0);
        r[u] = at + __popc(f & ((1u << lane) - 1u));
        if (x[u] > 0 || r[u] >= need) r[u] = -1;
        at += __popc(f);
        j[u] = 0;
      }
      for (int step = 1 << (31 - __clz(p.n)); step; step >>= 1) {
#pragma unroll
        for (int u = 0; u < 8; ++u)
          if (j[u] + step < p.n && ranks[j[u] + step] <= r[u]) j[u] += step;
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        x[u] = OP == kBookFork ? p.l1[j[u]] : p.l0[j[u]];
        if (OP == kBookFork) y[u] = p.l2[j[u]] >> p.page_log2;
      }
      if (OP == kBookExtend) {
#pragma unroll
        for (int u = 0; u < 8; ++u) y[u] = (int)(((int64_t)b.lens[x[u]] + mask) >> p.page_log2) + r[u] - ranks[j[u]];
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        if (r[u] < 0) continue;
        const int id = id0 + 32 * u + lane;
        if (KV_BAD(g_pages_counts, x[u] >= 0 && x[u] < b.rows && y[u] >= 0 && y[u] < b.width && id < b.n_pages && j[u] < p.n)) continue;
        b.table[(int64_t)x[u] * b.table_stride + y[u]] = id;
        b.refs[id] = 1;
        if (OP == kBookFork) p.copy_dst[j[u]] = id;
      }
    }
  }
  if (OP == kBookFork) cl.sync();  // counts are read above: a row may name a page whose count is 0
  if (flags == 0 && OP != kBookExtend) {
    for (int j = kScanWarps - 1 - gw; j < p.n; j += kScanWarps) {  // the last warps have no pages to hand out
      const int row = OP == kBookFork ? p.l1[j] : p.l0[j];
      if (KV_BAD(g_pages_counts, row >= 0 && row < b.rows && (OP != kBookFork || (p.l0[j] >= 0 && p.l0[j] < b.rows)))) continue;
      const int keep = OP == kBookFork ? p.l2[j] : b.lens[row];
      if (KV_BAD(g_pages_counts, keep >= 0 && keep <= room)) continue;
      int32_t* to = b.table + (int64_t)row * b.table_stride;
      const int32_t* from = OP == kBookFork ? b.table + (int64_t)p.l0[j] * b.table_stride : to;
      // Fork: the full pages, beside which entry `have` is written above if the rest is on a page.
      const int have = OP == kBookFork ? keep >> p.page_log2 : (int)(((int64_t)keep + mask) >> p.page_log2);
      const int part = OP == kBookFork && (keep & mask) != 0 ? from[have] : -1;
      for (int i0 = 0; i0 < b.width; i0 += 256) {
        int id[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) id[u] = i0 + 32 * u + lane < have ? from[i0 + 32 * u + lane] : -1;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const int i = i0 + 32 * u + lane;
          if (is_page(id[u])) atomicAdd(&b.refs[id[u]], OP == kBookFork ? 1 : -1);
          else id[u] = -1;
          if (i < b.width && !(i == have && is_page(part))) to[i] = OP == kBookFork ? id[u] : -1;
        }
      }
      __syncwarp();
      if (lane == 0) {
        b.lens[row] = OP == kBookFork ? keep : 0;
        if (OP == kBookFork) {
          p.copy_src[j] = is_page(part) ? part : -1;
          if (!is_page(part)) p.copy_dst[j] = -1;
        }
      }
    }
  } else if (OP == kBookFork) {
    for (int j = gw * 32 + lane; j < p.n; j += kScanWarps * 32) p.copy_src[j] = p.copy_dst[j] = -1;
  }
  cl.sync();  // nobody reads the first block's shared memory, or a row's old length, any more
  if (OP == kBookExtend && flags == 0)
    for (int j = gw * 32 + lane; j < p.n; j += kScanWarps * 32) {
      if (KV_BAD(g_pages_counts, p.l0[j] >= 0 && p.l0[j] < b.rows && (int64_t)b.lens[p.l0[j]] + p.l1[j] <= room)) continue;
      b.lens[p.l0[j]] += p.l1[j];
    }
  if (OP == kBookFree) {  // the pages that this call freed are counted too
    int n = 0, all;
#pragma unroll 8
    for (int at = run.lo; at < run.hi; at += 32) n += __popc(__ballot_sync(~0u, at + lane < run.hi && b.refs[at + lane] <= 0));
    cluster_prefix(cl, n, sh.mine, sh.all, &all);
    if (gw == 0 && lane == 0) {
      p.status[0] = flags;
      p.status[1] = all;
    }
    cl.sync();
  } else if (gw == 0 && lane == 0) {
    p.status[0] = flags;
    p.status[1] = free_all - (flags ? 0 : (int)need);
  }
}

__global__ void __cluster_dims__(kCluster, 1, 1) __launch_bounds__(kBookThreads) k_kv_compact(const __grid_constant__ BookParams p) {
  __shared__ BookShared sh;
  cg::cluster_group cl = cg::this_cluster();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = (int)cl.block_rank(), gw = rank * kBookWarps + warp, all_threads = kCluster * kBookThreads;
  const mpt_kv_book& b = p.b;
  int per;
  const Scan run = my_run(b.n_pages, gw, &per);
  int live = 0, n_live;
#pragma unroll 8
  for (int at = run.lo; at < run.hi; at += 32) live += __popc(__ballot_sync(~0u, at + lane < run.hi && b.refs[at + lane] > 0));
  int before = cluster_prefix(cl, live, sh.mine, sh.all, &n_live);
  // live pages of id < n_live: those of the warps before the one whose run holds n_live, and a part of its own
  const int border = n_live / per;  // may be past the last warp
  if (warp == 0) {
    int sum = 0;
    for (int i = lane; i < border && i < kScanWarps; i += 32) sum += sh.all[i];
#pragma unroll 8
    for (int at = border * per; at < n_live; at += 32) {
      const int c = __popc(__ballot_sync(~0u, at + lane < n_live && b.refs[at + lane] > 0));
      if (lane == 0) sum += c;
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
    if (lane == 0) sh.partial = sum;
  }
  __syncthreads();
  const int stay = sh.partial, moves = n_live - stay, half = b.n_pages / 2;
  for (int id0 = run.lo; id0 < run.hi; id0 += 256) {
    unsigned f[8];  // eight loads at a time
#pragma unroll
    for (int u = 0; u < 8; ++u) f[u] = __ballot_sync(~0u, id0 + 32 * u + lane < run.hi && b.refs[id0 + 32 * u + lane] > 0);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int id = id0 + 32 * u + lane;
      const bool in = id < run.hi, on = f[u] >> lane & 1u;
      const int ahead = before + __popc(f[u] & ((1u << lane) - 1u));  // live pages of a lower id
      if (in && !on && id < n_live && !KV_BAD(g_pages_counts, id - ahead >= 0 && id - ahead < half)) p.copy_dst[id - ahead] = id;
      if (on && id >= n_live && !KV_BAD(g_pages_counts, ahead - stay >= 0 && ahead - stay < half)) p.copy_src[ahead - stay] = id;
      before += __popc(f[u]);
    }
  }
  for (int k = moves + rank * kBookThreads + tid; k < half; k += all_threads) p.copy_src[k] = p.copy_dst[k] = -1;
  cl.sync();
  for (int k = rank * kBookThreads + tid; k < moves; k += all_threads) {
    if (KV_BAD(g_pages_counts, k < half)) continue;
    const int s = p.copy_src[k], d = p.copy_dst[k];
    if (KV_BAD(g_pages_counts, s >= n_live && s < b.n_pages && d >= 0 && d < n_live)) continue;
    b.refs[d] = b.refs[s];
    b.refs[s] = 0;
  }
  if (gw == 0 && lane == 0) {
    p.status[0] = 0;
    p.status[1] = b.n_pages - n_live;
  }
}

// Table entries of moved pages (id >= the number of live ones): the moves are in
// rising order of the old id, then -1.
__global__ void __launch_bounds__(256) k_kv_remap(const __grid_constant__ BookParams p) {
  wait_for_primary();
  const int n_live = p.b.n_pages - p.status[1], half = p.b.n_pages / 2;
  for (int row = blockIdx.y; row < p.b.rows; row += gridDim.y)
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < p.b.width; i += (int64_t)gridDim.x * 256) {
      int32_t* at = p.b.table + (int64_t)row * p.b.table_stride + i;
      const int id = *at;
      if (id < n_live || id >= p.b.n_pages) continue;
      int lo = 0, hi = half;  // the first move of an old id of at least `id`
      while (lo < hi) {
        const int mid = (lo + hi) / 2, old = p.copy_src[mid];
        if (old >= 0 && old < id) lo = mid + 1;
        else hi = mid;
      }
      if (lo < half && p.copy_src[lo] == id) *at = p.copy_dst[lo];
    }
}

template <int OP>
cudaError_t book(const BookParams& p, cudaStream_t stream) {
  const size_t smem = (size_t)(p.b.rows + 31) / 32 * 4 + (OP == kBookFree ? 0 : (size_t)p.n * 4);
  cudaError_t e = cudaSuccess;
  // the most that a call may need, whatever this one does: another thread's call may be between its own two steps
  constexpr int kMost = (1 << 20) / 8 + kBookList * 4;
  if (smem > 40 * 1024) e = cudaFuncSetAttribute(k_kv_book<OP>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
  if (e != cudaSuccess) return e;
  k_kv_book<OP><<<kCluster, kBookThreads, smem, stream>>>(p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_kv_merge(const MergeParams& p, int type, cudaStream_t stream) {
  if (type == MPT_KV_F32) return merge_of<MPT_KV_F32>(p, stream);
  return type == MPT_KV_F16 ? merge_of<MPT_KV_F16>(p, stream) : merge_of<MPT_KV_BF16>(p, stream);
}

cudaError_t launch_kv_write(const WriteParams& p, cudaStream_t stream) {
  k_kv_write<<<dim3((unsigned)((p.tokens + 3) / 4), 2), 128, 0, stream>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_kv_copy_pages(const CopyParams& p, cudaStream_t stream) {
  const int64_t segs = copy_segments(p.page_bytes), units = (int64_t)p.n * p.planes * segs;
  const int64_t most = sm_count() * 8;
  k_kv_copy_pages<<<(unsigned)(units < most ? units : most), kCopyThreads, 0, stream>>>(p);
  return cudaGetLastError();
}

cudaError_t launch_kv_book(const BookParams& p, BookOp op, cudaStream_t stream) {
  if (op == kBookFork) return book<kBookFork>(p, stream);
  if (op == kBookExtend) return book<kBookExtend>(p, stream);
  if (op == kBookFree) return book<kBookFree>(p, stream);
  k_kv_compact<<<kCluster, kBookThreads, 0, stream>>>(p);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || p.b.rows == 0) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((p.b.width + 255) / 256, p.b.rows < 32768 ? p.b.rows : 32768);
  cfg.blockDim = dim3(256);
  cfg.stream = stream;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_kv_remap, p);
}

cudaError_t kv_pages_counts(cudaStream_t stream, uint32_t* counts) {
  void* at = nullptr;
  const cudaError_t e = cudaGetSymbolAddress(&at, g_pages_counts);
  return e != cudaSuccess ? e : cudaMemcpyAsync(counts, at, sizeof(g_pages_counts), cudaMemcpyDeviceToHost, stream);
}

}  // namespace mpt
