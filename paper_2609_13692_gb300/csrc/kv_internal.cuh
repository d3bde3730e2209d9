// Internal declarations of the paged-cache operators (include/mpt_kv.h).
#pragma once

#include <atomic>

#include <cuda.h>

#include "../../include/mpt_kv.h"
#include "mpt_internal.cuh"

namespace mpt {

// Attention over a paged cache, as both kernels take it.  The tensor maps are
// 4-d: (element of the head, slot of the page, KV head, page).
struct alignas(128) AttnParams {
  CUtensorMap map_k, map_v, map_q;
  const char *q, *k, *v;
  char* out;
  float* lse;  // [tokens][heads] or nullptr
  int64_t q_tok, q_head, out_tok, out_head;  // strides in elements
  int64_t k_page, k_slot, k_head, v_page, v_slot, v_head;
  const int32_t* table;
  int64_t table_stride;
  const int32_t* q_offsets;
  const int32_t* kv_lens;
  float* part;  // partial results, see each kernel
  int4* desc;   // one per block: what its last, unfinished item is
  int64_t tokens;
  int32_t width, n_pages, page_log2, batch, heads, kv_heads, group, dim, causal;
  int32_t box, toks, item_toks;  // page slots per copy; whole tokens of 128 rows, and of an item
  int32_t wide;                  // out's heads are whole 32-byte pieces
  float scale_log2;  // scale * log2(e)
};

// Multiprocessors of the current device, asked once per device.
inline int kv_sm_count(int* device) {
  static std::atomic<int> known[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
    *device = 0;
    return (int)sm_count();
  }
  *device = dev;
  int n = known[dev].load(std::memory_order_relaxed);
  if (n == 0) known[dev].store(n = (int)sm_count(), std::memory_order_relaxed);
  return n;
}

// A kernel's limit of dynamic shared memory, raised once per device.  `done` is
// the kernel's own, a bit per device.
template <typename Kernel>
cudaError_t kv_allow_smem(Kernel kernel, int bytes, int device, std::atomic<uint64_t>& done) {
  const uint64_t bit = 1ull << (device & 63);
  if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

// Events that kernels count on a device, for mpt_kv_check; nothing clears them.
enum KvCount {
  kKvGaveUp,   // waits that gave up
  kKvOutside,  // bounds-checked build: indices that failed their check
  kKvCounts
};

// Bounds-checked build: counts an index that is out of range; the caller then
// skips the access.  The constant false in the default build.
#ifdef MPT_BOUNDS
#define KV_BAD(counts, ok) (!(ok) && (atomicAdd(&(counts)[::mpt::kKvOutside], 1u), true))
#else
#define KV_BAD(counts, ok) false
#endif

// One request's lengths, clamped to what the token axis and the table hold.
struct AttnReq {
  int q0, ql, kvl;  // first token, new tokens, keys
};

__device__ __forceinline__ AttnReq attn_req(const AttnParams& p, int i) {
  AttnReq r;
  const int64_t a = p.q_offsets[i], b = p.q_offsets[i + 1];
  const int64_t q0 = a < 0 ? 0 : a > p.tokens ? p.tokens : a;
  const int64_t q1 = b < q0 ? q0 : b > p.tokens ? p.tokens : b;
  const int64_t most = (int64_t)p.width << p.page_log2;
  const int64_t l = p.kv_lens[i];
  r.q0 = (int)q0;
  r.ql = (int)(q1 - q0);
  r.kvl = (int)(l < 0 ? 0 : l > most ? most : l);
  return r;
}

// Offsets that decrease could give many requests the same tokens, and a call
// more work than its tensors can hold: such a call does nothing.
__device__ __forceinline__ bool attn_falls(const AttnParams& p, int i) { return p.q_offsets[i + 1] < p.q_offsets[i]; }

// Bounds-checked build: an item's request and rows lie in the call's tensors.
__device__ __forceinline__ bool attn_inside(const AttnParams& p, int req, int head, int q0, int ql, int kvl) {
  return req >= 0 && req < p.batch && head >= 0 && head < p.kv_heads && q0 >= 0 && ql > 0 && (int64_t)q0 + ql <= p.tokens && kvl >= 0 &&
         kvl <= (int64_t)p.width << p.page_log2;
}

// Keys that token t of the request may see: j < the returned value.
__device__ __forceinline__ int attn_limit(const AttnParams& p, const AttnReq& r, int t) {
  if (!p.causal) return r.kvl;
  const int64_t lim = (int64_t)r.kvl - r.ql + t + 1;
  return lim < 0 ? 0 : lim > r.kvl ? r.kvl : (int)lim;
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, int x, int y, int z, int w,
                                            unsigned long long* bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], "
      "[%6];" ::"r"(smem_u32(dst)),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar))
      : "memory");
}

__device__ __forceinline__ unsigned long long now_ns() {
  unsigned long long t;
  asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
  return t;
}

// Bounded wait of one thread: false once the block has given up, or after four
// seconds (which it then counts).  The clock is looked at after the first polls
// only: reading it takes longer than most waits.
__device__ __forceinline__ bool wait_bar(unsigned long long* bar, uint32_t parity, int* gave_up, uint32_t* counts) {
  unsigned long long start = 0;
  for (;;) {
    for (int i = 0; i < 256; ++i)
      if (mbar_try_wait(bar, parity)) return true;
    const unsigned long long now = now_ns();
    if (start == 0) start = now;
    if (*(volatile int*)gave_up) return false;
    if (now - start > 4000000000ull) {
      *(volatile int*)gave_up = 1;
      atomicAdd(&counts[kKvGaveUp], 1u);
      return false;
    }
  }
}

// For copies in flight when a block ends early: a second at most.
__device__ __forceinline__ void wait_landed(unsigned long long* bar, uint32_t parity) {
  unsigned long long start = 0;
  while (!mbar_try_wait(bar, parity)) {
    const unsigned long long now = now_ns();
    if (start == 0) start = now;
    if (now - start > 1000000000ull) return;
  }
}

__device__ __forceinline__ void launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_primary() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// Work of both attention kernels is a line of units: the requests in order,
// the items of each (a KV head and a tile of query rows), and the key tiles of
// an item.  Block c of nc takes units [total c / nc, total (c + 1) / nc), so
// every block reads the same number of key tiles whatever the lengths; an item
// cut by a block's border leaves partial results, which a second kernel joins.
struct AttnRange {
  int64_t total, begin, end;
  int nc;       // blocks that have work
  int req;      // request of unit `begin`
  int64_t off;  // its place in that request
};

// All threads of the block call it; `scratch` holds 40 int64.  units(i): units
// of request i; where one is negative, or the line is too long for its products
// with the number of blocks, there is no work.
constexpr int64_t kMostUnits = 1ll << 53;
template <int kThreads, typename Units>
__device__ AttnRange attn_range(int batch, int block, int blocks, int64_t* scratch, Units units) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  constexpr int kWarps = kThreads / 32;
  const int per = (batch + kThreads - 1) / kThreads;
  const int lo = tid * per < batch ? tid * per : batch, hi = lo + per < batch ? lo + per : batch;
  int64_t sum = 0;
  bool bad = false;
  for (int i = lo; i < hi; ++i) {
    const int64_t u = units(i);
    bad |= u < 0;
    sum = sum + u < kMostUnits ? sum + u : kMostUnits;
  }
  int64_t inc = sum;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t v = __shfl_up_sync(~0u, inc, d);
    if (lane >= d) inc += v;
  }
  if (lane == 31) scratch[warp] = inc;
  bad = __syncthreads_or(bad);
  int64_t before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) before += scratch[w];
    total += scratch[w];
  }
  if (bad || total >= kMostUnits) total = 0;
  AttnRange r;
  r.total = total;
  r.nc = total < blocks ? (int)total : blocks;
  r.begin = r.end = 0;
  r.req = 0;
  r.off = 0;
  if (block >= r.nc) return r;  // uniform
  r.begin = total * block / r.nc;
  r.end = total * (block + 1) / r.nc;
  int64_t at = before + inc - sum;
  if (at <= r.begin && r.begin < at + sum) {
    int i = lo;
    for (; i < hi - 1; ++i) {
      const int64_t u = units(i);
      if (r.begin < at + u) break;
      at += u;
    }
    scratch[38] = i;
    scratch[39] = r.begin - at;
  }
  __syncthreads();
  r.req = (int)scratch[38];
  r.off = scratch[39];
  return r;
}

// The block that unit u belongs to.
__device__ __forceinline__ int attn_block_of(const AttnRange& r, int64_t u) {
  return (int)(((u + 1) * r.nc + r.total - 1) / r.total) - 1;
}

// f16 has no bits below 2^-24: of a probability against a reference of 1 the
// product with the values would see nothing below 2^-25, but the sum would, and
// many keys in such a tail would lose their weight.  So f16 probabilities are
// rounded at 2^kLift times their value, of which output and sum are both made;
// references are whole numbers there, so the lift adds no rounding.  The largest
// probability, 2^kLag above the reference in the kernel that rescales seldom,
// stays below 2^16.
template <bool F16, int kLag>
struct Lift {
  static constexpr float kLift = F16 ? 15 - kLag : 0;
  static __device__ __forceinline__ float reference(float top) { return F16 ? ceilf(top) : top; }
  static __device__ __forceinline__ float lse(float top, float sum) {
    return (top + log2f(sum) - kLift) * 0.6931471805599453f;
  }
};

// Few query rows per KV head (k_attend_few.cu): bytes of workspace and launch.
constexpr int kFewPerSm = 3;  // blocks per SM, at most
size_t attend_few_workspace(int sms);
cudaError_t launch_attend_few(const AttnParams& p, bool f16, int rows_hint, int sms, int device, cudaStream_t stream);
// The kernels' counts, read in the stream's order.
cudaError_t attend_few_counts(cudaStream_t stream, uint32_t* counts);

// Whole tiles of query rows on tcgen05 (k_attend_tile.cu); at
// most kTileBatch requests (its list of them, 16 bytes each, is in the room of
// the ring of slots).
constexpr int kTileBatch = 8192;
size_t attend_tile_workspace(int sms);
cudaError_t launch_attend_tile(const AttnParams& p, bool f16, int sms, int device, cudaStream_t stream);
cudaError_t attend_tile_counts(cudaStream_t stream, uint32_t* counts);

}  // namespace mpt
