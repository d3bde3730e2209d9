// Attention over a paged cache for few query rows per KV head (include/mpt_kv.h,
// mpt_kv_attend): single new tokens.  (It is right for any number of rows, and
// takes the calls of more than kTileBatch requests too.)
//
// For a KV head, the rows are its query heads' tokens, 16 to a tile: row
// (t, g) = token t, g-th query head of the KV head.  With s_j = scale q.k_j the
// running form over key tiles keeps per row m = max s_j, l = sum exp(s_j - m),
// o = sum exp(s_j - m) v_j; (m, l, o) of two sets of keys join to
// m' = max(m1, m2), l' = sum_i l_i exp(m_i - m'), o' likewise, so warps and
// blocks take disjoint keys and join once at the end.
//
// Bound: the cache is read once, 2 L Hkv d elements, for 4 d operations per
// element and query head of the group: with up to 16 rows that is below what
// the memory allows a tensor core to do, so the kernel is built around the
// copy.  A warp issues tensor-map copies of pages into a ring of stages (64 keys
// of K and V each); four others take 16 keys of a stage apiece through ldmatrix
// and m16n8k16 products with 32-bit accumulators, without a barrier among them
// until the item's end.  Two or three such blocks share an SM, so that one's
// reads of queries and joins do not hold up the other's products (200 requests
// of 200 to 400 keys: 57 us, 78 with one block of eight such warps).
//
// Measured (one GB300, 8 KV heads of 128): 3 requests of 100,001 to 131,072 keys,
// pages of 64: 203 us, 6.6 TB/s, 0.97 of the measured copy rate; 28 of 2,000 to
// 6,000, pages of 16: 79 us, 5.8 TB/s, 12 us of it start, end and join (16 KV heads
// of 64, 64 requests: 207 us, 5.2 TB/s; 8 of 256: 148 us, 6.2 TB/s); one of 777:
// 9.8 us, launches and a chain of dependent reads.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "kv_internal.cuh"

namespace mpt {
namespace {

__device__ uint32_t g_few_counts[kKvCounts];

constexpr int kKeys = 64;      // keys of a stage
constexpr int kRows = 16;      // query rows of an item

template <int HDP>
struct FewCfg {
  static constexpr int kPerSm = HDP == 64 ? 3 : HDP == 128 ? 2 : 1;  // blocks: an item's end in one, products in another
  static constexpr int kWarps = 4;                                   // each 16 keys of a stage
  // One warp issues a copy every 95 cycles or so: with pages of 16 (2 KB each)
  // that is 21 bytes a cycle, where an SM's share of the memory is 23.
  static constexpr int kCopyWarps = HDP == 256 ? 3 : 1;
  static constexpr int kThreads = 32 * (kWarps + kCopyWarps);
  static constexpr int kStage = 2 * kKeys * HDP * 2;
  // A stage always belongs to one copying warp, and every warp of products waits
  // for every stage: each sees all of a barrier's phases in order.  (A wait for
  // a phase before the one at hand is complete would pass at once.)
  static constexpr int kStages = HDP == 64 ? 4 : 3;
  static_assert(kStages % kCopyWarps == 0);
  static constexpr int kPad = HDP + 8;               // row of the joining buffer, in floats
  static constexpr int kBuf = kRows * kPad * 4;
  static constexpr int kQPad = HDP + 8;              // row of the staged queries (HDP 256)
  static constexpr int kQ = HDP == 256 ? kRows * kQPad * 2 : 0;
  static constexpr int kMl = kWarps * 2 * kRows * 4;
  static constexpr int kSmem = 1024 + kStages * kStage + kBuf + kQ + kMl + 128 + 320;
};

template <bool F16>
__device__ __forceinline__ void mma16816(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  if (F16)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void ldsm4(uint32_t* r, uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr));
}
__device__ __forceinline__ void ldsm4t(uint32_t* r, uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr));
}

template <bool F16>
using L = Lift<F16, 0>;

template <bool F16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  uint32_t r;
  if (F16)
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  else
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}

template <bool F16>
__device__ __forceinline__ float to_float(uint16_t x) {
  return F16 ? __half2float(__ushort_as_half(x)) : __uint_as_float((uint32_t)x << 16);
}

// Whether one of the two elements is an infinity or a NaN.
template <bool F16>
__device__ __forceinline__ bool not_finite2(uint32_t x) {
  constexpr uint32_t e = F16 ? 0x7C00u : 0x7F80u;
  return (x & e) == e || (x >> 16 & e) == e;
}

__device__ __forceinline__ void bar_consumers(int threads) { asm volatile("bar.sync 1, %0;" ::"r"(threads) : "memory"); }

// One item: rows of one KV head of one request.
struct FewItem {
  int req, head, row0, rows;  // rows: valid ones of the 16
  AttnReq r;
  int tiles;  // key tiles that any of its rows sees
};

__device__ __forceinline__ int row_tiles(const AttnParams& p, const AttnReq& r) {
  return (int)(((int64_t)r.ql * p.group + kRows - 1) / kRows);
}
// Key tiles of n keys (n + kKeys may not fit in 32 bits).
__device__ __forceinline__ int tiles_of(int n) { return n < 1 ? 0 : (n - 1) / kKeys + 1; }
__device__ __forceinline__ int key_tiles(const AttnReq& r) {
  const int n = tiles_of(r.kvl);
  return n < 1 ? 1 : n;
}

__device__ __forceinline__ FewItem few_item(const AttnParams& p, const AttnReq& r, int req, int64_t item, int rt) {
  FewItem it;
  it.req = req;
  it.head = (int)(item / rt);
  it.row0 = (int)(item % rt) * kRows;
  const int64_t left = (int64_t)r.ql * p.group - it.row0;
  it.rows = left < kRows ? (int)left : kRows;
  it.r = r;
  it.tiles = tiles_of(attn_limit(p, r, (it.row0 + it.rows - 1) / p.group));
  return it;
}

// Bounds-checked build: row `row` of the item's request lies in the call's tensors.
__device__ __forceinline__ bool few_inside(const AttnParams& p, const FewItem& x, int row) {
  return attn_inside(p, x.req, x.head, x.r.q0, x.r.ql, x.r.kvl) && row >= 0 && row / p.group < x.r.ql;
}

template <int HDP, bool F16>
__global__ void __launch_bounds__(FewCfg<HDP>::kThreads, FewCfg<HDP>::kPerSm) k_attend_few(const __grid_constant__ AttnParams p) {
  using C = FewCfg<HDP>;
  extern __shared__ char raw[];
  char* base = (char*)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
  char* ring = base;
  float* bufs = (float*)(base + C::kStages * C::kStage);
  uint16_t* qs = (uint16_t*)((char*)bufs + C::kBuf);
  float* ml = (float*)((char*)qs + C::kQ);  // [kWarps][2][kRows]
  unsigned long long* full = (unsigned long long*)((char*)ml + C::kMl);
  unsigned long long* empty = full + C::kStages;
  uint32_t* there = (uint32_t*)(empty + C::kStages);  // per stage: which groups of 8 keys the cache holds
  int64_t* scratch = (int64_t*)((char*)ml + C::kMl + 128);
  __shared__ int gave_up;

  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 4);
    }
    gave_up = 0;
    mbar_init_fence();
  }
  if (tid == 32) {  // the maps are read a good while before the first copy
    asm volatile("prefetch.tensormap [%0];" ::"l"(&p.map_k));
    asm volatile("prefetch.tensormap [%0];" ::"l"(&p.map_v));
  }
  launch_dependents();
  const AttnRange range = attn_range<C::kThreads>(p.batch, blockIdx.x, gridDim.x, scratch, [&](int i) -> int64_t {
    if (attn_falls(p, i)) return -1;
    const AttnReq r = attn_req(p, i);
    return (int64_t)p.kv_heads * row_tiles(p, r) * key_tiles(r);
  });
  if (tid == 0) p.desc[blockIdx.x] = make_int4(0, 0, 0, 0);
  if (range.begin >= range.end) return;
  __syncthreads();

  int req = range.req;
  AttnReq r = attn_req(p, req);
  int rt = row_tiles(p, r), cost = key_tiles(r);
  int64_t item = range.off / cost;
  int t0 = (int)(range.off % cost);
  int64_t left = range.end - range.begin;
  uint32_t it = 0;  // stages used so far (the products' count)

  if (warp >= C::kWarps) {
    // ---- copies: the warps take stages in turn ----
    const uint32_t me = warp - C::kWarps;
    const int per = kKeys >> p.page_log2 > 0 ? kKeys >> p.page_log2 : 1;  // boxes of a stage along the keys
    const int box = p.box;                                                // keys of one
    constexpr int kBlk = HDP / 64;
    bool ok = true;
    uint32_t it0 = 0, done = 0;  // stages before the item; this warp's last use and one
    while (left > 0 && ok) {
      const FewItem x = few_item(p, r, req, item, rt);
      const int seg = (int)(left < cost - t0 ? left : cost - t0);
      const int last = t0 + seg < x.tiles ? t0 + seg : x.tiles;
      const int32_t* row = p.table + (int64_t)req * p.table_stride;
      auto page_of = [&](int t, int sub) -> int {
        const int64_t key = (int64_t)t * kKeys + sub * box;
        if (t >= last || key >= r.kvl) return -1;
        const int id = row[key >> p.page_log2];
        return id < 0 || id >= p.n_pages ? -1 : id;
      };
      const int mine = lane % per;  // per is a power of two of at most 8
      // this warp's next tile, and its pages ahead of need
      int t = t0 + (int)((me + C::kCopyWarps - it0 % C::kCopyWarps) % C::kCopyWarps);
      int next = page_of(t, mine);
      for (; t < last; t += C::kCopyWarps) {
        const uint32_t it = it0 + (uint32_t)(t - t0);
        const int s = it % C::kStages;
        const int id = next;
        next = page_of(t + C::kCopyWarps, mine);
        if (it >= C::kStages) {  // a stage that was handed back by warps that gave up may still be filling
          ok = __all_sync(~0u, wait_bar(&empty[s], (it / C::kStages - 1) & 1, &gave_up, g_few_counts) && *(volatile int*)&gave_up == 0);
          if (!ok) break;
        }
        const unsigned held = __ballot_sync(~0u, id >= 0);  // bit q: box q % per
        if (lane == 0) {
          uint32_t m = 0;
          for (int g = 0; g < kKeys / 8; ++g) m |= (held >> (g * 8 / box) & 1u) << g;
          there[s] = m;
          mbar_arrive_expect_tx(&full[s], C::kStage);
        }
        __syncwarp();
        char* dst = ring + s * C::kStage;
        const int slot = ((t * kKeys) & ((1 << p.page_log2) - 1));  // pages larger than a stage
        for (int q = lane; q < per * kBlk * 2; q += 32) {
          const int b = q / per % kBlk, v = q / per / kBlk;
          if (KV_BAD(g_few_counts, id >= -1 && id < p.n_pages && x.head < p.kv_heads && slot < 1 << p.page_log2 && b < kBlk)) continue;
          tma_load_4d(dst + v * (C::kStage / 2) + b * kKeys * 128 + mine * box * 128, v ? &p.map_v : &p.map_k, b * 64,
                      slot, x.head, id, &full[s]);
        }
        done = it + 1;
      }
      if (!ok) break;
      if (last > t0) it0 += last - t0;
      left -= seg;
      t0 = 0;
      if (++item == (int64_t)p.kv_heads * rt) {
        item = 0;
        do {
          if (++req >= p.batch) break;
          r = attn_req(p, req);
          rt = row_tiles(p, r);
          cost = key_tiles(r);
        } while (rt == 0);
        if (req >= p.batch) break;
      }
    }
    // The block ends after this warp's copies have landed, also where the warps
    // that take them have given up.  (Its last use of a stage is that stage's
    // last phase.)
    for (uint32_t k = done > C::kStages ? done - C::kStages : 0; k < done; ++k)
      if (k % C::kCopyWarps == me) wait_landed(&full[k % C::kStages], (k / C::kStages) & 1);
    return;
  }

  // ---- products ----
  const int key0 = warp * 16;
  const int g = lane >> 2, c2 = (lane & 3) * 2;
  constexpr int kK = HDP / 16;
  while (left > 0) {
    const FewItem x = few_item(p, r, req, item, rt);
    const int seg = (int)(left < cost - t0 ? left : cost - t0);
    const int last = t0 + seg < x.tiles ? t0 + seg : x.tiles;
    const bool starts = t0 == 0, ends = t0 + seg == cost;

    // query rows g and g + 8 of this thread, and what they may see
    int lim[2];
    const char* qrow[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = x.row0 + g + 8 * h;
      const bool valid = g + 8 * h < x.rows && !KV_BAD(g_few_counts, few_inside(p, x, row));
      lim[h] = valid ? attn_limit(p, r, row / p.group) : 0;
      qrow[h] = valid ? p.q + 2 * ((int64_t)(r.q0 + row / p.group) * p.q_tok +
                                   ((int64_t)x.head * p.group + row % p.group) * p.q_head)
                      : nullptr;
    }
    const int lim_lo = attn_limit(p, r, x.row0 / p.group);  // what every valid row sees
    uint32_t qf[HDP <= 128 ? kK : 1][4];
    if (HDP <= 128) {
#pragma unroll
      for (int k = 0; k < kK; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int col = k * 16 + c2 + (e >> 1) * 8;
          const char* q = qrow[e & 1];
          qf[k][e] = q && col < p.dim ? *(const uint32_t*)(q + 2 * col) : 0u;
        }
    } else {
      for (int e = tid; e < kRows * (HDP / 8); e += C::kWarps * 32) {
        const int row = e / (HDP / 8), col = e % (HDP / 8) * 8, abs = x.row0 + row;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (row < x.rows && col < p.dim && !KV_BAD(g_few_counts, few_inside(p, x, abs)))
          v = *(const uint4*)(p.q + 2 * ((int64_t)(r.q0 + abs / p.group) * p.q_tok +
                                         ((int64_t)x.head * p.group + abs % p.group) * p.q_head + col));
        *(uint4*)(qs + row * C::kQPad + col) = v;
      }
      bar_consumers(C::kWarps * 32);
    }

    float o[HDP / 8][4];
#pragma unroll
    for (int n = 0; n < HDP / 8; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) o[n][e] = 0.f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};

    for (int t = t0; t < last; ++t, ++it) {
      const int s = it % C::kStages;
      // having given up, the block still ends in order
      (void)__all_sync(~0u, wait_bar(&full[s], (it / C::kStages) & 1, &gave_up, g_few_counts));
      const uint32_t kbase = smem_u32(ring + s * C::kStage), vbase = kbase + C::kStage / 2;

      // S = Q K^T for 16 keys
      float sc[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
      {
        const int row = key0 + (lane & 7) + ((lane >> 4) << 3);
#pragma unroll
        for (int k = 0; k < kK; ++k) {
          const int ch = k * 2 + ((lane >> 3) & 1);
          uint32_t b[4], a[4];
          ldsm4(b, kbase + (ch >> 3) * (kKeys * 128) + row * 128 + (((ch & 7) ^ (row & 7)) << 4));
          if (HDP <= 128) {
#pragma unroll
            for (int e = 0; e < 4; ++e) a[e] = qf[HDP <= 128 ? k : 0][e];
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              a[e] = *(const uint32_t*)(qs + (g + 8 * (e & 1)) * C::kQPad + k * 16 + c2 + (e >> 1) * 8);
          }
          mma16816<F16>(sc[0], a, b[0], b[1]);
          mma16816<F16>(sc[1], a, b[2], b[3]);
        }
      }

      const uint32_t held = there[s];
      const bool partly = lim_lo - t * kKeys < kKeys || held != 0xFFu;
      if (partly) {
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int col = key0 + n * 8 + c2 + (e & 1);
            if (t * kKeys + col >= lim[e >> 1] || !(held >> (col >> 3) & 1u)) sc[n][e] = -INFINITY;
          }
      }
      float alpha[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float mx = fmaxf(fmaxf(sc[0][2 * h], sc[0][2 * h + 1]), fmaxf(sc[1][2 * h], sc[1][2 * h + 1]));
        mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(~0u, mx, 2));
        const float mn = L<F16>::reference(fmaxf(m[h], mx * p.scale_log2));
        const float safe = mn == -INFINITY ? 0.f : mn;
        alpha[h] = ex2(m[h] - safe);
        m[h] = mn;
        float sum = 0.f;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float v = ex2(fmaf(sc[n][2 * h + e], p.scale_log2, L<F16>::kLift - safe));
            sc[n][2 * h + e] = v;
            sum += v;
          }
        l[h] = l[h] * alpha[h] + sum;
      }
      if (__any_sync(~0u, alpha[0] != 1.f || alpha[1] != 1.f)) {
#pragma unroll
        for (int n = 0; n < HDP / 8; ++n) {
          o[n][0] *= alpha[0];
          o[n][1] *= alpha[0];
          o[n][2] *= alpha[1];
          o[n][3] *= alpha[1];
        }
      }

      // A masked key's value may be an infinity or a NaN, and 0 times it is not
      // 0: such a group of 16 keys is added key by key, without the masked ones.
      bool odd = false;
      if (partly) {
        for (int e = lane; e < 16 * (HDP / 8); e += 32) {
          const int row = key0 + (e & 15), ch = e >> 4;
          uint4 v;
          asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                       : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                       : "r"(vbase + (ch >> 3) * (kKeys * 128) + row * 128 + (((ch & 7) ^ (row & 7)) << 4)));
          odd |= not_finite2<F16>(v.x) || not_finite2<F16>(v.y) || not_finite2<F16>(v.z) || not_finite2<F16>(v.w);
        }
        odd = __any_sync(~0u, odd);
      }
      if (odd) {
        for (int j = 0; j < 16; ++j) {
          const int row = key0 + j, from = (lane & ~3) | ((j & 7) >> 1);
          float pj[2];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const float lo = __shfl_sync(~0u, sc[0][2 * h + 0], from), hi = __shfl_sync(~0u, sc[0][2 * h + 1], from);
            const float lo1 = __shfl_sync(~0u, sc[1][2 * h + 0], from), hi1 = __shfl_sync(~0u, sc[1][2 * h + 1], from);
            pj[h] = j < 8 ? (j & 1 ? hi : lo) : (j & 1 ? hi1 : lo1);
          }
          const bool here = held >> (row >> 3) & 1u;
          const bool on0 = here && t * kKeys + row < lim[0], on1 = here && t * kKeys + row < lim[1];
#pragma unroll
          for (int n = 0; n < HDP / 8; ++n) {
            uint32_t v;
            asm volatile("ld.shared.u32 %0, [%1];"
                         : "=r"(v)
                         : "r"(vbase + (n >> 3) * (kKeys * 128) + row * 128 + (((n & 7) ^ (row & 7)) << 4) + c2 * 2));
            const float v0 = to_float<F16>((uint16_t)v), v1 = to_float<F16>((uint16_t)(v >> 16));
            if (on0) {
              o[n][0] = fmaf(pj[0], v0, o[n][0]);
              o[n][1] = fmaf(pj[0], v1, o[n][1]);
            }
            if (on1) {
              o[n][2] = fmaf(pj[1], v0, o[n][2]);
              o[n][3] = fmaf(pj[1], v1, o[n][3]);
            }
          }
        }
      } else {
        // O += P V, P rounded to the cache's type (the operand's; sums stay 32-bit)
        const uint32_t a[4] = {pack2<F16>(sc[0][0], sc[0][1]), pack2<F16>(sc[0][2], sc[0][3]),
                               pack2<F16>(sc[1][0], sc[1][1]), pack2<F16>(sc[1][2], sc[1][3])};
        const int row = key0 + (lane & 15);
#pragma unroll
        for (int n = 0; n < HDP / 16; ++n) {
          const int ch = n * 2 + (lane >> 4);
          uint32_t b[4];
          ldsm4t(b, vbase + (ch >> 3) * (kKeys * 128) + row * 128 + (((ch & 7) ^ (row & 7)) << 4));
          mma16816<F16>(o[2 * n], a, b[0], b[1]);
          mma16816<F16>(o[2 * n + 1], a, b[2], b[3]);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&empty[s]);
    }

    // ---- join the warps ----
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      l[h] += __shfl_xor_sync(~0u, l[h], 1);
      l[h] += __shfl_xor_sync(~0u, l[h], 2);
      if ((lane & 3) == 0) {
        ml[(warp * 2 + 0) * kRows + g + 8 * h] = m[h];
        ml[(warp * 2 + 1) * kRows + g + 8 * h] = l[h];
      }
    }
    bar_consumers(C::kWarps * 32);
    float f[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < C::kWarps; ++w) top = fmaxf(top, ml[(w * 2) * kRows + g + 8 * h]);
      f[h] = ex2(m[h] - (top == -INFINITY ? 0.f : top));
    }
    // A warp without a key in a row adds nothing (f = 0, its o is 0).  The warps
    // add one after the other into one buffer, the first half of the columns in
    // the order 3, 2, 1, 0 and the second in 2, 3, 0, 1, two warps at a time.
#pragma unroll
    for (int round = 0; round < 4; ++round) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        if (warp != (half == 0 ? 3 - round : (round + 2) & 3)) continue;
#pragma unroll
        for (int n = half * (HDP / 16); n < (half + 1) * (HDP / 16); ++n)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float2* at = (float2*)(bufs + (g + 8 * h) * C::kPad + n * 8 + c2);
            float2 v = make_float2(o[n][2 * h] * f[h], o[n][2 * h + 1] * f[h]);
            if (round > 0) {
              const float2 w = *at;
              v.x += w.x;
              v.y += w.y;
            }
            *at = v;
          }
      }
      bar_consumers(C::kWarps * 32);
    }
    const bool whole = starts && ends;
    const int slot = blockIdx.x * 2 + (starts ? 1 : 0);
    const bool outside = KV_BAD(g_few_counts, x.rows >= 1 && x.rows <= kRows && few_inside(p, x, x.row0) && few_inside(p, x, x.row0 + x.rows - 1) &&
                                                  slot < 2 * (int)gridDim.x);
    float* part = p.part + (int64_t)slot * (kRows * HDP + 2 * kRows);
    for (int e = tid; e < kRows * (HDP / 8); e += C::kWarps * 32) {
      const int row = e / (HDP / 8), col = e % (HDP / 8) * 8;
      if (row >= x.rows || outside) continue;
      float top = -INFINITY, sum = 0.f, v[8];
#pragma unroll
      for (int w = 0; w < C::kWarps; ++w) top = fmaxf(top, ml[(w * 2) * kRows + row]);
      const float safe = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int w = 0; w < C::kWarps; ++w) sum += ml[(w * 2 + 1) * kRows + row] * ex2(ml[(w * 2) * kRows + row] - safe);
#pragma unroll
      for (int q = 0; q < 8; q += 4) *(float4*)(v + q) = *(const float4*)(bufs + row * C::kPad + col + q);
      if (whole) {
        const int abs = x.row0 + row;
        const int64_t tok = r.q0 + abs / p.group, head = (int64_t)x.head * p.group + abs % p.group;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        if (col < p.dim) {
          uint4 w;
          w.x = pack2<F16>(v[0] * inv, v[1] * inv);
          w.y = pack2<F16>(v[2] * inv, v[3] * inv);
          w.z = pack2<F16>(v[4] * inv, v[5] * inv);
          w.w = pack2<F16>(v[6] * inv, v[7] * inv);
          *(uint4*)(p.out + 2 * (tok * p.out_tok + head * p.out_head + col)) = w;
        }
        if (p.lse && col == 0) p.lse[tok * p.heads + head] = L<F16>::lse(top, sum);
      } else {
        float4* to = (float4*)(part + row * HDP + col);
        to[0] = make_float4(v[0], v[1], v[2], v[3]);
        to[1] = make_float4(v[4], v[5], v[6], v[7]);
        if (col == 0) {
          part[kRows * HDP + row] = top;
          part[kRows * HDP + kRows + row] = sum;
        }
      }
    }
    if (starts && !ends && tid == 0) {
      const int64_t first = range.end - seg;  // the item's first unit
      p.desc[blockIdx.x] = make_int4(r.q0, x.row0, x.head | x.rows << 16, attn_block_of(range, first + cost - 1) - (int)blockIdx.x + 1);
    }
    bar_consumers(C::kWarps * 32);

    left -= seg;
    t0 = 0;
    if (++item == (int64_t)p.kv_heads * rt) {
      item = 0;
      do {
        if (++req >= p.batch) break;
        r = attn_req(p, req);
        rt = row_tiles(p, r);
        cost = key_tiles(r);
      } while (rt == 0);
      if (req >= p.batch) break;
    }
  }
}

// Joins the parts of the item that block c began and did not end: one block per
// (c, row), its four warps a quarter of the parts each.
template <int HDP, bool F16>
__global__ void __launch_bounds__(128) k_attend_few_join(const __grid_constant__ AttnParams p) {
  constexpr int kCols = HDP / 32, kSlot = kRows * HDP + 2 * kRows;
  __shared__ float acc[4][HDP], sums[4];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  wait_for_primary();
  const int4 d = p.desc[blockIdx.x];
  const int rows = d.z >> 16, head0 = d.z & 0xFFFF;
  const int parts = KV_BAD(g_few_counts, d.w >= 0 && d.w <= (int)(gridDim.x - blockIdx.x) && rows <= kRows && head0 < p.kv_heads &&
                                             d.x + (d.y + rows - (d.w > 0)) / p.group < p.tokens)
                        ? 0
                        : d.w;
  // part k: block c's last segment, then the first segments of the following blocks
  const float* const base = p.part + (int64_t)blockIdx.x * 2 * kSlot;
  auto slot = [&](int k) { return base + (int64_t)(k == 0 ? 1 : 2 * k) * kSlot; };
  for (int row = blockIdx.y; parts != 0 && row < rows; row += gridDim.y) {
    float top = -INFINITY;
    for (int k = lane; k < parts; k += 32) top = fmaxf(top, slot(k)[kRows * HDP + row]);
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
    const float safe = top == -INFINITY ? 0.f : top;
    float v[kCols], s = 0.f;
#pragma unroll
    for (int c = 0; c < kCols; ++c) v[c] = 0.f;
#pragma unroll 4
    for (int k = warp; k < parts; k += 4) {
      const float* at = slot(k);
      const float f = ex2(at[kRows * HDP + row] - safe);
      s = fmaf(f, at[kRows * HDP + kRows + row], s);
#pragma unroll
      for (int c = 0; c < kCols; c += 2) {
        const float2 x = *(const float2*)(at + row * HDP + c * 32 + lane * 2);
        v[c] = fmaf(f, x.x, v[c]);
        v[c + 1] = fmaf(f, x.y, v[c + 1]);
      }
    }
#pragma unroll
    for (int c = 0; c < kCols; c += 2) *(float2*)&acc[warp][c * 32 + lane * 2] = make_float2(v[c], v[c + 1]);
    if (lane == 0) sums[warp] = s;
    __syncthreads();
    s = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    const int abs = d.y + row;
    const int64_t tok = d.x + abs / p.group, head = (int64_t)head0 * p.group + abs % p.group;
    for (int col = threadIdx.x * 2; col < p.dim; col += 256) {
      const float inv = s == 0.f ? 0.f : 1.f / s;
      const float a = (acc[0][col] + acc[1][col]) + (acc[2][col] + acc[3][col]);
      const float b = (acc[0][col + 1] + acc[1][col + 1]) + (acc[2][col + 1] + acc[3][col + 1]);
      *(uint32_t*)(p.out + 2 * (tok * p.out_tok + head * p.out_head + col)) = pack2<F16>(a * inv, b * inv);
    }
    if (p.lse && threadIdx.x == 0) p.lse[tok * p.heads + head] = L<F16>::lse(top, s);
    __syncthreads();
  }
}

template <int HDP, bool F16>
cudaError_t launch(const AttnParams& p, int rows_hint, int sms, int device, cudaStream_t stream) {
  using C = FewCfg<HDP>;
  static std::atomic<uint64_t> allowed;
  cudaError_t e = kv_allow_smem(k_attend_few<HDP, F16>, C::kSmem, device, allowed);
  if (e != cudaSuccess) return e;
  const int blocks = sms * C::kPerSm;
  k_attend_few<HDP, F16><<<blocks, C::kThreads, C::kSmem, stream>>>(p);
  if ((e = cudaGetLastError()) != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(blocks, rows_hint < 1 || rows_hint > kRows ? kRows : rows_hint);
  cfg.blockDim = dim3(128);
  cfg.stream = stream;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_attend_few_join<HDP, F16>, p);
}

}  // namespace

size_t attend_few_workspace(int sms) {
  // slots of 64 columns for three blocks an SM, 128 for two, 256 for one: 256 hold any
  return (size_t)sms * kFewPerSm * sizeof(int4) + 256 + (size_t)sms * 2 * (kRows * 256 + 2 * kRows * kFewPerSm) * sizeof(float);
}

cudaError_t launch_attend_few(const AttnParams& p, bool f16, int rows_hint, int sms, int device, cudaStream_t stream) {
  if (p.dim <= 64) return f16 ? launch<64, true>(p, rows_hint, sms, device, stream) : launch<64, false>(p, rows_hint, sms, device, stream);
  if (p.dim <= 128)
    return f16 ? launch<128, true>(p, rows_hint, sms, device, stream) : launch<128, false>(p, rows_hint, sms, device, stream);
  return f16 ? launch<256, true>(p, rows_hint, sms, device, stream) : launch<256, false>(p, rows_hint, sms, device, stream);
}

cudaError_t attend_few_counts(cudaStream_t stream, uint32_t* counts) {
  void* at = nullptr;
  const cudaError_t e = cudaGetSymbolAddress(&at, g_few_counts);
  return e != cudaSuccess ? e : cudaMemcpyAsync(counts, at, sizeof(g_few_counts), cudaMemcpyDeviceToHost, stream);
}

}  // namespace mpt
