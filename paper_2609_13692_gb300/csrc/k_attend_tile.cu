// Attention over a paged cache for many query rows per KV head (include/mpt_kv.h,
// mpt_kv_attend): chunks of new tokens, on tcgen05 with accumulators in tensor
// memory.
//
// The running form over key tiles is that of k_attend_few.cu.  An item is a KV
// head and two tiles of up to 128 query rows (row = token t, query head g of
// the group; one tile with heads above 128 elements), so both products of a key
// tile, S = Q K^T and O += P V, are 128 x 128 x 128 and every key tile read
// serves 256 rows.
//
// Bound: 4 d operations per visible pair, on the tensor cores; per key tile two
// S and two PV products (512 cycles each), beside which 2 x 128 x 128
// exponentials have to fit.  So the two row tiles alternate: while one's
// products run, the other's probabilities are computed.
//
// Measured (one GB300, 32 query heads on 8 KV heads of 128, pages of 16): 4,096
// tokens over 20,480 keys, call after call at the power limit, 0.83 ms, 1.49
// PFLOP/s, 0.87 of the sustained matrix rate; a few calls at full clocks 0.77 ms,
// 1.61 PFLOP/s, 0.86 of the burst rate.  28 requests of 28 to 685 tokens over 700
// to 6,000 keys, 24 heads of 96, a tenth of the pages absent: 0.37 ms.  2,048
// tokens over 10,000 keys: heads of 64, 128 and 256 180, 220 and 600 us (floors
// 81, 162 and 323).  On a smaller case at full clocks the tensor pipe is busy 63 %
// of the time: a row tile's chain of scores, probabilities (about
// 1,300 cycles, half of it exponentials), outputs and the hand-over between
// warps takes 2,600 to 3,200 cycles, and only two such chains fit in tensor
// memory.  Per key tile warp 8 spends 2,400 cycles on the pipe's 2,048 and 780
// waiting for P.  An item costs 8 us besides (7 a block in the 0.37 ms): its last
// outputs, queries and first scores follow one another.
//
// Tried and slower: P handed over in halves (the products wait for the second
// half), P against the last maximum while the new one is found (1.20 ms), one
// code path for an item's first scores (0.87 ms); two threads a row, sixteen
// warps of rows that exchange maxima (0.94 ms); an item's first keys copied
// before its queries (0.38 -> 0.40 ms), the second row tile's first scores
// issued once the first's P stands (0.89 and 0.40 ms), what the roles compute of
// an item kept in its list entry (few tokens 1 to 4 % faster, but the long chunk
// 2 % and heads of 64 9 % slower).
//
//   warps 0-3, 4-7  one row tile each, one thread per row (no exchange between
//                   threads): S from tensor memory, running maximum, P back
//                   over S, O rescaled where the maximum grew, O out at the end
//   warp 8          issues the products
//   warps 9, 10     copies: queries once an item and keys, and values, of each
//                   tile page by page into a ring of slots (with pages of 16 one
//                   warp's 32 copies a tile take longer than its products)
//   warp 11         waits for the copies on the products' behalf, and looks at
//                   the values of tiles with masked keys (below)
//
// Rescaling O costs a pass over its 128 columns, so it waits until the maximum
// has grown by 2^8 (f16: 2^4, below): any reference below the maximum gives the
// same quotient, and with 2^8 of room neither P nor its sum can overflow.
//
// A masked key's probability is 0, but 0 times an infinite or NaN value is NaN.
// Tiles with masked keys are few (the last of an item); warp 11 looks at the
// values that some row of the item must not see, blanks those that are not
// finite, and notes the ones that other rows do see; these rows add them at the
// item's end, key by key.
#include "kv4.cuh"

namespace mpt {
namespace {

__device__ uint32_t g_tile_counts[kKvCounts];

constexpr int kKeys = 128;     // keys of a tile
template <bool kCodes>
constexpr int kThreads = kCodes ? 512 : 384;
constexpr int kOddSets = 4;    // items whose notes are kept apart
constexpr int kList = 32;      // items listed at a time
constexpr int kHeldSets = 16;  // key tiles whose page marks are kept apart

template <int HDP>
struct TileCfg {
  static constexpr int kBlk = HDP / 64;
  // Row tiles of an item: O takes HDP columns each, S 128, of 512.  With one, S
  // has two buffers, and the scores of the next key tile are made while P of this
  // one is (2,048 tokens over 10,000 keys, 32 heads of 256: 719 -> 600 us).  For
  // single row tiles of smaller heads the same was slower (28 rows over 20,001
  // keys 43 -> 50 us): the ring then holds less ahead.
  static constexpr int kTiles = HDP == 256 ? 1 : 2;
  static constexpr int kRows = 128 * kTiles;         // rows of a slot of partial results
  static constexpr int kSlot = kKeys * HDP * 2;
  static constexpr int kQ = kRows * HDP * 2;
  static constexpr int kSlots = HDP == 64 ? 8 : HDP == 128 ? 5 : 2;
  // Who waits for keys.  Warp 11 may, as it may skip an item's first ones, where
  // the slot's next use is far enough off to imply that they have landed; with
  // two slots the next key tile is the slot's next phase, and a wait for it
  // before the one at hand has landed would pass at once.
  static constexpr bool kWatchKeys = kSlots > 2;
  // Registers a thread: of the four warps without rows, and of the rows' eight.
  // (Of 88 with 208 and 72 with 216: 2,048 tokens over 10,000 keys, heads of 64,
  // 200 and 180 us; 28 ragged chunks, heads of 96, 372 and 383.)
  // (The cache in 4 bits has eight warps without rows.)
  template <bool kCodes>
  static constexpr int kRoleRegs = kCodes || HDP == 64 ? 72 : 88;
  template <bool kCodes>
  static constexpr int kRowRegs = kCodes ? 184 : HDP == 64 ? 216 : 208;
  // Warps that widen codes: 9 to 15, and those of the absent row tile.
  static constexpr int kCodeWarps = kTiles == 1 ? 11 : 7;
  static_assert(kRoleRegs<false> + 2 * kRowRegs<false> <= 3 * 168 && 2 * kRoleRegs<true> + 2 * kRowRegs<true> <= 4 * 128);
  static constexpr int kSmem = 1024 + kQ + kSlots * kSlot + 2048;
};

// One entry of a block's list of items: the item, and the part of its key tiles
// that is the block's.
struct alignas(16) TileEntry {
  int req, head, pair, q0, ql, kvl, t0, seg;
};

struct TileShared {
  unsigned long long full[8], empty[8], q_full, q_empty, s_full[3], p_ready[3], o_full[2], o_step, drain;
  unsigned long long odd_read[kOddSets];  // the rows of both tiles have done with a set of notes
  uint32_t tmem;
  uint32_t sent[2], asked;  // copies issued, for the block's end: tiles of keys and of values, items' queries
  int gave_up;
  unsigned long long q_ready[2];  // cache in 4 bits: queries of a row tile
  uint32_t held[kHeldSets];
  uint32_t odd[kOddSets][9];  // 8 words of keys from the item's first ambiguous one, and whether any is set
  int64_t scratch[40];
  int64_t left;  // key tiles that the list has yet to take
  int items, stride, item, column, t0;  // all items; of the line: its step, and where the list goes on
  int count, more;
  alignas(16) TileEntry list[kList];
};
static_assert(sizeof(TileShared) <= 2048);

// Bounded wait of a whole warp: false once the block has given up, or after four
// seconds.  The block's end counts it (with an atomic at each of the waits the
// long chunk took 20 to 40 us more).  The clock is looked at after the first
// polls only: reading it takes longer than most waits.
__device__ __forceinline__ bool wait_on(unsigned long long* bar, uint32_t parity, int* gave_up) {
  unsigned long long start = 0;
  for (;;) {
    for (int i = 0; i < 256; ++i)
      if (__all_sync(~0u, mbar_try_wait(bar, parity))) return true;
    const unsigned long long now = now_ns();
    if (start == 0) start = now;
    bool over = *(volatile int*)gave_up != 0;
    if (now - start > 4000000000ull) {
      over = true;
      *(volatile int*)gave_up = 1;
    }
    if (__any_sync(~0u, over)) return false;
  }
}
__device__ __forceinline__ bool wait_all(unsigned long long* bar, uint32_t parity, int* gave_up) {
  return __all_sync(~0u, mbar_try_wait(bar, parity)) || wait_on(bar, parity, gave_up);
}

// Several arrivals at once.
__device__ __forceinline__ void mbar_arrive_n(unsigned long long* bar, uint32_t n) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(n) : "memory");
}
template <bool kCodes>
__device__ __forceinline__ void bar_all() {
  asm volatile("bar.sync 1, %0;" ::"n"(kThreads<kCodes>) : "memory");
}

// The same for the warps that have time: polls take issue slots that the rows'
// arithmetic needs.  (4,096 tokens over 20,480 keys: 797 us with warp 11's polls
// back to back, 770 with 20 to 400 ns between them; 20 ns between the copying
// warps' polls for free slots: 772 -> 765 us, 28 ragged chunks 380 -> 372.  The
// others' waits are on the chain, and any longer sleep costs.)
template <int kNs>
__device__ __forceinline__ bool wait_spaced(unsigned long long* bar, uint32_t parity, int* gave_up) {
  unsigned long long start = 0;
  for (int n = 1;; ++n) {
    if (__all_sync(~0u, mbar_try_wait(bar, parity))) return true;
    __nanosleep(kNs);
    if (n % 256 != 0) continue;
    const unsigned long long now = now_ns();
    if (start == 0) start = now;
    bool over = *(volatile int*)gave_up != 0;
    if (now - start > 4000000000ull) {
      over = true;
      *(volatile int*)gave_up = 1;
    }
    if (__any_sync(~0u, over)) return false;
  }
}

// The first lane's value in every lane, which the compiler then knows to be uniform.
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __shfl_sync(~0u, v, 0); }

__device__ __forceinline__ bool elect_one() {
  uint32_t one;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(one));
  return one != 0;
}

// Shared-memory operands of tcgen05.mma, 128-byte swizzle: the low word holds the
// address and, for an operand whose contiguous axis is not the summed one (V),
// the distance of its blocks of 64 along that axis; the high word the distance
// of groups of 8 rows (1,024 bytes) and the form.
constexpr uint32_t kOperandHigh = 1024 >> 4 | 1u << 14 | 2u << 29;
__device__ __forceinline__ uint32_t operand_low(uint32_t addr, uint32_t blocks) { return addr >> 4 | blocks >> 4 << 16; }

__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t desc, uint32_t add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 x, y;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "mov.b64 x, {%1, %5};\n\tmov.b64 y, {%2, %5};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n\t}" ::"r"(d), "r"(a), "r"(b), "r"(desc), "r"(add), "r"(kOperandHigh)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t desc, uint32_t add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 y;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "mov.b64 y, {%2, %5};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n\t}" ::"r"(d), "r"(a), "r"(b), "r"(desc), "r"(add), "r"(kOperandHigh)
      : "memory");
}
__device__ __forceinline__ void commit(unsigned long long* bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void tmem_ld32(float* r, uint32_t addr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]),
        "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]), "=f"(r[16]),
        "=f"(r[17]), "=f"(r[18]), "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]), "=f"(r[24]),
        "=f"(r[25]), "=f"(r[26]), "=f"(r[27]), "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_ld16(float* r, uint32_t addr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]),
        "=f"(r[9]), "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}

__device__ __forceinline__ void tma_load_3d(void* dst, const CUtensorMap* map, int x, int y, int z, unsigned long long* bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
          smem_u32(dst)),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(smem_u32(bar))
      : "memory");
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// Pairs of 32-bit values in one instruction.
__device__ __forceinline__ uint64_t pair(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpair(uint64_t x, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
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

// Scores may exceed a row's reference by 2^kLag before its outputs are rescaled
// (f16: the less, the further down probabilities are rounded; 28 ragged chunks
// take 381, 385 and 400 us with 8, 4 and 2).
template <bool F16>
constexpr int kLag = F16 ? 4 : 8;
template <bool F16>
using L = Lift<F16, kLag<F16>>;

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
__device__ __forceinline__ float2 unpack2(uint32_t x) {
  if (F16) {
    float2 f;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, h;\n\t}" : "=f"(f.x), "=f"(f.y) : "r"(x));
    return f;
  }
  return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xFFFF0000u));
}
// Nonzero if one of the eight elements is an infinity or a NaN: an exponent of
// ones carries into the sign's place when one is added to it.
template <bool F16>
__device__ __forceinline__ uint32_t not_finite8(const uint4& x) {
  constexpr uint32_t e = F16 ? 0x7C007C00u : 0x7F807F80u, one = F16 ? 0x04000400u : 0x00800080u;
  return (((x.x & e) + one) | ((x.y & e) + one) | ((x.z & e) + one) | ((x.w & e) + one)) & 0x80008000u;
}

__device__ __forceinline__ void store32(void* to, const uint32_t* v) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(to), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]),
               "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}

// Items in their natural order: the requests, the KV heads of each, the pairs of
// row tiles of each (single row tiles with heads above 128).  Where the call's keys and values fit in L2 the blocks share
// the line as it is.  Where they do not, every block would at any time be at
// heads of its own, each read from memory for every pair: then the line takes
// the items in columns, c, c + n, c + 2 n, .. of an n-block grid for c = 0, 1, ..,
// and the blocks work on neighbouring items, mostly pairs of the same head.
// (Natural order and columns: 28 requests of up to 700 tokens over 6,000 keys of
// 24 heads, 380 MB: 541 and 488 us; 4,096 tokens over 20,480 keys of 8 heads,
// 84 MB: 785 and 840 us, the blocks reading the same keys at the same time.)
// The cache in 4 bits is always taken in columns: besides, they mix items of two
// row tiles with those of one among the blocks (28 requests of up to 700 tokens
// over 700 to 6,000 keys, 24 heads on 8 of 96: 678 and 507 us; of 128: 719 and
// 520; 4,096 tokens over 20,480 keys: 968 and 969).
constexpr int64_t kNaturalBytes = 100ll << 20;  // of 126 MB of L2
__device__ __forceinline__ int pairs_of(const AttnParams& p, int ql) {
  return (int)(((int64_t)ql + p.item_toks - 1) / p.item_toks);
}
// Key tiles that the pair has to take, one at least (a row without keys is written too).
__device__ __forceinline__ int pair_cost(const AttnParams& p, int ql, int kvl, int pair) {
  int lim = kvl;
  if (p.causal) {
    const int64_t tok = (int64_t)p.item_toks * (pair + 1);
    lim = kvl - ql + (tok < ql ? (int)tok : ql);  // > -2^31 + 1
  }
  return lim <= kKeys ? 1 : (lim - 1) / kKeys + 1;
}

// The cache in 4 bits: what an item costs beside its key tiles, in their time,
// counted before them as units of the line without work.  (28 ragged chunks: 482 us
// without, 460, 450, 451 and 451 with 2, 4, 6 and 8.)
template <bool kCodes>
constexpr int kItem = kCodes ? 4 : 0;

// What a role needs of an entry.
struct TileItem {
  TileEntry e;
  int tok0, n0, n1, tiles;  // first token; key tiles of each row tile from t0; their maximum
  int lim_first;            // what the item's first row sees
  __device__ __forceinline__ void load(const AttnParams& p, const TileEntry* at) {
    const int4 a = ((const int4*)at)[0], b = ((const int4*)at)[1];
    e = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    tok0 = e.pair * p.item_toks;
    lim_first = limit(p, tok0);
    n0 = key_count(p, tok0);
    n1 = p.item_toks > p.toks ? key_count(p, (int64_t)tok0 + p.toks) : 0;
    tiles = n0 > n1 ? n0 : n1;
  }
  __device__ __forceinline__ int limit(const AttnParams& p, int t) const { return attn_limit(p, {e.q0, e.ql, e.kvl}, t); }
  // Key tiles from t0 on that some row of the tile beginning at token `first` sees.
  __device__ __forceinline__ int key_count(const AttnParams& p, int64_t first) const {
    if (first >= e.ql) return 0;
    const int end = (int)(first + p.toks < e.ql ? first + p.toks : e.ql);
    const int lim = limit(p, end - 1), need = lim == 0 ? 0 : (lim - 1) / kKeys + 1;
    const int stop = e.t0 + e.seg < need ? e.t0 + e.seg : need;
    return stop > e.t0 ? stop - e.t0 : 0;
  }
  __device__ __forceinline__ int count(int s) const { return s ? n1 : n0; }
  // Whether some row of the item does not see every key of tile t0 + j.
  __device__ __forceinline__ bool partly(int j) const { return (int64_t)(e.t0 + j + 1) * kKeys > lim_first; }
};

// By one warp: the next entries of the block's list, from `item` on (its first
// t0 units are another block's), `left` units in all.  Lane k finds the
// k-th item; the requests are gone through 32 at a time.
template <bool kCodes>
__device__ void fill_list(const AttnParams& p, TileShared& sh) {
  const int lane = threadIdx.x & 31, n = sh.stride;
  const int items = sh.items;
  int item = sh.item, column = sh.column;
  for (int j = lane; item < items;) {  // j items on, through the ends of columns
    const int rest = (items - item - 1) / n + 1;
    if (j < rest) {
      item += j * n;
      break;
    }
    j -= rest;
    item = ++column < n ? column : items;
  }
  TileEntry e{};
  int cost = 0;
  int start = 0;
  bool found = false;
  for (int base = 0; base < p.batch && __any_sync(~0u, !found && item < items); base += 32) {
    AttnReq r{0, 0, 0};
    if (base + lane < p.batch) r = attn_req(p, base + lane);
    const int pairs = pairs_of(p, r.ql);
    int inc = pairs * p.kv_heads;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int v = __shfl_up_sync(~0u, inc, d);
      if (lane >= d) inc += v;
    }
    const int end = start + inc, total = __shfl_sync(~0u, end, 31);
    const bool here = !found && item < items && item < total;
    // the request: how many of these 32 end at or before the item
    int at = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) at += __shfl_sync(~0u, end, i) <= item;
    const int from = at < 32 ? at : 31;
    const int before = __shfl_sync(~0u, end - pairs * p.kv_heads, from);
    const int q0 = __shfl_sync(~0u, r.q0, from), ql = __shfl_sync(~0u, r.ql, from), kvl = __shfl_sync(~0u, r.kvl, from);
    const int np = __shfl_sync(~0u, pairs, from);
    if (here) {
      const int local = item - before;
      e.req = base + from;
      e.head = local / np;
      e.pair = local % np;
      e.q0 = q0, e.ql = ql, e.kvl = kvl;
      cost = pair_cost(p, ql, kvl, e.pair) + kItem<kCodes>;
      found = true;
    }
    start = total;
  }
  if (lane == 0) e.t0 = sh.t0;
  const int mine = found ? cost - e.t0 : 0;
  int64_t inc = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t v = __shfl_up_sync(~0u, inc, d);
    if (lane >= d) inc += v;
  }
  const int64_t left = sh.left, open = left - (inc - mine);
  e.seg = (int)(open < 0 ? 0 : open < mine ? open : mine);
  if (kBoundsChecked) {  // the list ends before an entry that is out of range
    const bool bad = KV_BAD(g_tile_counts, e.seg == 0 || (attn_inside(p, e.req, e.head, e.q0, e.ql, e.kvl) && e.pair >= 0 &&
                                                          (int64_t)e.pair * p.item_toks < e.ql && e.t0 >= 0 && e.t0 + e.seg <= cost));
    if (__ballot_sync(~0u, bad) & ((2u << lane) - 1u)) e.seg = 0;
  }
  const int n_used = __popc(__ballot_sync(~0u, e.seg > 0));  // a run from lane 0
  const int64_t taken = inc - mine + e.seg;
  int count = n_used;
  if (kCodes) {  // from units to key tiles; the last item may have none of them here
    const int end = e.t0 + e.seg - kItem<kCodes>;
    e.t0 = e.t0 > kItem<kCodes> ? e.t0 - kItem<kCodes> : 0;
    e.seg = e.seg > 0 && end > e.t0 ? end - e.t0 : 0;
    count = __popc(__ballot_sync(~0u, e.seg > 0));
  }
  __syncwarp();
  if (e.seg > 0) sh.list[lane] = e;
  const int last = n_used > 0 ? n_used - 1 : 0;
  if (lane == last) {
    sh.count = count;
    sh.left = left - taken;
    sh.more = n_used == kList && left > taken;
    if ((kBoundsChecked || kCodes) && count == 0) {  // a list has an entry: one without rows
      sh.list[0] = {0, 0, 0, 0, 0, 0, 1, 0};
      sh.count = 1;
    }
    // after a full list whose last item is whole: the one that follows it in its column
    sh.t0 = 0;
    sh.item = item + n < items ? item + n : column + 1;
    sh.column = item + n < items ? column : column + 1;
  }
  __syncwarp();
}

// ---- the cache in 4 bits ----
//
// Its kernel is the same but for where the operands come from: warps 9 to 15
// read codes and write f16 keys and values where the copies would have put
// them, and each row's thread its own query.  Codes stand for finite values
// whatever their bytes, so there is nothing to look for in masked ones.
//
// Measured (one GB300, 32 query heads on 8 KV heads of 128, pages of 16): 4,096
// tokens over 20,480 keys, call after call, 0.94 ms, 1.31 PFLOP/s, of which 0.10
// are the widening's (0.85 with codes left as they are, 0.83 over 16 bits); 28
// requests of 28 to 685 tokens over 700 to 6,000 keys, 24 heads of 96, a tenth of
// the pages absent, 0.45 ms.  Widening costs a warp about 85 operations for a
// tile of 8 tokens, in a chain that one warp in a scheduler cannot hide: with three
// warps instead of seven the long chunk takes 1.40 ms (divisions for the places in
// a slot inside the loop: 3.0).
//
// Tried and no faster: 192 registers a row and 64 for the others (2 % slower),
// longer sleeps between polls, the fence between codes' stores and the
// products on the products' side (2 % less), page lookups a tile further ahead (2 %
// more); with heads above 128 five slots of half a key tile (1.25 -> 1.70 ms).
template <bool F16, bool kCodes>
__device__ __forceinline__ uint32_t pack_as(const AttnParams& p, float lo, float hi) {
  if (!kCodes) return pack2<F16>(lo, hi);
  return p.f16 ? pack2<true>(lo, hi) : pack2<false>(lo, hi);
}

// A row's query into row r of its tile's operand, each 8 elements in the order
// 0 4 1 5 2 6 3 7 that a word of codes gives (widen_codes).  bf16: divided by the
// power of two 2^e that leaves the largest element in [1, 2), so that f16 holds what
// is at least 2^-17 exactly and the rest to 2^-25; returns 2^e.  nullptr: zeros.
template <int HDP>
__device__ __forceinline__ float stage_query(const char* q, int dim, bool f16, char* to, int r) {
  uint4 u[HDP / 8];  // all loads are in flight together
#pragma unroll
  for (int c = 0; c < HDP / 8; ++c) {
    u[c] = make_uint4(0, 0, 0, 0);
    if (q && c * 8 < dim) u[c] = __ldg((const uint4*)(q + 16 * c));
  }
  float by = 1.f, back = 1.f;
  if (!f16) {
    uint32_t top = 0;
#pragma unroll
    for (int c = 0; c < HDP / 8; ++c) {
      const uint32_t v[4] = {u[c].x, u[c].y, u[c].z, u[c].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) top = max(top, max(v[i] << 16 & 0x7FFFFFFFu, v[i] & 0x7FFF0000u));
    }
    int e = (int)(top >> 23) - 127;
    e = top == 0 ? 0 : e < -126 ? -126 : e > 126 ? 126 : e;
    by = __uint_as_float((uint32_t)(127 - e) << 23);
    back = __uint_as_float((uint32_t)(127 + e) << 23);
  }
#pragma unroll
  for (int c = 0; c < HDP / 8; ++c) {
    uint32_t v[4] = {u[c].x, u[c].y, u[c].z, u[c].w};
    if (!f16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = pack2<true>(__uint_as_float(v[i] << 16) * by, __uint_as_float(v[i] & 0xFFFF0000u) * by);
    }
    uint4 o;
    o.x = __byte_perm(v[0], v[2], 0x5410);
    o.y = __byte_perm(v[0], v[2], 0x7632);
    o.z = __byte_perm(v[1], v[3], 0x5410);
    o.w = __byte_perm(v[1], v[3], 0x7632);
    *(uint4*)(to + (c >> 3) * 128 * 128 + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = o;
  }
  return back;
}

// 16 bytes of codes (32 elements of a key, or 16 of a pair of values) with their marks.
struct CodeChunk {
  uint4 w;
  uint32_t marks;
};

// By kCodeWarps warps: f16 keys and values of the block's key tiles, each in its
// slot of the ring.  A tile of 8 tokens has 8 n chunks of 16 bytes of either;
// a warp takes tiles of 8 in turn (half of one with more than 4 groups, two at
// once with 2), a lane the same chunk of each.  A chunk is read as soon as the one
// before it in its registers has been used, which is half a key tile ahead.
// (2,048 tokens over 10,000 keys of 32 heads of 256 on 8: the four warps of the
// absent row tile among them, 1.50 -> 1.25 ms.)
template <int HDP, typename Next, typename Leave>
__device__ __forceinline__ void widen_codes(const AttnParams& p, TileShared& sh, char* ring, int me, Next next_item, Leave leave) {
  using C = TileCfg<HDP>;
  constexpr int kCodeWarps = C::kCodeWarps;
  constexpr int kTogether = HDP == 64 ? 2 : 1, kPer = HDP == 256 ? 2 : 1;
  constexpr int kUnits = kKeys / kCodeTokens / kTogether * kPer;       // steps of all warps in half a key tile
  constexpr int kSteps = (kUnits + kCodeWarps - 1) / kCodeWarps;       // of a warp
  const int lane = threadIdx.x & 31;
  const int n = kv4_groups(p.dim);
  int* const gave_up = &sh.gave_up;
  const int second = kTogether == 2 ? lane >> 4 : 0, in = kTogether == 2 ? lane & 15 : lane;

  // Where the lane's chunks of a tile of 8 come from and go to.  A slot has rows
  // of 128 bytes (64 elements) with their 16-byte pieces permuted by row: piece c of
  // row r at c ^ (r & 7).  Lanes of odd blocks of 64 elements take a chunk's halves
  // in the other order, so that 8 lanes write to 8 places.
  bool has[kPer], odd[kPer][2];
  uint32_t mark_from[kPer][2], to[kPer][2];  // (the second index is known where they are used, the first chosen)
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int x = in + 32 * i;
    has[i] = x < 8 * n;
    const int tok = x / n, g = x - tok * n;  // of a key
    mark_from[i][0] = kv4_key_marks(n, 0) + 2 * x;  // [token][group], as the chunks
    odd[i][0] = g >> 1 & 1;
    to[i][0] = (g >> 1) * kKeys * 128 + tok * 128 + ((((g & 1) << 2 | (g & 2)) ^ tok) << 4);
    const int pair = x / (2 * n), piece4 = x - pair * 2 * n;  // of a pair of values, 4 pieces of 4 elements
    mark_from[i][1] = kv4_value_marks(n, pair) + 4 * (piece4 >> 1);
    odd[i][1] = piece4 >> 2 & 1;
    to[i][1] = (piece4 >> 2) * kKeys * 128 + 2 * pair * 128 + ((((piece4 & 3) << 1 | (piece4 >> 2 & 1)) ^ 2 * pair) << 4);
  }
  const uint32_t from = 16 * in, values_from = kv4_value(n, 0);

  // Step i, half v (0 keys, 1 values): the tile of 8 that it is about, and which of the lane's chunks.
  // (The warps that have one step more than the others are others for values.)
  auto unit = [&](int v, int i) { return i * kCodeWarps + (v ? (me + 2) % kCodeWarps : me); };
  auto tile8 = [&](int u) { return u / kPer * kTogether + second; };

  // Lane b: the b-th tile of 8 of a key tile, nullptr without a page.
  auto tile_of = [&](const TileItem& w, int j, int tiles) -> const char* {
    const int64_t key = (int64_t)(w.e.t0 + j) * kKeys + (lane & 15) * kCodeTokens;
    if (j >= tiles || key >= w.e.kvl) return nullptr;
    const int id = p.table[(int64_t)w.e.req * p.table_stride + (key >> p.page_log2)];
    if (id < 0 || id >= p.n_pages) return nullptr;
    const int slot = (int)(key & ((1 << p.page_log2) - 1));
    if (KV_BAD(g_tile_counts, id < p.n_pages && slot + kCodeTokens <= 1 << p.page_log2 && w.e.head < p.kv_heads)) return nullptr;
    return p.k + (int64_t)id * p.k_page + (int64_t)w.e.head * p.k_head + (int64_t)(slot / kCodeTokens) * kv4_tile(n);
  };
  auto load = [&](CodeChunk& c, int v, int i, const char* tiles) {
    const int x = unit(v, i), t8 = tile8(x), which = x % kPer;
    const char* at = (const char*)__shfl_sync(~0u, (unsigned long long)tiles, t8 & 15);
    c.w = make_uint4(0, 0, 0, 0);
    c.marks = 0;
    if (t8 >= kKeys / kCodeTokens || !has[which] || !at) return;  // without a page: zeros
    c.w = __ldg((const uint4*)(at + (v ? values_from : 0) + from + 512 * which));
    const char* m = at + mark_from[which][v];
    c.marks = v ? __ldg((const uint32_t*)m) : (uint32_t)__ldg((const uint16_t*)m);
  };
  auto store = [&](const CodeChunk& c, int v, int i, uint32_t slot_at) {
    const int x = unit(v, i), t8 = tile8(x), which = x % kPer;
    if (t8 >= kKeys / kCodeTokens || !has[which]) return;
    const uint32_t at = slot_at + to[which][v] + t8 * kCodeTokens * 128;
    const bool swap = odd[which][v];
    const uint32_t u[4] = {swap ? c.w.z : c.w.x, swap ? c.w.w : c.w.y, swap ? c.w.x : c.w.z, swap ? c.w.y : c.w.w};
    uint32_t step, off;
    if (v == 0) {
      kv4_key_step(c.marks, step, off);
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        uint32_t o[4];
        kv4_word(u[h], step, off, o);
        asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at ^ 16 * h), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]) : "memory");
      }
    } else {
      kv4_value_step(c.marks, step, off);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t x0[4], x1[4];
        kv4_word(u[2 * h], step, off, x0);
        kv4_word(u[2 * h + 1], step, off, x1);
#pragma unroll
        for (int e = 0; e < 2; ++e) {  // the pair's tokens
          const uint32_t sel = e ? 0x7632 : 0x5410;
          asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"((at ^ 16 * (h ^ e)) + 128 * e), "r"(__byte_perm(x0[0], x0[1], sel)),
                       "r"(__byte_perm(x0[2], x0[3], sel)), "r"(__byte_perm(x1[0], x1[1], sel)), "r"(__byte_perm(x1[2], x1[3], sel))
                       : "memory");
        }
      }
    }
  };

  CodeChunk c[kSteps];
  TileItem w;
  int k = 0;
  uint32_t gt = 0;
  bool ok = true;
  do {
    w.load(p, &sh.list[k]);
    const int tiles = w.tiles;
    if (tiles == 0) continue;
    const char *now = tile_of(w, 0, tiles), *next = tile_of(w, 1, tiles);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) load(c[i], 0, i, now);
    for (int j = 0; j < tiles && ok; ++j, ++gt) {
#pragma unroll
      for (int v = 0; v < 2; ++v) {
        const uint32_t idx = 2 * gt + v;
        const int s = idx % C::kSlots;
        if (idx >= C::kSlots) ok = ok && wait_spaced<20>(&sh.empty[s], (idx / C::kSlots - 1) & 1, gave_up);
        if (!ok) break;
        if (v == 0 && me == 0) {
          const unsigned held = __ballot_sync(~0u, now != nullptr) & 0xFFFFu;
          if (lane == 0) sh.held[gt % kHeldSets] = held;
        }
        const uint32_t slot_at = smem_u32(ring + s * C::kSlot);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
          store(c[i], v, i, slot_at);
          load(c[i], 1 - v, i, v == 0 ? now : next);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.full[s]);
      }
      now = next;
      next = tile_of(w, j + 2, tiles);
    }
  } while (ok && uniform(next_item(k)));
  if (!ok) leave();
}

// kCodes: over the cache in 4 bits, F16 being the type of its products.
template <int HDP, bool F16, bool kCodes>
__global__ void __launch_bounds__(kThreads<kCodes>, 1) k_attend_tile(const __grid_constant__ AttnParams p) {
  using C = TileCfg<HDP>;
  extern __shared__ char raw[];
  char* base = (char*)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
  char* qbuf = base;
  char* ring = base + C::kQ;
  TileShared& sh = *(TileShared*)(ring + C::kSlots * C::kSlot);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

  if (tid == 0) {
    for (int s = 0; s < C::kSlots; ++s) {
      mbar_init(&sh.full[s], kCodes ? C::kCodeWarps : 1);
      mbar_init(&sh.empty[s], 1);
    }
    mbar_init(&sh.q_full, 1);
    mbar_init(&sh.q_empty, 1);
    mbar_init(&sh.q_ready[0], 4);
    mbar_init(&sh.q_ready[1], 4);
    for (int s = 0; s < 3; ++s) {  // 2: the second score buffer with one row tile
      mbar_init(&sh.s_full[s], 1);
      mbar_init(&sh.p_ready[s], kCodes ? 4 : 5);  // four warps of rows, and warp 11
    }
    mbar_init(&sh.o_full[0], 1);
    mbar_init(&sh.o_full[1], 1);
    mbar_init(&sh.o_step, 1);
    mbar_init(&sh.drain, 1);
    for (int i = 0; i < kOddSets; ++i) mbar_init(&sh.odd_read[i], 8);
    sh.gave_up = 0;
    mbar_init_fence();
  }
  launch_dependents();
  // The requests, in the room of the ring: first item, new tokens, keys, pairs.
  int4* const reqs = (int4*)ring;
  {
    const int per = (p.batch + kThreads<kCodes> - 1) / kThreads<kCodes>, lo = min(tid * per, p.batch), hi = min(lo + per, p.batch);
    int64_t sum = 0, keys = 0;  // items and keys
    bool bad = false;
    for (int i = lo; i < hi; ++i) {
      bad |= attn_falls(p, i);
      const AttnReq r = attn_req(p, i);
      const int pairs = pairs_of(p, r.ql);
      reqs[i] = make_int4((int)sum, r.ql, r.kvl, pairs);
      sum += (int64_t)pairs * p.kv_heads;
      keys += pairs > 0 ? r.kvl : 0;
    }
    int64_t inc = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t v = __shfl_up_sync(~0u, inc, d);
      if (lane >= d) inc += v;
      keys += __shfl_xor_sync(~0u, keys, d);
    }
    if (lane == 31) {
      sh.scratch[warp] = inc;
      sh.scratch[16 + warp] = keys;
    }
    bad = __syncthreads_or(bad);
    int64_t before = inc - sum, all = 0;
    keys = 0;
    for (int w = 0; w < kThreads<kCodes> / 32; ++w) {
      if (w < warp) before += sh.scratch[w];
      all += sh.scratch[w];
      keys += sh.scratch[16 + w];
    }
    for (int i = lo; i < hi; ++i) reqs[i].x += (int)before;
    if (tid == 0) {
      sh.items = bad || all > INT32_MAX ? 0 : (int)all;  // (2^31 items: q would not fit in memory)
      sh.stride = kCodes || keys * p.kv_heads * p.dim * 4 > kNaturalBytes ? (int)gridDim.x : 1;
    }
    __syncthreads();
  }
  const int items = sh.items, stride = sh.stride;
  // column c begins at item c, or in natural order at the c-th of equal runs
  const int run = (items + (int)gridDim.x - 1) / (int)gridDim.x;
  int at_req = 0;  // request of the thread's last item (they mostly come in rising order)
  auto cost_of = [&](int item) -> int {
    int hi = p.batch - 1;
    if (reqs[at_req].x > item) at_req = 0;
    while (at_req < hi) {
      const int mid = (at_req + hi + 1) / 2;
      if (reqs[mid].x <= item) at_req = mid;
      else hi = mid - 1;
    }
    const int4 r = reqs[at_req];
    return pair_cost(p, r.y, r.z, (item - r.x) % r.w) + kItem<kCodes>;
  };
  const AttnRange range = attn_range<kThreads<kCodes>>((int)gridDim.x, blockIdx.x, gridDim.x, sh.scratch, [&](int c) -> int64_t {
    int64_t sum = 0;
    const int64_t end = stride > 1 ? items : min((int64_t)items, (int64_t)(c + 1) * run);
    for (int64_t i = stride > 1 ? c : (int64_t)c * run; i < end; i += stride) sum += cost_of((int)i);
    return sum;
  });
  if (tid == 0) p.desc[blockIdx.x] = make_int4(0, 0, 0, 0);
  if (range.begin >= range.end) return;
  if (warp == 11) {  // the block's first item, in column range.req
    int64_t item = stride > 1 ? range.req : (int64_t)range.req * run, rest = range.off;
    for (;;) {
      const int64_t mine = item + (int64_t)lane * stride;
      const int cost = mine < items ? cost_of((int)mine) : 0;
      int64_t inc = cost;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int64_t v = __shfl_up_sync(~0u, inc, d);
        if (lane >= d) inc += v;
      }
      const unsigned past = __ballot_sync(~0u, inc > rest);
      if (past) {
        const int k = __ffs(past) - 1;
        rest -= __shfl_sync(~0u, inc - cost, k);
        item += (int64_t)k * stride;
        break;
      }
      rest -= __shfl_sync(~0u, inc, 31);
      item += (int64_t)32 * stride;
    }
    if (lane == 0) {
      sh.item = (int)item;
      sh.column = stride > 1 ? range.req : 0;
      sh.t0 = (int)rest;
      sh.left = range.end - range.begin;
    }
    __syncwarp();
    fill_list<kCodes>(p, sh);
  }
  __syncthreads();  // the requests are done with: the ring is free

  // rows that no copy fills (whole tokens only in a tile) stay 0
  for (int e = tid; e < C::kQ / 16; e += kThreads<kCodes>) ((uint4*)qbuf)[e] = make_uint4(0, 0, 0, 0);
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&sh.tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = sh.tmem;  // S0/P0 at 0, S1/P1 at 128, O0 at 256, O1 at 384
  int* const gave_up = &sh.gave_up;
  // The next entry of the list; at its end, where the block has more items, all
  // roles meet and warp 11 writes the next ones.
  auto next_item = [&](int& k) -> bool {
    if (++k < sh.count) return true;
    if (!sh.more) return false;
    bar_all<kCodes>();
    if (warp == 11) fill_list<kCodes>(p, sh);
    bar_all<kCodes>();
    k = 0;
    return true;
  };
  // A role that has given up still meets the others.
  auto leave = [&] {
    while (sh.more) {
      bar_all<kCodes>();
      if (warp == 11) fill_list<kCodes>(p, sh);
      bar_all<kCodes>();
    }
  };

  if (kCodes && C::kTiles == 1 && warp >= 4 && warp < 8) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::template kRowRegs<kCodes>));
    widen_codes<HDP>(p, sh, ring, warp + 3, next_item, leave);
  } else if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::template kRoleRegs<kCodes>));
    if (kCodes && warp > 8) {
      // ---- codes: warps 9 to 15 make f16 keys and values of them ----
      widen_codes<HDP>(p, sh, ring, warp - 9, next_item, leave);
    } else if (warp == 9 || warp == 10) {
      // ---- copies: warp 9 queries and keys, warp 10 values ----
      // Tile g of the block (over all its items) has its keys in use 2 g of the
      // ring and its values in use 2 g + 1.  A warp waits for every second use's
      // slot only; the products release the uses in order, so a use that has
      // been released implies all before it, and no wait is a phase early.
      TileItem w;
      int k = 0;
      const int v = warp - 9, box = p.box, per = kKeys / box;
      const CUtensorMap* const map = v ? &p.map_v : &p.map_k;
      uint32_t item = 0, gt = 0;
      bool ok = true;
      do {
        w.load(p, &sh.list[k]);
        if (w.tiles == 0) continue;
        const int head = (int)uniform((uint32_t)w.e.head), t0 = (int)uniform((uint32_t)w.e.t0), tiles = (int)uniform((uint32_t)w.tiles);
        if (v == 0) {
          if (item > 0) ok = ok && wait_all(&sh.q_empty, (item - 1) & 1, gave_up);
          if (!ok) break;
          const int rows = w.n1 > 0 ? 2 : 1;  // the second row tile sees at least what the first does
          const int tok = (int)uniform((uint32_t)(w.e.q0 + w.tok0)), toks = p.toks;
          if (lane == 0) mbar_arrive_expect_tx(&sh.q_full, rows * toks * p.group * 128 * C::kBlk);
          __syncwarp();
          if (elect_one())
            for (int s = 0; s < rows; ++s)
#pragma unroll
              for (int b = 0; b < C::kBlk; ++b)
                tma_load_3d(qbuf + (s * C::kBlk + b) * 128 * 128, &p.map_q, b * 64, head * p.group, tok + s * toks, &sh.q_full);
          __syncwarp();
          ++item;
        } else {
          // Warp 11 writes an item's notes once its first values are there, and
          // they are copied once the set's last notes have been read: a row tile
          // that adds keys one by one may be several items behind the other,
          // where those have no part of it.  For an absent row tile this warp arrives.
          const uint32_t set = item % kOddSets;
          if (item >= kOddSets) ok = ok && wait_spaced<100>(&sh.odd_read[set], (item / kOddSets - 1) & 1, gave_up);
          if (!ok) break;
          if (lane == 0 && (w.n0 == 0 || w.n1 == 0)) mbar_arrive_n(&sh.odd_read[set], 4);
          ++item;
        }
        const int32_t* row = p.table + (int64_t)w.e.req * p.table_stride;
        const int kvl = w.e.kvl;
        auto page_of = [&](int j) -> int {  // lane b: page of the tile's b-th box
          const int64_t key = (int64_t)(t0 + j) * kKeys + lane * box;
          if (j >= tiles || lane >= per || key >= kvl) return -1;
          const int id = row[key >> p.page_log2];
          return id < 0 || id >= p.n_pages ? -1 : id;
        };
        int next = page_of(0);
        for (int j = 0; j < tiles; ++j, ++gt) {
          const int id = next;
          next = page_of(j + 1);
          const uint32_t idx = 2 * gt + v;
          const int s = idx % C::kSlots;
          if (idx >= C::kSlots) ok = ok && wait_spaced<20>(&sh.empty[s], (idx / C::kSlots - 1) & 1, gave_up);
          if (!ok) break;
          const unsigned held = __ballot_sync(~0u, id >= 0);
          if (lane == 0) {
            if (v == 0) {
              uint32_t m = 0;
              for (int g = 0; g < kKeys / 8; ++g) m |= (held >> (g * 8 / box) & 1u) << g;
              sh.held[gt % kHeldSets] = m;
            }
            mbar_arrive_expect_tx(&sh.full[s], C::kSlot);
          }
          __syncwarp();
          const int slot = ((t0 + j) * kKeys) & ((1 << p.page_log2) - 1);
          char* const dst = ring + s * C::kSlot;
          for (int i = 0; i < per; ++i) {
            const int page = __shfl_sync(~0u, id, i);
            if (elect_one()) {
#pragma unroll
              for (int b = 0; b < C::kBlk; ++b)
                if (!KV_BAD(g_tile_counts, page >= -1 && page < p.n_pages && slot < 1 << p.page_log2 && i < per))
                tma_load_4d(dst + b * kKeys * 128 + i * box * 128, map, b * 64, slot, head, page, &sh.full[s]);
            }
          }
          __syncwarp();
        }
      } while (ok && uniform(next_item(k)));
      if (lane == 0) {
        sh.sent[v] = gt;
        if (v == 0) sh.asked = item;
      }
      if (!ok) leave();
    } else if (warp == 8) {
      // ---- products ----
      // The whole warp takes every step and one lane issues, with operands that
      // the compiler knows to be the same in all lanes (the broadcasts): issued
      // from a branch of one lane, each product cost about 100 cycles.
      TileItem w;
      int k = 0;
      constexpr uint32_t acc = 0;  // all 512 columns are this block's: they begin at 0
      const int steps = (p.dim + 15) / 16;  // of 16 elements of a head; columns of O likewise
      const uint32_t kind = 1u << 4 | (F16 ? 0u : 1u << 7 | 1u << 10) | 8u << 24;  // 32-bit sums, 128 rows
      const uint32_t desc_s = kind | (kKeys >> 3) << 17, desc_o = kind | 1u << 16 | (uint32_t)(steps * 16 >> 3) << 17;
      const uint32_t q_at = operand_low(smem_u32(qbuf), 0), ring_at = operand_low(smem_u32(ring), 0);
      constexpr uint32_t kSlotStep = C::kSlot >> 4, kBlocks = (uint32_t)(kKeys * 128) >> 4 << 16;
      uint32_t item = 0, ready = 0;
      bool ok = true;
      // from P at column `at`, into row tile s's output
      auto outputs = [&](int s, int at, int slot, bool add) {  // by one lane
        const uint32_t v_at = (ring_at + slot * kSlotStep) | kBlocks;
#pragma unroll
        for (int k = 0; k < kKeys / 16; ++k)
          mma_ts(acc + 256 + s * 128, acc + at + k * 8, v_at + k * (2048 >> 4), desc_o, add || k > 0);
      };
      // of row tile s, into column `at`
      auto scores = [&](int s, int at, int bar, int slot) {  // by one lane
        const uint32_t a = q_at + s * (C::kBlk * 128 * 128 >> 4), b = ring_at + slot * kSlotStep;
#pragma unroll
        for (int k = 0; k < HDP / 16; ++k) {
          const uint32_t off = (k >> 2) * (128 * 128 >> 4) + (k & 3) * 2;
          if (k < steps) mma_ss(acc + at, a + off, b + off, desc_s, k > 0);
        }
        commit(&sh.s_full[bar]);
      };
      auto after = [](int slot, int n) { return slot + n < C::kSlots ? slot + n : slot + n - C::kSlots; };
      int sk = 0;          // slot of the next key tile; its values follow
      uint32_t phase = 0;  // of the ring at that slot
      do {
        w.load(p, &sh.list[k]);
        const int tiles = (int)uniform((uint32_t)w.tiles), n0 = (int)uniform((uint32_t)w.n0), n1 = (int)uniform((uint32_t)w.n1);
        if (tiles == 0) continue;
        if constexpr (kCodes) {  // bits 0 and 1 of item: phases of the row tiles' queries
          if (n0 > 0) ok = wait_all(&sh.q_ready[0], item & 1, gave_up);
          if (n1 > 0) ok = ok && wait_all(&sh.q_ready[1], item >> 1, gave_up);
          item ^= (n0 > 0 ? 1 : 0) | (n1 > 0 ? 2 : 0);
          ok = ok && wait_all(&sh.full[sk], phase, gave_up);
        } else {
          ok = wait_all(&sh.q_full, item & 1, gave_up) && wait_all(&sh.full[sk], phase, gave_up);
          ++item;
        }
        if (!ok) break;
        fence_after();
        if (elect_one()) {
          if (n0 > 0) scores(0, 0, 0, sk);
          if (n1 > 0) scores(1, 128, 1, sk);
          commit(&sh.empty[sk]);
          if (tiles == 1) commit(&sh.q_empty);
        }
        __syncwarp();
        // kCodes: the phase of the values in slot `at`, which the keys in `key_slot` came before in phase `ph`
        auto values_in = [&](int at, int key_slot, uint32_t ph) { return wait_all(&sh.full[at], at < key_slot ? ph ^ 1 : ph, gave_up); };
        if constexpr (C::kTiles == 1) {
          // The next scores are made while this tile's P is.
          int sv = after(sk, 1);
          uint32_t v_phase = sv < sk ? phase ^ 1 : phase;
          auto step = [&] {
            if (sk + 2 >= C::kSlots) phase ^= 1;
            sk = after(sk, 2);
          };
          step();
          if (tiles > 1) {
            ok = wait_all(&sh.full[sk], phase, gave_up);
            if (!ok) break;
            fence_after();
            if (elect_one()) {
              scores(0, 128, 2, sk);
              commit(&sh.empty[sk]);
              if (tiles == 2) commit(&sh.q_empty);
            }
            __syncwarp();
            step();
          }
          for (int j = 0; j < tiles; ++j) {
            const int b = j & 1 ? 2 : 0;
            ok = wait_all(&sh.p_ready[b], ready >> b & 1, gave_up);
            ready ^= 1u << b;
            if (kCodes) ok = ok && wait_all(&sh.full[sv], v_phase, gave_up);
            if (!ok) break;
            fence_after();
            if (elect_one()) {
              outputs(0, j & 1 ? 128 : 0, sv, j > 0);
              commit(&sh.empty[sv]);
              if (j + 2 == tiles) commit(&sh.o_step);
              if (j + 1 == tiles) commit(&sh.o_full[0]);
            }
            __syncwarp();
            if (sv + 2 >= C::kSlots) v_phase ^= 1;
            sv = after(sv, 2);
            if (j + 2 < tiles) {
              if (!C::kWatchKeys || kCodes) ok = wait_all(&sh.full[sk], phase, gave_up);
              if (!ok) break;
              if (kCodes) fence_after();
              if (elect_one()) {
                scores(0, j & 1 ? 128 : 0, b, sk);
                commit(&sh.empty[sk]);
                if (j + 3 == tiles) commit(&sh.q_empty);
              }
              __syncwarp();
              step();
            }
          }
        } else {
          for (int j = 0; j < tiles; ++j) {
            const int sv = after(sk, 1), sk0 = sk;
            const uint32_t phase0 = phase;
            if (sk + 2 >= C::kSlots) phase ^= 1;
            sk = after(sk, 2);
            const bool more = j + 1 < tiles;
            if constexpr (kCodes) {  // long there, mostly
              ok = values_in(sv, sk0, phase0) && (!more || wait_all(&sh.full[sk], phase, gave_up));
              if (!ok) break;
            }
            // p_ready is complete once P stands, and this tile's values and the
            // next one's keys are there (warp 11 waits for those): one wait here
            if (j < n0) {
              ok = wait_all(&sh.p_ready[0], ready & 1, gave_up);
              ready ^= 1;
              if (!ok) break;
              fence_after();
              if (elect_one()) {
                outputs(0, 0, sv, j > 0);
                if (j >= n1) commit(&sh.empty[sv]);
                if (j + 1 < n0) scores(0, 0, 0, sk);
                else commit(&sh.o_full[0]);
                if (more && j + 1 >= n1) {
                  commit(&sh.empty[sk]);
                  if (j + 2 == tiles) commit(&sh.q_empty);  // no more scores
                }
              }
              __syncwarp();
            }
            if (j < n1) {
              ok = wait_all(&sh.p_ready[1], ready >> 1, gave_up);
              ready ^= 2;
              if (!ok) break;
              fence_after();
              if (elect_one()) {
                outputs(1, 128, sv, j > 0);
                commit(&sh.empty[sv]);
                if (j + 1 < n1) {
                  scores(1, 128, 1, sk);
                  commit(&sh.empty[sk]);
                  if (j + 2 == tiles) commit(&sh.q_empty);
                } else {
                  commit(&sh.o_full[1]);
                }
              }
              __syncwarp();
            }
          }
        }
      } while (ok && uniform(next_item(k)));
      // nothing in flight when the tensor memory goes
      if (elect_one()) commit(&sh.drain);
      __syncwarp();
      for (int i = 0; i < 1 << 20 && !mbar_try_wait(&sh.drain, 0); ++i) {
      }
      __syncwarp();
      if (!ok) leave();
    } else {
      // ---- copies that have landed, and values that some row must not see ----
      TileItem w;
      int k = 0;
      uint32_t idx = 0, item = 0, ready = 0, due = 0;  // idx: ring use of tile j's keys; due: score buffers with a phase to end
      bool ok = true;
      do {
        w.load(p, &sh.list[k]);
        if (w.tiles == 0) continue;
        uint32_t* odd = sh.odd[item % kOddSets];
        ++item;
        for (int j = 0; j < w.tiles && ok; ++j, idx += 2) {
          const uint32_t vi = idx + 1, ki = idx + 2;
          const int s = vi % C::kSlots;
          ok = wait_spaced<100>(&sh.full[s], (vi / C::kSlots) & 1, gave_up);
          if (!ok) break;
          if (j == 0) {
            if (lane < 9) odd[lane] = 0;
            __syncwarp();
          }
          if (w.partly(j)) {
            const uint32_t at = smem_u32(ring + s * C::kSlot);
            const int key0 = (w.e.t0 + j) * kKeys;
            const int from = w.lim_first > key0 ? w.lim_first - key0 : 0;
            bool wrote = false;
            // lane i looks at the i-th 16 bytes of two rows (four where a head has 64 elements)
            constexpr int kChunks = HDP / 8, kAtOnce = 32 / kChunks, kLoads = 8;
            const int ch = lane % kChunks;
            const uint32_t mine = at + (ch >> 3) * (kKeys * 128) + ((ch & 7) << 4);  // any order within a row's 128 bytes
#pragma unroll 1
            for (int row0 = from / (kLoads * kAtOnce) * (kLoads * kAtOnce); row0 < kKeys; row0 += kLoads * kAtOnce) {
              uint4 x[kLoads];
              uint32_t any = 0;
#pragma unroll
              for (int u = 0; u < kLoads; ++u)
                asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                             : "=r"(x[u].x), "=r"(x[u].y), "=r"(x[u].z), "=r"(x[u].w)
                             : "r"(mine + (row0 + u * kAtOnce + lane / kChunks) * 128));
#pragma unroll
              for (int u = 0; u < kLoads; ++u) any |= not_finite8<F16>(x[u]);
              if (!__any_sync(~0u, any != 0)) continue;
#pragma unroll 1
              for (int row = row0 > from ? row0 : from; row < row0 + kLoads * kAtOnce; ++row) {  // row by row; seldom
                uint4 y = make_uint4(0, 0, 0, 0);
                if (lane < kChunks)
                  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(y.x), "=r"(y.y), "=r"(y.z), "=r"(y.w) : "r"(mine + row * 128));
                if (!__any_sync(~0u, not_finite8<F16>(y) != 0)) continue;
                wrote = true;
                if (lane < kChunks) asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(mine + row * 128), "r"(0) : "memory");
                const int key = key0 + row, a = key - w.lim_first;  // a < 256 for every token of the item
                if (lane == 0 && key < w.e.kvl && a < 256 && !KV_BAD(g_tile_counts, a >= 0 && row < kKeys)) {
                  odd[a >> 5] |= 1u << (a & 31);
                  odd[8] = 1;
                }
              }
            }
            if (wrote) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
          }
          if (C::kWatchKeys && j + 1 < w.tiles) ok = wait_spaced<100>(&sh.full[ki % C::kSlots], (ki / C::kSlots) & 1, gave_up);
          if (!ok) break;
          // not a tile ahead of the rows, or two arrivals would count in one phase
          constexpr int kSecond = C::kTiles == 1 ? 2 : 1;
          if (due & 1) ok = wait_spaced<100>(&sh.p_ready[0], ready & 1, gave_up);
          if (ok && (due & 2)) ok = wait_spaced<100>(&sh.p_ready[kSecond], ready >> 1, gave_up);
          if (!ok) break;
          ready ^= due;
          due = C::kTiles == 1 ? 1 + (j & 1) : (j < w.n0 ? 1 : 0) | (j < w.n1 ? 2 : 0);
          if (lane == 0) {
            if (due & 1) mbar_arrive(&sh.p_ready[0]);
            if (due & 2) mbar_arrive(&sh.p_ready[kSecond]);
          }
          __syncwarp();
        }
      } while (ok && uniform(next_item(k)));
      if (!ok) leave();
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::template kRowRegs<kCodes>));
    // ---- one row per thread ----
    TileItem w;
    int k = 0;
    const int s = warp >> 2, r = tid & 127, r_tok = r / p.group, sub = r % p.group;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21, t_s = tmem + s * 128 + lanes, t_o = tmem + 256 + s * 128 + lanes;
    uint32_t scored = 0, done = 0, item = 0, gt = 0, steps = 0;  // scored: phases of this row tile's buffer and of buffer 2
    bool ok = true;
    // kCodes: an item's queries for this row tile; returns the row's scale.  Where
    // the row has read the last scores of the item before, its queries are free.
    auto stage = [&](const TileItem& x) -> float {
      if (x.count(s) == 0) return p.scale_log2;
      const int64_t t = (int64_t)x.tok0 + s * p.toks + r_tok, at = x.e.q0 + t, head = (int64_t)x.e.head * p.group + sub;
      const bool mine = r_tok < p.toks && t < x.e.ql && !KV_BAD(g_tile_counts, at >= 0 && at < p.tokens && head >= 0 && head < p.heads);
      const float back =
          stage_query<HDP>(mine ? p.q + 2 * (at * p.q_tok + head * p.q_head) : nullptr, p.dim, p.f16, qbuf + s * C::kBlk * 128 * 128, r);
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.q_ready[s]);
      return kv4_scale(p.scale_log2, back);
    };
    bool staged = false;
    float scale_next = 0.f;
    do {
      w.load(p, &sh.list[k]);
      const int64_t first_tok = (int64_t)w.tok0 + s * p.toks;
      const bool valid = r_tok < p.toks && first_tok + r_tok < w.e.ql;
      const int tok = valid ? (int)first_tok + r_tok : 0;
      float scale_log2 = p.scale_log2;
      if constexpr (kCodes) {
        scale_log2 = staged ? scale_next : stage(w);
        staged = false;
      }
      const int lim = valid ? w.limit(p, tok) : INT32_MAX;
      const int lim_tile = first_tok < w.e.ql ? w.limit(p, (int)first_tok) : 0;  // what every row of the tile sees
      float m = -INFINITY, l = 0.f;
      for (int j = 0; j < w.count(s); ++j) {
        const bool second = C::kTiles == 1 && (j & 1);  // of the two score buffers
        const int buf = second ? 2 : s;
        const uint32_t t_p = second ? t_s + 128 : t_s;
        ok = wait_all(&sh.s_full[buf], second ? scored >> 1 : scored & 1, gave_up);
        scored ^= second ? 2 : 1;
        if (C::kTiles == 1 && ok && j > 0 && j + 1 == w.n0) {  // no scores follow: the outputs before the last tile
          ok = wait_all(&sh.o_step, steps & 1, gave_up);
          ++steps;
        }
        if (!ok) break;
        fence_after();
        float f[128];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32(f + 32 * c, t_p + 32 * c);
        wait_ld();
        const uint32_t held = sh.held[(gt + j) % kHeldSets];
        const int key0 = (w.e.t0 + j) * kKeys;
        if (held != 0xFFFFu) {  // pages that the cache does not hold, 8 keys at a time
#pragma unroll
          for (int g = 0; g < 16; ++g)
            if (!(held >> g & 1u)) {
#pragma unroll
              for (int c = 8 * g; c < 8 * g + 8; ++c) f[c] = -INFINITY;
            }
        }
        if (lim_tile - key0 < kKeys) {
          const int sees = lim - key0;
#pragma unroll
          for (int c = 0; c < 128; ++c) f[c] = c < sees ? f[c] : -INFINITY;
        }
        float mx[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) mx[q] = max3(f[q], f[4 + q], f[8 + q]);
#pragma unroll
        for (int c = 12; c + 8 <= 128; c += 8)
#pragma unroll
          for (int q = 0; q < 4; ++q) mx[q] = max3(mx[q], f[c + q], f[c + 4 + q]);
#pragma unroll
        for (int q = 0; q < 4; ++q) mx[q] = fmaxf(mx[q], f[124 + q]);
        const float top = L<F16>::reference(fmaxf(m, fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * scale_log2));
        if (j == 0) {
          m = top;
        } else if (__any_sync(~0u, top - m > kLag<F16>)) {
          if (C::kTiles == 1 && j + 1 < w.n0) {
            // These scores did not wait for the outputs of the tile before; the
            // next ones, issued after those outputs, do.
            ok = wait_all(&sh.s_full[second ? 0 : 2], (second ? scored : scored >> 1) & 1, gave_up);
            if (!ok) break;
            fence_after();
          }
          const bool grows = top - m > kLag<F16>;
          const float a = grows ? ex2(m - top) : 1.f;
          m = grows ? top : m;
          l *= a;
#pragma unroll 1
          for (int c = 0; c < HDP; c += 16) {
            float o[16];
            uint32_t u[16];
            tmem_ld16(o, t_o + c);
            wait_ld();
#pragma unroll
            for (int e = 0; e < 16; ++e) u[e] = __float_as_uint(o[e] * a);
            tmem_st16(t_o + c, u);
          }
          wait_st();
        }
        const float ref = m == -INFINITY ? 0.f : m;
        // P, rounded to the cache's type (the operand's), over S
        uint64_t sum[2] = {0, 0};  // pairs of 32-bit sums
        const uint64_t mul = pair(scale_log2, scale_log2), off = pair(L<F16>::kLift - ref, L<F16>::kLift - ref);
#pragma unroll
        for (int c = 0; c < 128; c += 32) {
          uint32_t x[16];
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            float a, b;
            unpair(fma2(pair(f[c + e], f[c + e + 1]), mul, off), a, b);
            a = ex2(a);
            b = ex2(b);
            sum[e / 2 & 1] = add2(sum[e / 2 & 1], pair(a, b));
            x[e / 2] = pack2<F16>(a, b);
          }
          tmem_st16(t_p + c / 2, x);
        }
        float s0, s1;
        unpair(add2(sum[0], sum[1]), s0, s1);
        l += s0 + s1;
        wait_st();
        fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.p_ready[buf]);
      }
      if (!ok) break;
      if constexpr (kCodes) {
        // The next item's queries before this one's output, so that its first
        // scores are made meanwhile.
        if (k + 1 < sh.count) {
          TileItem next;
          next.load(p, &sh.list[k + 1]);
          scale_next = stage(next);
          staged = true;
        }
      }
      gt += w.tiles;
      const uint32_t* odd = nullptr;
      if (!kCodes && w.tiles > 0) odd = sh.odd[item++ % kOddSets];
      if (w.count(s) > 0) {
        ok = wait_all(&sh.o_full[s], done & 1, gave_up);
        ++done;
        if (!ok) break;
        fence_after();
      }
      // ---- out ----
      const int cost = pair_cost(p, w.e.ql, w.e.kvl, w.e.pair);
      const bool starts = w.e.t0 == 0, ends = w.e.t0 + w.e.seg == cost, whole = starts && ends;
      if (s < C::kTiles && first_tok < w.e.ql) {
        const bool extra = odd && w.count(s) > 0 && odd[8];
        const float inv = l == 0.f ? 0.f : 1.f / l, scale = whole ? inv : 1.f;
        const int64_t tok_at = (int64_t)w.e.q0 + tok, head = (int64_t)w.e.head * p.group + sub;
        const bool inside = valid && !KV_BAD(g_tile_counts, tok_at >= 0 && tok_at < p.tokens && head >= 0 && head < p.heads);
        char* const out = p.out + 2 * (tok_at * p.out_tok + head * p.out_head);
        float* part = p.part + ((int64_t)blockIdx.x * 2 + (starts ? 1 : 0)) * (C::kRows * HDP + 2 * C::kRows);
        for (int c = 0; c < HDP / 32; ++c) {
          float o[32];
          if (w.count(s) > 0) {
            tmem_ld32(o, t_o + 32 * c);
            wait_ld();
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = 0.f;
          }
          if (!kCodes && extra && valid) {
            // seen keys whose values were blanked for the other rows
            const char* q = p.q + 2 * (tok_at * p.q_tok + head * p.q_head);
            for (int a = 0; a < 256; ++a) {
              if (!(odd[a >> 5] >> (a & 31) & 1u) || a >= lim - w.lim_first) continue;
              const int key = w.lim_first + a;
              if (KV_BAD(g_tile_counts, key >= 0 && key < w.e.kvl)) continue;
              const int64_t id = p.table[(int64_t)w.e.req * p.table_stride + (key >> p.page_log2)];
              if (id < 0 || id >= p.n_pages) continue;
              const int64_t slot = key & ((1 << p.page_log2) - 1);
              const char* kp = p.k + 2 * (id * p.k_page + slot * p.k_slot + w.e.head * p.k_head);
              const char* vp = p.v + 2 * (id * p.v_page + slot * p.v_slot + w.e.head * p.v_head);
              float dot = 0.f;
              for (int d = 0; d < p.dim; d += 2) {
                const float2 a2 = unpack2<F16>(*(const uint32_t*)(q + 2 * d)), b2 = unpack2<F16>(*(const uint32_t*)(kp + 2 * d));
                dot = fmaf(a2.x, b2.x, fmaf(a2.y, b2.y, dot));
              }
              const float pr = ex2(fmaf(dot, p.scale_log2, L<F16>::kLift - (m == -INFINITY ? 0.f : m)));
#pragma unroll
              for (int e = 0; e < 32; e += 2)
                if (32 * c + e < p.dim) {
                  const float2 v2 = unpack2<F16>(*(const uint32_t*)(vp + 2 * (32 * c + e)));
                  o[e] = fmaf(pr, v2.x, o[e]);
                  o[e + 1] = fmaf(pr, v2.y, o[e + 1]);
                }
            }
          }
          if (whole) {
            uint32_t v[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = pack_as<F16, kCodes>(p, o[2 * e] * scale, o[2 * e + 1] * scale);
            if (inside && p.wide) {  // whole 32-byte sectors
#pragma unroll
              for (int e = 0; e < 2; ++e)
                if (32 * c + 16 * e < p.dim) store32(out + 2 * (32 * c + 16 * e), v + 8 * e);
            } else if (inside) {
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (32 * c + 8 * e < p.dim)
                  *(uint4*)(out + 2 * (32 * c + 8 * e)) = make_uint4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
            }
          } else {
            // [column / 4][row][4]: a warp's 32 rows are 512 contiguous bytes
#pragma unroll
            for (int e = 0; e < 32; e += 4)
              *(float4*)(part + ((int64_t)(8 * c + e / 4) * C::kRows + s * 128 + r) * 4) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
          }
        }
        if (whole) {
          if (inside && p.lse) p.lse[tok_at * p.heads + head] = L<F16>::lse(m, l);
        } else {
          part[C::kRows * HDP + s * 128 + r] = m;
          part[C::kRows * HDP + C::kRows + s * 128 + r] = l;
        }
      }
      if (!kCodes && w.count(s) > 0) {  // the notes are read
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.odd_read[(item - 1) % kOddSets]);
      }
      if (starts && !ends && tid == 0) {
        const int64_t first = range.end - w.e.seg;  // the item's first unit
        p.desc[blockIdx.x] = make_int4(w.e.req, w.e.head, w.e.pair, attn_block_of(range, first + cost - 1) - (int)blockIdx.x + 1);
      }
      fence_before();  // O is read before the next item's first product may write it
    } while (next_item(k));
    if (!ok) leave();
  }

  __syncthreads();
  // Where a role gave up, copies may be in flight that nobody waited for: the
  // last uses of the ring (all before them were released, so they have landed)
  // and the last queries.  They land before the block ends.
  if ((warp == 9 || warp == 10) && *(volatile int*)gave_up) {
    if (tid == 9 * 32) atomicAdd(&g_tile_counts[kKvGaveUp], 1u);
    if (!kCodes) {
      const uint32_t v = warp - 9, n = sh.sent[v], last = (C::kSlots + 1) / 2;
      for (uint32_t k = n > last ? n - last : 0; k < n; ++k) {
        const uint32_t idx = 2 * k + v;
        wait_landed(&sh.full[idx % C::kSlots], (idx / C::kSlots) & 1);
      }
      if (v == 0 && sh.asked > 0) wait_landed(&sh.q_full, (sh.asked - 1) & 1);
    }
  }
  if (warp == 8) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
}

// Joins the parts of the item that block c began and did not end: a block per
// (c, 32 rows), a lane per row, a warp per eighth of the columns.  (Four times the
// blocks for a quarter of the columns each: 1 us less where 20 parts of 8 items
// are joined, 20 us more where 152 items of 2 parts are.)
template <int HDP, bool F16, bool kCodes>
__global__ void __launch_bounds__(256) k_attend_tile_join(const __grid_constant__ AttnParams p) {
  wait_for_primary();
  const int4 d = p.desc[blockIdx.x];
  if (d.w == 0) return;
  if (KV_BAD(g_tile_counts, d.w > 0 && d.w <= (int)(gridDim.x - blockIdx.x) && d.x >= 0 && d.x < p.batch && d.y >= 0 && d.y < p.kv_heads && d.z >= 0))
    return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const AttnReq r = attn_req(p, d.x);
  const int slot_row = blockIdx.y * 32 + lane, s = slot_row >> 7, row = slot_row & 127;
  const int64_t row_tok = (int64_t)d.z * p.item_toks + s * p.toks + row / p.group;
  if (row >= p.toks * p.group || row_tok >= r.ql) return;
  using C = TileCfg<HDP>;
  constexpr int64_t kSlot = C::kRows * HDP + 2 * C::kRows;
  constexpr int kCols = HDP / 8;
  const float* first = p.part + ((int64_t)blockIdx.x * 2 + 1) * kSlot;
  const float* rest = p.part + ((int64_t)blockIdx.x * 2 + 2) * kSlot;  // then every second slot
  float top = -INFINITY, sum = 0.f, acc[kCols];
#pragma unroll
  for (int c = 0; c < kCols; ++c) acc[c] = 0.f;
#pragma unroll 8
  for (int k = 0; k < d.w; ++k) top = fmaxf(top, (k ? rest + 2 * (k - 1) * kSlot : first)[C::kRows * HDP + slot_row]);
  const float safe = top == -INFINITY ? 0.f : top;
#pragma unroll 8  // reads in flight: 20 parts of 8 items 42.5 -> 40.6 us a call (4); 16, or rounds with absent parts, no better
  for (int k = 0; k < d.w; ++k) {
    const float* at = k ? rest + 2 * (k - 1) * kSlot : first;
    const float f = ex2(at[C::kRows * HDP + slot_row] - safe);
    sum = fmaf(f, at[C::kRows * HDP + C::kRows + slot_row], sum);
#pragma unroll
    for (int c = 0; c < kCols; c += 4) {
      const float4 v = *(const float4*)(at + ((int64_t)(warp * kCols + c) / 4 * C::kRows + slot_row) * 4);
      acc[c] = fmaf(f, v.x, acc[c]);
      acc[c + 1] = fmaf(f, v.y, acc[c + 1]);
      acc[c + 2] = fmaf(f, v.z, acc[c + 2]);
      acc[c + 3] = fmaf(f, v.w, acc[c + 3]);
    }
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  const int64_t tok = r.q0 + row_tok, head = (int64_t)d.y * p.group + row % p.group;
#pragma unroll
  for (int c = 0; c < kCols; c += 8) {
    const int col = warp * kCols + c;
    if (col >= p.dim) break;
    uint4 v;
    v.x = pack_as<F16, kCodes>(p, acc[c] * inv, acc[c + 1] * inv);
    v.y = pack_as<F16, kCodes>(p, acc[c + 2] * inv, acc[c + 3] * inv);
    v.z = pack_as<F16, kCodes>(p, acc[c + 4] * inv, acc[c + 5] * inv);
    v.w = pack_as<F16, kCodes>(p, acc[c + 6] * inv, acc[c + 7] * inv);
    *(uint4*)(p.out + 2 * (tok * p.out_tok + head * p.out_head + col)) = v;
  }
  if (p.lse && warp == 0) p.lse[tok * p.heads + head] = L<F16>::lse(top, sum);
}

template <int HDP, bool F16, bool kCodes = false>
cudaError_t launch(const AttnParams& p, int sms, int device, cudaStream_t stream) {
  using C = TileCfg<HDP>;
  // the warpgroups' shares have to fit the registers of the launch, or they would wait for ever
  static const cudaError_t fits = [] {
    cudaFuncAttributes a;
    const cudaError_t e = cudaFuncGetAttributes(&a, k_attend_tile<HDP, F16, kCodes>);
    return e != cudaSuccess ? e : a.numRegs * (kThreads<kCodes> / 128) >= (kCodes ? 2 : 1) * C::template kRoleRegs<kCodes> + 2 * C::template kRowRegs<kCodes> ? cudaSuccess : cudaErrorInvalidConfiguration;
  }();
  if (fits != cudaSuccess) return fits;
  static std::atomic<uint64_t> allowed;
  cudaError_t e = kv_allow_smem(k_attend_tile<HDP, F16, kCodes>, C::kSmem, device, allowed);
  if (e != cudaSuccess) return e;
  k_attend_tile<HDP, F16, kCodes><<<sms, kThreads<kCodes>, C::kSmem, stream>>>(p);
  if ((e = cudaGetLastError()) != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(sms, C::kRows / 32);
  cfg.blockDim = dim3(256);
  cfg.stream = stream;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_attend_tile_join<HDP, F16, kCodes>, p);
}

}  // namespace

// Floats of the partial results (after the blocks' descriptions).
static size_t tile_parts(int sms) { return (size_t)sms * 2 * (256 * 128 + 2 * 256); }

size_t attend4_tile_workspace(int sms) { return attn4_part_offset(sms) + tile_parts(sms) * sizeof(float); }

cudaError_t launch_attend4_tile(const AttnParams& p, int sms, int device, cudaStream_t stream) {
  if (p.dim <= 64) return launch<64, true, true>(p, sms, device, stream);
  if (p.dim <= 128) return launch<128, true, true>(p, sms, device, stream);
  return launch<256, true, true>(p, sms, device, stream);
}

size_t attend_tile_workspace(int sms) {  // a slot has as much room for 128 rows of 256 columns as for 256 of 128
  return (size_t)sms * kFewPerSm * sizeof(int4) + 256 + tile_parts(sms) * sizeof(float);
}

cudaError_t launch_attend_tile(const AttnParams& p, bool f16, int sms, int device, cudaStream_t stream) {
  if (p.dim <= 64) return f16 ? launch<64, true>(p, sms, device, stream) : launch<64, false>(p, sms, device, stream);
  if (p.dim <= 128) return f16 ? launch<128, true>(p, sms, device, stream) : launch<128, false>(p, sms, device, stream);
  return f16 ? launch<256, true>(p, sms, device, stream) : launch<256, false>(p, sms, device, stream);
}

cudaError_t attend_tile_counts(cudaStream_t stream, uint32_t* counts) {
  void* at = nullptr;
  const cudaError_t e = cudaGetSymbolAddress(&at, g_tile_counts);
  return e != cudaSuccess ? e : cudaMemcpyAsync(counts, at, sizeof(g_tile_counts), cudaMemcpyDeviceToHost, stream);
}

}  // namespace mpt
