// New keys and values on their way into the pages (include/mpt_kv.h): turned by
// their positions, in 16 bits (mpt_kv_write_rotated) or as codes of 4 bits
// (mpt_kv4_write), the queries turned beside them; and codes read back
// (mpt_kv4_read).
//
// A warp takes a token, or a part of its heads where tokens are few: 8 elements
// a lane, as many heads at once as fit.  Cosines and sines of the token's row
// are read once and kept for all its heads.  An element's partner in the turn
// is in the same lane (adjacent ones) or rot / 16 lanes away, from where a
// shuffle brings it; so a head may be written where it was read.
//
// Bound: the memory.  What is turned is read and written once, and codes are
// 4.5 bits an element.  A token's chain of reads (request, page, cosines, values)
// is long, so what counts is how many warps are there to hide it: eight blocks of
// four an SM, which 64 registers allow, are worth more than more loads in flight in
// each (31,175 tokens of 32 query and 8 KV heads of 128, turned: 151 us with 88
// registers, 180 with 92 and loads that run ahead, 119 with 64; of codes, seven
// blocks and two steps at once).  The arithmetic of the codes, about 12 operations
// an element, does not hide whole: without it the write takes 10 us less.
//
// Measured (one GB300): the turned write 119 us, 6.5 TB/s, 0.97 of the copy rate;
// as codes 137 us, 4.9 TB/s; codes read back 36 us, 4.5 TB/s; 28 tokens 3.0 us.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "kv4.cuh"
#include "kv_pages.cuh"

namespace mpt {
namespace {

__device__ uint32_t g_append_counts[kKvCounts];

// The request of token t and its position there; false if no request has it.
// All lanes of the warp ask for the same token.
struct Place {
  int req;
  int64_t pos;
};
template <typename P>
__device__ __forceinline__ bool find_request(const P& p, int64_t t, int lane, Place& at) {
  // how many of q_offsets[1..batch] are at most t, 32 probes at a time
  int lo = 0, hi = p.batch;
  while (lo < hi) {
    const int step = (hi - lo + 31) / 32, j = lo + (lane + 1) * step;
    const int n = __popc(__ballot_sync(~0u, j <= hi && p.q_offsets[j] <= t));
    hi = min(hi, lo + (n + 1) * step - 1);
    lo += n * step;
  }
  if (lo >= p.batch) return false;
  const int64_t q0 = p.q_offsets[lo], q1 = p.q_offsets[lo + 1];
  if (t < q0 || t >= q1) return false;  // the latter only where offsets decrease
  at.req = lo;
  at.pos = (int64_t)p.kv_lens[lo] - (q1 - q0) + (t - q0);
  return true;
}
// The page of a position, -1 if the cache has none.
template <typename P>
__device__ __forceinline__ int find_page(const P& p, const Place& at) {
  if (at.pos < 0 || at.pos >> p.page_log2 >= p.width) return -1;
  const int id = p.table[(int64_t)at.req * p.table_stride + (at.pos >> p.page_log2)];
  return id < 0 || id >= p.n_pages ? -1 : id;
}

template <bool F16>
__device__ __forceinline__ void widen(const uint4& u, float* f) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (F16) {
      f[2 * i] = __half2float(__ushort_as_half((unsigned short)w[i]));
      f[2 * i + 1] = __half2float(__ushort_as_half((unsigned short)(w[i] >> 16)));
    } else {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
}
template <bool F16>
__device__ __forceinline__ uint4 narrow(const float* f) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (F16)
      asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(f[2 * i + 1]), "f"(f[2 * i]));
    else
      asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(f[2 * i + 1]), "f"(f[2 * i]));
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Cosines and sines of a lane's elements, and where their partners are.
struct Turn {
  alignas(16) float c[8];  // of an element's pair; adjacent: four of each
  alignas(16) float s[8];
  int partner;       // lane
  bool on;           // this lane's elements turn
};

// Products and sums are rounded one by one, not fused, so that codes of turned
// keys do not depend on how a formula is compiled.
template <bool F16>
__device__ __forceinline__ void turn(const Turn& u, bool adjacent, bool first, const uint4& x, float* f) {
  widen<F16>(x, f);
  if (adjacent) {
    if (!u.on) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float a = f[2 * i], b = f[2 * i + 1];
      f[2 * i] = __fsub_rn(__fmul_rn(a, u.c[i]), __fmul_rn(b, u.s[i]));
      f[2 * i + 1] = __fadd_rn(__fmul_rn(b, u.c[i]), __fmul_rn(a, u.s[i]));
    }
    return;
  }
  uint4 y;
  y.x = __shfl_sync(~0u, x.x, u.partner);
  y.y = __shfl_sync(~0u, x.y, u.partner);
  y.z = __shfl_sync(~0u, x.z, u.partner);
  y.w = __shfl_sync(~0u, x.w, u.partner);
  if (!u.on) return;
  float g[8];
  widen<F16>(y, g);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = __fmul_rn(f[i], u.c[i]), b = __fmul_rn(g[i], u.s[i]);
    f[i] = first ? __fsub_rn(a, b) : __fadd_rn(a, b);
  }
}

// x / y as a division rounds it, with inv = 1 / y rounded to nearest: one
// correction of the product gives the nearest quotient (Markstein, 1990), but
// where it is below the normal numbers, which no step or code depends on.
__device__ __forceinline__ float quotient(float x, float y, float inv) {
  const float q = __fmul_rn(x, inv);
  return __fmaf_rn(__fmaf_rn(-q, y, x), inv, q);
}

// Codes of a group of 32 elements, 8 a lane: the lane's two pieces, and in every
// lane the group's marks (step | offset << 8).  `has`: the lane has elements.
__device__ __forceinline__ uint32_t encode(float* f, bool has, int lane, uint32_t& marks) {
  float lo = f[0], hi = f[0], odd = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    lo = fminf(lo, f[i]);
    hi = fmaxf(hi, f[i]);
    odd = __fmaf_rn(f[i], 0.f, odd);  // NaN from then on, if f[i] is that or an infinity
  }
  if (__any_sync(~0u, odd != 0.f || lo < -kv4_most || hi > kv4_most)) {
    lo = INFINITY, hi = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      f[i] = fminf(fmaxf(f[i] == f[i] ? f[i] : 0.f, -kv4_most), kv4_most);
      lo = fminf(lo, f[i]);
      hi = fmaxf(hi, f[i]);
    }
  }
  if (!has) lo = INFINITY, hi = -INFINITY;
#pragma unroll
  for (int d = 1; d < 4; d <<= 1) {
    lo = fminf(lo, __shfl_xor_sync(~0u, lo, d));
    hi = fmaxf(hi, __shfl_xor_sync(~0u, hi, d));
  }
  const float own = __shfl_sync(~0u, f[0], lane & ~3);  // the group's first element
  float step = fmaxf(fmaxf(quotient(__fsub_rn(hi, lo), 15.f, 1.f / 15.f), quotient(fmaxf(hi, -lo), 120.f, 1.f / 120.f)), 0x1p-18f);
  step = __uint_as_float((__float_as_uint(step) + 0xFFFFFu) & ~0xFFFFFu);
  const float inv = __frcp_rn(step);
  // Added to 1.5 2^23, a quotient is rounded to a whole number that stands in the sum's last bits.
  auto whole = [&](float x) { return __float_as_int(__fadd_rn(quotient(x, step, inv), 0x1.8p23f)); };
  const int z = whole(lo);
  marks = ((__float_as_uint(step * 16.f) >> 20) - ((127 - 15) << 3)) | (uint32_t)(z - __float_as_int(0x1.8p23f) + 128) << 8;
  uint32_t piece[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i)  // never below z: x is at least lo, and rounding keeps that
    piece[i >> 2] += (uint32_t)min(whole(has ? f[i] : own) - z, 15) << 4 * (i & 3);
#pragma unroll
  for (int i = 0; i < 2; ++i) piece[i] = (piece[i] << 6 | piece[i] >> 10) & 0xFFFFu;
  return piece[0] | piece[1] << 16;
}

template <bool F16, bool kCodes>
__global__ void __launch_bounds__(128, kCodes ? 7 : 8) k_kv_append(const __grid_constant__ AppendParams p) {
  const int lane = threadIdx.x & 31;
  const int64_t warp = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  const int64_t t = warp / p.parts;
  const int part = (int)(warp - t * p.parts);
  if (t >= p.tokens) return;
  Place at;
  if (!find_request(p, t, lane, at)) return;
  const int lanes = 1 << p.lane_log2, sub = lane & (lanes - 1), which = lane >> p.lane_log2, heads = 32 >> p.lane_log2;
  const bool has = sub * 8 < p.dim;

  int64_t row = -1;
  if (p.turn) row = p.positions ? (int64_t)p.positions[t] : at.pos;
  const bool turns = row >= 0 && row < p.rows;
  int page = find_page(p, at);
  if (p.turn && !turns) page = -1;
  const int64_t slot = at.pos & ((1 << p.page_log2) - 1);
  if (KV_BAD(g_append_counts, page < 0 || (t < p.tokens && at.pos >= 0 && at.pos < (int64_t)p.width << p.page_log2 && page < p.n_pages &&
                                          (!turns || row < p.rows))))
    return;

  Turn u;
  u.on = turns && sub * 8 < p.rot;
  const int half = p.rot / 16;  // lanes of the first elements of the pairs
  const bool first = sub < half;
  u.partner = u.on && !p.adjacent ? (first ? lane + half : lane - half) : lane;
#pragma unroll
  for (int i = 0; i < 8; ++i) u.c[i] = 1.f, u.s[i] = 0.f;
  if (u.on) {
    const float* c = p.turn + row * p.turn_stride + (p.adjacent ? sub * 4 : (first ? sub : sub - half) * 8);
    const float* s = c + p.rot / 2;
    *(float4*)u.c = *(const float4*)c;
    *(float4*)u.s = *(const float4*)s;
    if (!p.adjacent) {
      *(float4*)(u.c + 4) = *(const float4*)(c + 4);
      *(float4*)(u.s + 4) = *(const float4*)(s + 4);
    }
  }

  // A step takes `heads` heads of the queries, the keys or the values; a token's
  // steps are dealt out to its parts in that order.  take(x, head, here) for the
  // lane's 8 elements of each; all lanes of the warp come to it together.  The
  // loads of at_once steps are in flight together.
  auto stream = [&](auto at_once, const char* base, int64_t tok, int64_t stride, int count, int before, auto take) {
    const uint4* from = (const uint4*)base + t * tok + which * stride + sub;
    const int n = (count + heads - 1) / heads;
    const int skip = before % p.parts;
    constexpr int kAtOnce = decltype(at_once)::value;
    for (int j = part >= skip ? part - skip : part - skip + p.parts; j < n; j += kAtOnce * p.parts) {
      uint4 x[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int k = j + i * p.parts;
        x[i] = make_uint4(0, 0, 0, 0);
        if (has && k * heads + which < count) x[i] = from[(int64_t)(k * heads) * stride];
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const int k = j + i * p.parts;
        if (k >= n) break;
        take(x[i], k * heads + which, k * heads + which < count);
      }
    }
    return n;
  };
  int before = 0;
  if (p.q) {
    uint4* const to = (uint4*)p.q_out + t * p.q_out_tok + sub;
    before = stream(std::integral_constant<int, 4>(), p.q, p.q_tok, p.q_head, p.q_heads, 0, [&](const uint4& x, int head, bool here) {
      float f[8];
      turn<F16>(u, p.adjacent, first, x, f);
      if (has && here) to[head * p.q_out_head] = u.on ? narrow<F16>(f) : x;
    });
  }
  if (page < 0) return;
  if constexpr (!kCodes) {
    uint4* const k = (uint4*)p.k + page * p.k_page + slot * p.k_slot + sub;
    uint4* const v = (uint4*)p.v + page * p.v_page + slot * p.v_slot + sub;
    before += stream(std::integral_constant<int, 4>(), p.k_new, p.k_new_tok, p.k_new_head, p.kv_heads, before, [&](const uint4& x, int head, bool here) {
      float f[8];
      turn<F16>(u, p.adjacent, first, x, f);
      if (has && here) k[head * p.k_head] = u.on ? narrow<F16>(f) : x;
    });
    stream(std::integral_constant<int, 4>(), p.v_new, p.v_new_tok, p.v_new_head, p.kv_heads, before, [&](const uint4& x, int head, bool here) {
      if (has && here) v[head * p.v_head] = x;
    });
  } else {
    const int n = kv4_groups(p.dim), tok = (int)slot & 7, g = sub >> 2;
    const bool writes = sub < 4 * n;
    char* const tile = p.pages + page * p.page_bytes + (slot >> 3) * kv4_tile(n);
    before += stream(std::integral_constant<int, 2>(), p.k_new, p.k_new_tok, p.k_new_head, p.kv_heads, before, [&](const uint4& x, int head, bool here) {
      float f[8];
      uint32_t marks;
      turn<F16>(u, p.adjacent, first, x, f);
      const uint32_t w = encode(f, has, lane, marks);
      if (!here || !writes) return;
      char* const to = tile + head * p.head_bytes;
      *(uint32_t*)(to + kv4_key(n, tok) + sub * 4) = w;
      if ((sub & 3) == 0) *(uint16_t*)(to + kv4_key_marks(n, tok) + g * 2) = (uint16_t)marks;
    });
    stream(std::integral_constant<int, 2>(), p.v_new, p.v_new_tok, p.v_new_head, p.kv_heads, before, [&](const uint4& x, int head, bool here) {
      float f[8];
      uint32_t marks;
      widen<F16>(x, f);
      const uint32_t w = encode(f, has, lane, marks);
      if (!here || !writes) return;
      char* const to = tile + head * p.head_bytes;
      uint16_t* const v = (uint16_t*)(to + kv4_value(n, tok >> 1)) + sub * 4 + (tok & 1);
      v[0] = (uint16_t)w;
      v[2] = (uint16_t)(w >> 16);
      if ((sub & 3) == 0) {
        uint8_t* const m = (uint8_t*)to + kv4_value_marks(n, tok >> 1) + g * 4 + (tok & 1);
        m[0] = (uint8_t)marks;
        m[2] = (uint8_t)(marks >> 8);
      }
    });
  }
}

// kType: of the output.  A warp a token (or a part of its heads), 8 elements a lane.
template <int kType>
__global__ void __launch_bounds__(128) k_kv4_read(const __grid_constant__ AppendParams p) {
  constexpr int kAtOnce = 4;  // steps whose loads are in flight together
  const int lane = threadIdx.x & 31;
  const int64_t warp = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  const int64_t t = warp / p.parts;
  const int part = (int)(warp - t * p.parts);
  if (t >= p.tokens) return;
  Place at;
  if (!find_request(p, t, lane, at)) return;
  const int lanes = 1 << p.lane_log2, sub = lane & (lanes - 1), which = lane >> p.lane_log2, heads = 32 >> p.lane_log2;
  const int page = find_page(p, at);
  const int64_t slot = at.pos & ((1 << p.page_log2) - 1);
  if (KV_BAD(g_append_counts, page < 0 || (t < p.tokens && at.pos >= 0 && at.pos < (int64_t)p.width << p.page_log2 && page < p.n_pages)))
    return;
  if (sub * 8 >= p.dim) return;
  const int nk = (p.kv_heads + heads - 1) / heads, n = kv4_groups(p.dim), tok = (int)slot & 7, g = sub >> 2;
  const char* const tile = p.pages + (int64_t)page * p.page_bytes + (slot >> 3) * kv4_tile(n);
  const uint32_t half = tok & 1 ? 0x7632 : 0x5410;
  for (int st = part; st < 2 * nk; st += kAtOnce * p.parts) {
    // A value's pieces stand beside those of the other token of its pair.
    uint2 w[kAtOnce];
    uint32_t m[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int k = st + i * p.parts, head = (k < nk ? k : k - nk) * heads + which;
      w[i] = make_uint2(0, 0);
      m[i] = 0;
      if (page < 0 || k >= 2 * nk || head >= p.kv_heads) continue;
      const char* from = tile + head * p.head_bytes;
      if (k < nk) {
        w[i].x = *(const uint32_t*)(from + kv4_key(n, tok) + sub * 4);
        m[i] = *(const uint16_t*)(from + kv4_key_marks(n, tok) + g * 2);
      } else {
        w[i] = *(const uint2*)(from + kv4_value(n, tok >> 1) + sub * 8);
        m[i] = *(const uint32_t*)(from + kv4_value_marks(n, tok >> 1) + g * 4);
      }
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int k = st + i * p.parts, head = (k < nk ? k : k - nk) * heads + which;
      if (k >= 2 * nk || head >= p.kv_heads) continue;
      const bool value = k >= nk;
      const uint32_t word = value ? __byte_perm(w[i].x, w[i].y, half) : w[i].x;
      const uint32_t marks = value ? m[i] >> 8 * (tok & 1) : m[i];  // the step's byte the lowest
      // c + z in f16, then times the step in 32 bits: exact whatever bytes are there
      const uint32_t offset = value ? marks >> 16 & 0xFFu : marks >> 8, z = hadd2((offset | offset << 16) | 0x64006400u, 0xE490E490u);
      const float step = __half2float(__ushort_as_half((unsigned short)(min(marks & 0xFFu, 222u) << 7))) * 0.0625f;
      const uint32_t at[4] = {word, word >> 4, __byte_perm(word, 0, 0x2301), word << 4};
      float f[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) {  // elements e and e + 4
        const uint32_t o = hadd2(kv4_code_bits(at[e]), z);
        f[e] = __half2float(__ushort_as_half((unsigned short)o)) * step;
        f[4 + e] = __half2float(__ushort_as_half((unsigned short)(o >> 16))) * step;
      }
      const int64_t out = value ? t * p.v_new_tok + head * p.v_new_head : t * p.k_new_tok + head * p.k_new_head;  // 8 elements each
      char* const to = (char*)(value ? p.v_new : p.k_new);
      if (kType == MPT_KV_F32) {
        float4* const o4 = (float4*)to + 2 * (out + sub);
        o4[0] = make_float4(f[0], f[1], f[2], f[3]);
        o4[1] = make_float4(f[4], f[5], f[6], f[7]);
      } else {
        ((uint4*)to)[out + sub] = narrow<kType == MPT_KV_F16>(f);
      }
    }
  }
}

// Lanes of a head, a power of two (four at least: a group of codes); parts of a
// token: one step each where tokens are few, else all steps in one.
void divide(AppendParams& p, int sms) {
  p.lane_log2 = 2;
  while (8 << p.lane_log2 < p.dim) ++p.lane_log2;
  const int heads = 32 >> p.lane_log2;
  const int64_t steps = (p.q ? (p.q_heads + heads - 1) / heads : 0) + 2 * ((p.kv_heads + heads - 1) / heads);
  const int64_t warps = 32ll * sms;  // in flight at once
  int64_t parts = (warps + p.tokens - 1) / p.tokens;
  if (parts > steps) parts = steps;
  p.parts = (int)(parts < 1 ? 1 : parts);
}

}  // namespace

cudaError_t launch_kv_append(AppendParams p, bool f16, bool codes, int sms, cudaStream_t stream) {
  divide(p, sms);
  const int64_t blocks = (p.tokens * p.parts + 3) / 4;
  if (blocks > INT32_MAX) return cudaErrorInvalidValue;
  const unsigned grid = (unsigned)blocks;
  if (codes) {
    if (f16) k_kv_append<true, true><<<grid, 128, 0, stream>>>(p);
    else k_kv_append<false, true><<<grid, 128, 0, stream>>>(p);
  } else {
    if (f16) k_kv_append<true, false><<<grid, 128, 0, stream>>>(p);
    else k_kv_append<false, false><<<grid, 128, 0, stream>>>(p);
  }
  return cudaGetLastError();
}

cudaError_t launch_kv4_read(AppendParams p, int type, int sms, cudaStream_t stream) {
  p.q = nullptr;
  divide(p, sms);
  const int64_t blocks = (p.tokens * p.parts + 3) / 4;
  if (blocks > INT32_MAX) return cudaErrorInvalidValue;
  const unsigned grid = (unsigned)blocks;
  if (type == MPT_KV_F32) k_kv4_read<MPT_KV_F32><<<grid, 128, 0, stream>>>(p);
  else if (type == MPT_KV_F16) k_kv4_read<MPT_KV_F16><<<grid, 128, 0, stream>>>(p);
  else k_kv4_read<MPT_KV_BF16><<<grid, 128, 0, stream>>>(p);
  return cudaGetLastError();
}

cudaError_t kv_append_counts(cudaStream_t stream, uint32_t* counts) {
  void* at = nullptr;
  const cudaError_t e = cudaGetSymbolAddress(&at, g_append_counts);
  return e != cudaSuccess ? e : cudaMemcpyAsync(counts, at, sizeof(g_append_counts), cudaMemcpyDeviceToHost, stream);
}

}  // namespace mpt
