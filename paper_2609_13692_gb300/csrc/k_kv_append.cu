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
// 4.5 bits an element; the arithmetic of the codes (a quotient, its rounding and
// the packing: about 15 operations an element) hides behind it.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

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

// Codes of a group of 32 elements, 8 a lane: the lane's two pieces, and in every
// lane the group's marks (step | offset << 8).  `has`: the lane has elements.
__device__ __forceinline__ uint32_t encode(float* f, bool has, int lane, uint32_t& marks) {
  float lo = INFINITY, hi = -INFINITY;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = f[i] == f[i] ? f[i] : 0.f;
    f[i] = fminf(fmaxf(x, -kv4_most), kv4_most);
    lo = fminf(lo, f[i]);
    hi = fmaxf(hi, f[i]);
  }
  if (!has) lo = INFINITY, hi = -INFINITY;
#pragma unroll
  for (int d = 1; d < 4; d <<= 1) {
    lo = fminf(lo, __shfl_xor_sync(~0u, lo, d));
    hi = fmaxf(hi, __shfl_xor_sync(~0u, hi, d));
  }
  const float own = __shfl_sync(~0u, f[0], lane & ~3);  // the group's first element
  float step = fmaxf(fmaxf(__fdiv_rn(__fsub_rn(hi, lo), 15.f), __fdiv_rn(fmaxf(hi, -lo), 120.f)), 0x1p-18f);
  step = __uint_as_float((__float_as_uint(step) + 0xFFFFFu) & ~0xFFFFFu);
  const float inv = __frcp_rn(step), z = rintf(__fdiv_rn(lo, step));
  marks = ((__float_as_uint(step * 16.f) >> 20) - ((127 - 15) << 3)) | (uint32_t)((int)z + 128) << 8;
  uint32_t piece[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = has ? f[i] : own;
    // x / step rounded as a division is: with the inverse rounded to nearest,
    // one correction of the product gives the nearest quotient (Markstein)
    const float q = __fmul_rn(x, inv);
    const float c = fminf(fmaxf(__fsub_rn(rintf(__fmaf_rn(__fmaf_rn(-q, step, x), inv, q)), z), 0.f), 15.f);
    piece[i >> 2] |= (uint32_t)(int)c << 4 * (i & 3);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) piece[i] = (piece[i] << 6 | piece[i] >> 10) & 0xFFFFu;
  return piece[0] | piece[1] << 16;
}

constexpr int kAtOnce = 4;  // steps whose loads are in flight together

template <bool F16, bool kCodes>
__global__ void __launch_bounds__(128) k_kv_append(const __grid_constant__ AppendParams p) {
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

  // steps: of the queries, then of the keys, then of the values
  const int nq = p.q ? (p.q_heads + heads - 1) / heads : 0, nk = (p.kv_heads + heads - 1) / heads;
  const int steps = page >= 0 ? nq + 2 * nk : nq;
  const int n = kv4_groups(p.dim);
  for (int base = part; base < steps; base += p.parts * kAtOnce) {
    uint4 x[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int st = base + i * p.parts;
      x[i] = make_uint4(0, 0, 0, 0);
      if (st >= steps) continue;
      const int kind = st < nq ? 0 : st < nq + nk ? 1 : 2, head = (st - (kind == 0 ? 0 : kind == 1 ? nq : nq + nk)) * heads + which;
      const uint4* from = kind == 0   ? (const uint4*)p.q + t * p.q_tok + head * p.q_head
                          : kind == 1 ? (const uint4*)p.k_new + t * p.k_new_tok + head * p.k_new_head
                                      : (const uint4*)p.v_new + t * p.v_new_tok + head * p.v_new_head;
      if (has && head < (kind == 0 ? p.q_heads : p.kv_heads)) x[i] = from[sub];
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int st = base + i * p.parts;
      if (st >= steps) break;  // the warp's lanes agree
      const int kind = st < nq ? 0 : st < nq + nk ? 1 : 2, head = (st - (kind == 0 ? 0 : kind == 1 ? nq : nq + nk)) * heads + which;
      const bool here = head < (kind == 0 ? p.q_heads : p.kv_heads);
      float f[8];
      if (kind == 2) {
        if (!kCodes) {
          if (has && here) ((uint4*)p.v + page * p.v_page + slot * p.v_slot + head * p.v_head)[sub] = x[i];
          continue;
        }
        widen<F16>(x[i], f);
      } else {
        turn<F16>(u, p.adjacent, first, x[i], f);
        if (kind == 0) {
          if (has && here) ((uint4*)p.q_out + t * p.q_out_tok + head * p.q_out_head)[sub] = u.on ? narrow<F16>(f) : x[i];
          continue;
        }
        if (!kCodes) {
          if (has && here) ((uint4*)p.k + page * p.k_page + slot * p.k_slot + head * p.k_head)[sub] = u.on ? narrow<F16>(f) : x[i];
          continue;
        }
      }
      if constexpr (kCodes) {
        uint32_t marks;
        const uint32_t w = encode(f, has, lane, marks);
        if (!here || sub >= 4 * n) continue;
        char* tile = p.pages + page * p.page_bytes + head * p.head_bytes + (slot >> 3) * kv4_tile(n);
        const int tok = slot & 7, g = sub >> 2;
        if (kind == 1) {
          *(uint32_t*)(tile + kv4_key(n, tok) + sub * 4) = w;
          if ((sub & 3) == 0) *(uint16_t*)(tile + kv4_key_marks(n, tok) + g * 2) = (uint16_t)marks;
        } else {
          uint16_t* to = (uint16_t*)(tile + kv4_value(n, tok >> 1)) + sub * 4 + (tok & 1);
          to[0] = (uint16_t)w;
          to[2] = (uint16_t)(w >> 16);
          if ((sub & 3) == 0) {
            uint8_t* m = (uint8_t*)tile + kv4_value_marks(n, tok >> 1) + g * 4 + (tok & 1);
            m[0] = (uint8_t)marks;
            m[2] = (uint8_t)(marks >> 8);
          }
        }
      }
    }
  }
}

// (c + z) s of a piece's four elements.
__device__ __forceinline__ void decode(uint32_t piece, uint32_t step_byte, uint32_t offset_byte, float* f) {
  const float s = __half2float(__ushort_as_half((unsigned short)(min(step_byte, 222u) << 7))) * 0.0625f;
  const float z = (float)((int)offset_byte - 128);
  const uint32_t c = (piece >> 6 | piece << 10) & 0xFFFFu;
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = ((float)(c >> 4 * i & 15u) + z) * s;
}

// kType: of the output.  A warp a token (or a part of its heads), 8 elements a lane.
template <int kType>
__global__ void __launch_bounds__(128) k_kv4_read(const __grid_constant__ AppendParams p) {
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
  const int nk = (p.kv_heads + heads - 1) / heads, n = kv4_groups(p.dim), tok = (int)slot & 7, g = sub >> 2;
  if (sub * 8 >= p.dim) return;
#pragma unroll 4
  for (int st = part; st < 2 * nk; st += p.parts) {
    const bool value = st >= nk;
    const int head = (st - (value ? nk : 0)) * heads + which;
    if (head >= p.kv_heads) continue;
    float f[8];
    if (page >= 0) {
      const char* tile = p.pages + page * p.page_bytes + head * p.head_bytes + (slot >> 3) * kv4_tile(n);
      uint32_t a, b, s, z;
      if (!value) {
        const uint32_t w = *(const uint32_t*)(tile + kv4_key(n, tok) + sub * 4);
        const uint32_t m = *(const uint16_t*)(tile + kv4_key_marks(n, tok) + g * 2);
        a = w & 0xFFFFu, b = w >> 16, s = m & 0xFFu, z = m >> 8;
      } else {
        const uint16_t* w = (const uint16_t*)(tile + kv4_value(n, tok >> 1)) + sub * 4 + (tok & 1);
        const uint8_t* m = (const uint8_t*)tile + kv4_value_marks(n, tok >> 1) + g * 4 + (tok & 1);
        a = w[0], b = w[2], s = m[0], z = m[2];
      }
      decode(a, s, z, f);
      decode(b, s, z, f + 4);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = 0.f;
    }
    const int64_t out = value ? t * p.v_new_tok + head * p.v_new_head : t * p.k_new_tok + head * p.k_new_head;  // 8 elements each
    char* to = (char*)(value ? p.v_new : p.k_new);
    if (kType == MPT_KV_F32) {
      float4* o = (float4*)to + 2 * (out + sub);
      o[0] = make_float4(f[0], f[1], f[2], f[3]);
      o[1] = make_float4(f[4], f[5], f[6], f[7]);
    } else {
      ((uint4*)to)[out + sub] = narrow<kType == MPT_KV_F16>(f);
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
