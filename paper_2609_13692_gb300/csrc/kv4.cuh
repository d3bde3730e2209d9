// The cache in 4 bits (include/mpt_kv.h): where a tile's parts lie, and the
// values of its codes.
#pragma once

#include "kv_internal.cuh"

namespace mpt {

constexpr int kCodeTokens = 8;  // of a tile
__host__ __device__ constexpr int kv4_groups(int dim) { return (dim + 31) / 32; }
// Bytes of a tile of n groups, and where in it a token's or a pair's part begins.
__host__ __device__ constexpr int kv4_tile(int n) { return 288 * n; }
__host__ __device__ constexpr int kv4_key(int n, int token) { return token * 16 * n; }
__host__ __device__ constexpr int kv4_key_marks(int n, int token) { return 128 * n + token * 2 * n; }
__host__ __device__ constexpr int kv4_value(int n, int pair) { return 144 * n + pair * 32 * n; }
__host__ __device__ constexpr int kv4_value_marks(int n, int pair) { return 272 * n + pair * 4 * n; }

constexpr float kv4_most = 3360.f;  // of a value: its step's byte is then 222 at most

// A word of two pieces as four pairs of f16: (c + z) s of the i-th element of
// the low piece and of the high one.  Rotated left by six bits, a piece has its
// first code at bits 6 to 9 of 16, where under the exponent of 16 it reads as
// 16 + c; the last comes there by a shift of four, the third by exchanging the
// bytes, the second by both.  (16 + c) s + (z - 16) s is then one fused
// operation on both halves, and every term is a whole number below 2^11 of
// step's last place: exact.
__device__ __forceinline__ uint32_t kv4_code_bits(uint32_t x) {
  uint32_t r;  // (x & mask) | exponent
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(x), "n"(0x03C003C0), "r"(0x4C004C00));
  return r;
}
__device__ __forceinline__ uint32_t hfma2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t r;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}
__device__ __forceinline__ uint32_t hmul2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t hadd2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t hmin2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("min.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ void kv4_word(uint32_t w, uint32_t step, uint32_t off, uint32_t* v) {
  const uint32_t x = __byte_perm(w, 0, 0x2301);
  v[0] = hfma2(kv4_code_bits(w), step, off);
  v[1] = hfma2(kv4_code_bits(x << 4), step, off);
  v[2] = hfma2(kv4_code_bits(x), step, off);
  v[3] = hfma2(kv4_code_bits(w << 4), step, off);
}
// s and (z - 16) s, two at a time, from the bytes of 16 s (at bits 0 and 16 of
// `steps`) and of z + 128 (likewise).  0x6400 | byte is 1024 + byte in f16.
__device__ __forceinline__ void kv4_marks(uint32_t steps, uint32_t offsets, uint32_t& step, uint32_t& off) {
  step = hmul2(hmin2(steps << 7, 0x6F006F00), 0x2C002C00);               // at most 7168, times 1/16
  off = hmul2(hadd2(offsets | 0x64006400, 0xE490E490), step);            // - 1168
}
// Of a key's group: both halves the same.  `marks`: its two bytes.
__device__ __forceinline__ void kv4_key_step(uint32_t marks, uint32_t& step, uint32_t& off) {
  kv4_marks(__byte_perm(marks, 0, 0x4040), __byte_perm(marks, 0, 0x4141), step, off);
}
// Of two keys' groups at once.
__device__ __forceinline__ uint32_t kv4_low(uint32_t x) {
  uint32_t r;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tmov.b32 %0, {l, l};\n\t}" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ uint32_t kv4_high(uint32_t x) {
  uint32_t r;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tmov.b32 %0, {h, h};\n\t}" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ void kv4_key_steps(uint32_t marks_a, uint32_t marks_b, uint32_t& step_a, uint32_t& off_a, uint32_t& step_b,
                                              uint32_t& off_b) {
  uint32_t step, off;
  // (of 16 bits each: bytes 2 and 3 are 0)
  kv4_marks(__byte_perm(marks_a, marks_b, 0x2420), __byte_perm(marks_a, marks_b, 0x2521), step, off);
  step_a = kv4_low(step), off_a = kv4_low(off), step_b = kv4_high(step), off_b = kv4_high(off);
}
// Of a pair of values' group, low half the even token.  `marks`: its four bytes.
__device__ __forceinline__ void kv4_value_step(uint32_t marks, uint32_t& step, uint32_t& off) {
  kv4_marks(__byte_perm(marks, 0, 0x4140), __byte_perm(marks, 0, 0x4342), step, off);
}

// The scale of a row's scores once its power of two is back in it, between the
// smallest and the largest normal number: 0 times a masked score, or infinity
// times one of 0, would be NaN.
__device__ __forceinline__ float kv4_scale(float scale, float back) {
  return fminf(fmaxf(scale * back, 1.17549435e-38f), 3.40282347e38f);
}

}  // namespace mpt
