// Rows of 128 elements in 4 bits: 64 bytes of codes (e2m1, element 2 i in the
// low half of byte i) and 8 scales (e4m3), one to 16 elements; an element is
// code * scale * factor, the factor its KV head's.
//
// A code has two significant bits and a scale four, so that code * scale has at
// most six and lies within 2^-10 .. 2688: exact in fp16 (and in bf16).  What is
// decoded below is that product; the factor goes to the scores or the result.
#pragma once

#include "kernels.cuh"

namespace stl {

constexpr int kQ4Row = kD / 2;         // bytes of a row's codes
constexpr int kQ4Group = 16;           // elements of a scale
constexpr int kQ4Scales = kD / kQ4Group;
constexpr uint32_t kQ4NaN = 0x7f;      // the scale of a group that holds an infinity or a NaN

__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
// The two e4m3 scales of the low 16 bits, as fp16.
__device__ __forceinline__ uint32_t q4_scales(uint32_t two) {
  uint32_t d;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(d) : "h"((unsigned short)two));
  return d;
}
// The eight codes of a word as four pairs of fp16, each byte a pair.
__device__ __forceinline__ void q4_codes(uint32_t word, uint32_t (&h)[4]) {
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "mov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
      : "r"(word));
}

// How a group is put into 4 bits: its scale is the largest magnitude over six
// times the factor, rounded to e4m3, at least the smallest (a group of zeros
// divides by something) and at most the largest.
//
// Quotients x / t are x r + x r_lo, the first product and the sum rounded
// together: r is below 1 / t by some 2^-23 of it and r_lo what is missing, to
// 2^-45.  So a quotient that fp32 holds comes out exact, a border between two
// codes (or scales) with it, where bf16 elements often lie, for two operations
// instead of a division.  Both parts have t's sign: zeros keep theirs.
struct Q4Recip {
  float r, r_lo;
  __device__ __forceinline__ explicit Q4Recip(float t) {
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(t));
    r *= 0x1.fffffcp-1f;
    r_lo = fmaf(-r, t, 1.f) * r;
  }
  __device__ __forceinline__ float quotient(float x) const { return fmaf(x, r, x * r_lo); }
  __device__ __forceinline__ float nearest() const { return r + r_lo; }  // 1 / t in fp32
};

// The e4m3 number nearest to one within 2^-9 .. 448, and its value.
__device__ __forceinline__ uint32_t q4_scale_byte(float want) {
  unsigned short two;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(two) : "f"(0.f), "f"(want));
  return two;  // the upper half is zero
}
__device__ __forceinline__ float q4_scale_value(uint32_t byte) {
  const uint32_t half = q4_scales(byte);
  return __low2float(*reinterpret_cast<const __half2*>(&half));
}

// top: the bits of the group's largest magnitude as integers order them, which
// puts infinities and NaN above every number; by_six: of 6 factor.
struct Q4Scale {
  uint32_t byte;
  Q4Recip by;  // of scale * factor
  __device__ __forceinline__ Q4Scale(uint32_t top, const Q4Recip& by_six, float factor)
      : by(init(top, by_six, factor)) {}

 private:
  __device__ __forceinline__ float init(uint32_t top, const Q4Recip& by_six, float factor) {
    const uint32_t nearest = q4_scale_byte(fminf(fmaxf(by_six.quotient(__uint_as_float(top)), 0x1p-9f), 448.f));
    byte = top >= 0x7f800000u ? kQ4NaN : nearest;
    return q4_scale_value(nearest) * factor;
  }
};
// The codes of eight quotients, and of eight elements.
__device__ __forceinline__ uint32_t q4_codes_of(const float (&x)[8]) {
  uint32_t w;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(w)
      : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]));
  return w;
}
__device__ __forceinline__ uint32_t q4_word(const float (&x)[8], const Q4Scale& s) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = s.by.quotient(x[i]);
  return s.byte == kQ4NaN ? 0u : q4_codes_of(y);
}
__device__ __forceinline__ uint32_t q4_top(const float (&x)[8]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  return top;
}

// Row r of head h in page `page` of pools [n_pages][hkv][page_rows].
__device__ __forceinline__ size_t q4_row(const PageView& pg, int page, int r, int h, int hkv) {
  return ((size_t)page * hkv + h) * pg.page_rows + r;
}

}  // namespace stl
