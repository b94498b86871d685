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

__device__ __forceinline__ __half2 as_half2(uint32_t x) { return *reinterpret_cast<const __half2*>(&x); }
__device__ __forceinline__ uint32_t mul_half2(uint32_t x, __half2 y) {
  const __half2 z = __hmul2(as_half2(x), y);
  return *reinterpret_cast<const uint32_t*>(&z);
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
// Quotients x / t, t the exact product of two numbers, are x r + x r_lo, the first
// product and the sum rounded together: r is below 1 / t by some 2^-21 of it and
// r_lo what is missing, to 2^-43.  So a quotient that fp32 holds comes out exact, a
// border between two codes (or scales) with it, where bf16 elements often lie, for
// two operations instead of a division.  Both parts have t's sign: zeros keep
// theirs.
struct Q4Recip {
  float r, r_lo;
  __device__ __forceinline__ Q4Recip(float a, float b) {
    const float t = __fmul_rn(a, b), t_lo = fmaf(a, b, -t);
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(t));
    r *= 0x1.fffffp-1f;
    r_lo = fmaf(-r, t_lo, fmaf(-r, t, 1.f)) * r;
  }
  __device__ __forceinline__ float quotient(float x) const { return fmaf(x, r, x * r_lo); }
  __device__ __forceinline__ float nearest() const { return r + r_lo; }  // the quotient of 1
};

// A quotient that fp32 does not hold may round to a border, where ties to even would
// then choose for it.  Not where the factor has at most 13 bits: a border (3 bits; of
// scales, times six, 7) times t is an fp32 number then, and the quotient of the
// next x is further from the border than half a step by 2^-41 of it.  Otherwise:
//
// fp32 elements: a rounded quotient of no more bits than a border goes one step to
// the side that the exact remainder tells (q4_beside).
//
// bf16 elements, of 8 bits: x / (p factor), p the odd part of a border times its
// scale, is near 1 for all of a head's elements that lie near borders or for none,
// as two such x / p are 2^-15 or more apart; and never 1.  So a factor with an x / p
// within two steps of it is moved 2^-20 away from that: all these quotients come to
// their side, and no other passes a border.
//
// 28 layers of 10,720 bf16 rows of 4 heads 113 us without a factor and 118 with one
// of 24 bits (144 where every warp moves its factors itself, 216 with q4_beside), 14
// of fp32 rows 103 and 104 (115 with q4_beside for every element).
struct Q4Factor {
  float f;      // what quotients are formed with
  bool beside;  // they may have to go beside a border
};
__device__ __forceinline__ float q4_beside(float y, float x, float a, float b) {  // y: of x and a b
  const float t = __fmul_rn(a, b), left = fmaf(-y, fmaf(a, b, -t), fmaf(-y, t, x));
  const int bits = __float_as_int(y);
  if ((bits & 0x7ffff) != 0 || left == 0.f || fabsf(y) > 448.f) return y;  // no border above (y may be an infinity)
  return __int_as_float(bits + ((__float_as_int(left) ^ bits) < 0 ? -1 : 1));
}
__device__ __forceinline__ bool q4_long(float f) { return (__float_as_uint(f) & 0x7ffu) != 0u; }
// Whole warp; LANES of it, 8 or 32, have the same head.
template <typename T, int LANES>
__device__ __forceinline__ Q4Factor q4_factor(float f) {
  const bool is_long = q4_long(f);
  if (sizeof(T) == 4) return {f, is_long};
  if (__any_sync(0xffffffffu, is_long)) {
    const int lane = threadIdx.x & 31, odd = 2 * (lane & 7) + 1;
    bool up = false, down = false;
    auto look = [&](int p) {
      const float t = __fmul_rn((float)p, f), t_lo = fmaf((float)p, f, -t);
      const int over = (short)__float_as_uint(t);  // the steps by which t is above 8 bits
      up |= is_long && over >= -2 && (over < 0 || (over == 0 && t_lo < 0.f));
      down |= is_long && over <= 2 && (over > 0 || (over == 0 && t_lo > 0.f));
    };
    // odd parts: of codes' borders 1 to 7, of scales 1 to 15; of scales' borders, times six, 3 to 93
    if (LANES == 32) {
      look((lane >> 2 | 1) * odd);
    } else {
#pragma unroll
      for (int i = 1; i < 8; i += 2) look(i * odd);
    }
    look(3 * (odd + 16));
    const uint32_t mine = LANES == 32 ? 0xffffffffu : 0xffu << (lane & 24);
    up = __ballot_sync(0xffffffffu, up) & mine;
    down = __ballot_sync(0xffffffffu, down) & mine;
    f = fmaf(f, up ? -0x1p-20f : (down ? 0x1p-20f : 0.f), f);
  }
  return {f, false};
}

// The e4m3 number nearest to one within 2^-9 .. 448, and its value.
__device__ __forceinline__ uint32_t q4_scale_byte(float want) {
  unsigned short two;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(two) : "f"(0.f), "f"(want));
  return two;  // the upper half is zero
}
__device__ __forceinline__ float q4_scale_value(uint32_t byte) {
  return __low2float(as_half2(q4_scales(byte)));
}

// top: the bits of the group's largest magnitude as integers order them, which
// puts infinities and NaN above every number; by_six: of 6 factor.
struct Q4Scale {
  uint32_t byte;
  Q4Recip by;  // of scale * factor
  __device__ __forceinline__ Q4Scale(uint32_t top, const Q4Recip& by_six, const Q4Factor& factor)
      : by(init(top, by_six, factor), factor.f) {}

 private:
  __device__ __forceinline__ float init(uint32_t top, const Q4Recip& by_six, const Q4Factor& factor) {
    const float most = __uint_as_float(top);
    float want = by_six.quotient(most);
    if (factor.beside) want = q4_beside(want, most, 6.f, factor.f);
    const uint32_t nearest = q4_scale_byte(fminf(fmaxf(want, 0x1p-9f), 448.f));
    byte = top >= 0x7f800000u ? kQ4NaN : nearest;
    return q4_scale_value(nearest);
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
__device__ __forceinline__ uint32_t q4_word(const float (&x)[8], const Q4Scale& s, const Q4Factor& factor) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = s.by.quotient(x[i]);
  if (factor.beside) {
    uint32_t least = ~0u;  // 0: one has no more bits than a border
#pragma unroll
    for (int i = 0; i < 8; ++i) least = min(least, __float_as_uint(y[i]) << 11);
    if (least == 0u) {
      const float scale = q4_scale_value(s.byte);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = q4_beside(y[i], x[i], scale, factor.f);
    }
  }
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
