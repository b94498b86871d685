// New tokens' heads normed and rotated, queries packed, keys and values into 4-bit pages.
#include "kernels.cuh"
#include "paged.cuh"
#include "q4.cuh"
#include "rotate.cuh"

namespace stl {

// k_rotate with keys and values going to 4-bit pages, unrounded before that: codes
// and scales are those of the rotation in 64 bits, not of its fp32 form.  An
// element at a border between two codes (or a group's scale between two) would go
// where the fp32 rotation's error puts it; one in some 20,000 lies so near a border
// that this could be the wrong side.  Both ends of what it may be are put into 4
// bits, and where they differ, settle_keys decides.
//
// A unit is a warp's: a segment of a token's query heads, as k_rotate's, or four of
// its key and value heads, whose lanes share a group of 16 elements by twos (one
// lane has it where pairs are interleaved).  Instructions bound long prompts of
// bf16: 8,616 tokens of 28 + 4 heads take 31 us, 0.70 of a plain copy's rate, where
// the append in 16 bits, with the same rotation, has 0.89.  They execute 22 million
// warp instructions, 62 % of the cycles that could issue one, with the integer pipe
// (conversions, comparisons of codes, masks) busy for 57 % and 44 % of the warps
// resident; a norm adds 4 us, the keys' second end and what it decides 3.  fp32 has
// twice the bytes for them: 46 us, 0.92.  Latency bounds the rest (2,096 tokens of
// 12 + 2 heads 6.7 us, one 2.3).  Keys are most of a warp's work, so that warps of
// four tokens' keys share a CTA and those of the first kAhead tokens come before
// anything else.
//
// A lane's elements of a key: as they are in memory, the norm's weights, rotated in fp32 and how far (each pair, and
// all pairs of the groups) they may be off by that; codes, the scales of their groups, and which codes (nibbles that
// are not 0) and scales are open.
struct KeyPart {
  float x[2][8], w[2][8], y[2][8], off[8], most;
  uint32_t code[2], scale[2], open[2];
  bool open_scale[2];
};
// Element j of part e belongs to this of the lane's eight pairs.
template <bool IL>
__device__ __forceinline__ int pair_of(int e, int j) { return IL ? 4 * e + (j >> 1) : j; }

// The codes of eight elements; *open: the nibbles that would be others (but for the
// sign of a 0) for elements within off[..] of theirs, or, where off may be more
// than an eighth of a code's step, all.  (Up to there the two ends of what an
// element may be have one sign, or are both nearest to 0.)
template <bool IL>
__device__ __forceinline__ uint32_t codes_within(const float (&x)[8], int e, const float (&off)[8], float most,
                                                 const Q4Recip& by, uint32_t* open) {
  const float r = by.nearest();
  float lo[8], hi[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float o = off[pair_of<IL>(e, j)];
    lo[j] = (x[j] - o) * r;
    hi[j] = (x[j] + o) * r;
  }
  const uint32_t code = q4_codes_of(hi);
  *open = most * r > 0.0625f ? 0x77777777u : (code ^ q4_codes_of(lo)) & 0x77777777u;
  return code;
}

// Whether the scale of a group whose largest magnitude may be off by so much is; *byte: then the largest it may be.
__device__ __forceinline__ bool open_scale(uint32_t top, float off, const Q4Recip& by_six, uint32_t* byte) {
  auto of = [&](float x) { return q4_scale_byte(fminf(fmaxf(by_six.quotient(x), 0x1p-9f), 448.f)); };
  const float most = __uint_as_float(top);
  const uint32_t high = of(most + off);
  if (top >= 0x7f800000u || of(fmaxf(most - off, 0.f)) == high) return false;
  *byte = high;
  return true;
}

// What is open is formed in pairs of fp32, some 45 bits: in fp64, whose operations
// are few a clock on this chip, the same took 2.9 us longer.
struct TwoFloats {
  float h, l;  // h + l, l no more than half a step of h
};
__device__ __forceinline__ TwoFloats joined(float h, float l) {  // |h| >= |l|
  const float s = h + l;
  return {s, l - (s - h)};
}
__device__ __forceinline__ TwoFloats sum_of(float a, float b) {
  const float s = a + b, t = s - a;
  return {s, (a - (s - t)) + (b - t)};
}
__device__ __forceinline__ TwoFloats product_of(float a, float b) {
  const float p = __fmul_rn(a, b);
  return {p, fmaf(a, b, -p)};
}
__device__ __forceinline__ TwoFloats operator+(TwoFloats a, TwoFloats b) {
  const TwoFloats s = sum_of(a.h, b.h);
  return joined(s.h, s.l + (a.l + b.l));
}
__device__ __forceinline__ TwoFloats operator*(TwoFloats a, TwoFloats b) {
  const TwoFloats p = product_of(a.h, b.h);
  return joined(p.h, fmaf(a.h, b.l, fmaf(a.l, b.h, p.l)));
}
__device__ __forceinline__ TwoFloats operator-(TwoFloats a) { return {-a.h, -a.l}; }
// A rotated element: what it is at the nearest 64th of a turn, and the rest.  (Of
// keys at the first positions the first part is the key itself, and a rest below
// every bit of it still tells the side of a border.)
struct Turned {
  TwoFloats near, rest;
  __device__ __forceinline__ float sign_of_less(TwoFloats b) const { return (near + -b + rest).h; }  // of this - b
};
__device__ __forceinline__ Turned magnitude(Turned a) {
  return a.sign_of_less({0.f, 0.f}) < 0.f ? Turned{-a.near, -a.rest} : a;
}
__device__ __forceinline__ bool below(Turned a, Turned b) { return (a.near + -b.near + (a.rest + -b.rest)).h < 0.f; }
// Whether the code (scale) behind a border is not that of a magnitude; on it, the even one is.
__device__ __forceinline__ bool misses(Turned a, TwoFloats border, uint32_t code) {
  const float d = a.sign_of_less(border);
  return d < 0.f || (d == 0.f && (code & 1));
}

// Sine and cosine of a * 2^-64 turns: those of the nearest 64th of a turn and,
// times those, of what is left, x of at most 0.05, by Taylor series; cosine less 1.
// The terms behind x and x^2 / 2 are below 2^-15, so that fp32 has them to 2^-38.
// (A table in constant memory would cost every launch of this file's kernels 0.4 us.)
__device__ const float2 kSin64[17] = {  // of 0 .. 16 64ths, as pairs
    {0.0f, 0.0f}, {0.0980171412f, -8.93393193e-10f}, {0.195090324f, -1.67047143e-09f},
    {0.290284663f, 1.38156651e-08f}, {0.382683426f, 6.22335072e-09f}, {0.471396744f, -7.42525375e-09f},
    {0.555570245f, -1.17695214e-08f}, {0.634393275f, 9.37955758e-09f}, {0.707106769f, 1.21016175e-08f},
    {0.773010433f, 2.06425526e-08f}, {0.831469595f, 1.68702634e-08f}, {0.881921291f, -2.70029634e-08f},
    {0.923879504f, 2.83074897e-08f}, {0.956940353f, -1.7184508e-08f}, {0.980785251f, 2.97394731e-08f},
    {0.99518472f, 7.10966619e-09f}, {1.0f, 0.0f}};
__device__ __forceinline__ void turn_sincos(uint64_t a, TwoFloats (&sn)[2], TwoFloats (&cs)[2]) {
  const uint32_t k = (uint32_t)((a + (1ull << 57)) >> 58);
  const long long left = (long long)(a - ((uint64_t)k << 58));
  const float h = (float)left;
  const TwoFloats two_pi = {3.40612167e-19f, -9.47839643e-27f};  // times 2^-64
  const TwoFloats x = TwoFloats{h, (float)(left - (long long)h)} * two_pi;
  const TwoFloats x2 = product_of(x.h, x.h);
  const TwoFloats s = {x.h, fmaf(x.h * x2.h, fmaf(x2.h, fmaf(x2.h, -1.f / 5040, 1.f / 120), -1.f / 6), x.l)};
  const TwoFloats c = {-0.5f * x2.h,
                       fmaf(x2.h * x2.h, fmaf(x2.h, -1.f / 720, 1.f / 24), -fmaf(x.h, x.l, 0.5f * x2.l))};
  const float2 s0 = kSin64[k & 15], c0 = kSin64[16 - (k & 15)];
  sn[0] = k & 16 ? TwoFloats{c0.x, c0.y} : TwoFloats{s0.x, s0.y};
  cs[0] = k & 16 ? TwoFloats{-s0.x, -s0.y} : TwoFloats{c0.x, c0.y};
  if (k & 32) {
    sn[0] = -sn[0];
    cs[0] = -cs[0];
  }
  sn[1] = cs[0] * s + sn[0] * c;
  cs[1] = cs[0] * c + -(sn[0] * s);
}

// Settles what is open of a warp's keys, eight lanes to a head; every lane takes
// the first of its open elements, then the next.  Scales start at the largest they
// could be, codes at the last, and go down until the border below is not above.
template <bool IL>
__device__ __noinline__ void settle_keys(KeyPart* part, bool has_norm, float eps, const int32_t* pos, int n, int t,
                                         int end0, int end1, const uint64_t* turn, float factor) {
  const int c = threadIdx.x & 7;
  TwoFloats r = {1.f, 0.f};
  if (has_norm) {
    TwoFloats ss = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float x = part->x[i >> 3][i & 7];
      const TwoFloats sq = product_of(x, x), s = sum_of(ss.h, sq.h);
      ss = {s.h, ss.l + (s.l + sq.l)};
    }
    ss = joined(ss.h, ss.l);
    for (int o = 1; o < 8; o <<= 1)
      ss = ss + TwoFloats{__shfl_xor_sync(0xffffffffu, ss.h, o), __shfl_xor_sync(0xffffffffu, ss.l, o)};
    const TwoFloats mean = TwoFloats{ss.h * (1.f / kD), ss.l * (1.f / kD)} + TwoFloats{eps, 0.f};
    const float r0 = rsqrtf(mean.h);  // and a step of Newton's iteration
    const TwoFloats one = mean * TwoFloats{r0, 0.f} * TwoFloats{r0, 0.f};
    r = joined(r0, 0.5f * r0 * ((1.f - one.h) - one.l));
  }
  auto exact = [&](int e, int j) {
    const int i = pair_of<IL>(e, j), pair = 8 * c + i, axis = pair < end0 ? 0 : (pair < end1 ? 1 : 2);
    const bool second = IL ? j & 1 : e;
    const int e0 = IL ? e : 0, j0 = IL ? j & ~1 : j, e1 = IL ? e : 1, j1 = IL ? j | 1 : j;
    TwoFloats p = {part->x[e0][j0], 0.f}, q = {part->x[e1][j1], 0.f}, sn[2], cs[2];
    if (has_norm) {
      p = r * p * TwoFloats{part->w[e0][j0], 0.f};
      q = r * q * TwoFloats{part->w[e1][j1], 0.f};
    }
    turn_sincos((uint64_t)(int64_t)pos[(size_t)axis * n + t] * turn[pair], sn, cs);
    if (second) return Turned{q * cs[0] + p * sn[0], q * cs[1] + p * sn[1]};
    return Turned{p * cs[0] + -(q * sn[0]), p * cs[1] + -(q * sn[1])};
  };
  if (__any_sync(0xffffffffu, part->open_scale[0] || part->open_scale[1])) {
    // the largest magnitudes, of the elements that are within their errors of the largest
    float near[2];
    for (int e = 0; e < 2; ++e) {
      near[e] = 0.f;
      for (int j = 0; j < 8; ++j) near[e] = fmaxf(near[e], fabsf(part->y[e][j]) - part->off[pair_of<IL>(e, j)]);
    }
    if (IL)
      near[0] = near[1] = fmaxf(near[0], near[1]);
    else
      for (int e = 0; e < 2; ++e) near[e] = fmaxf(near[e], __shfl_xor_sync(0xffffffffu, near[e], 1));
    uint32_t left = 0;
    for (int i = 0; i < 16; ++i) {
      const int e = i >> 3, j = i & 7;
      if (part->open_scale[e] && fabsf(part->y[e][j]) + part->off[pair_of<IL>(e, j)] >= near[e]) left |= 1u << i;
    }
    Turned top[2] = {};
    while (__any_sync(0xffffffffu, left != 0u)) {
      if (left) {
        const int i = __ffs(left) - 1;
        left &= left - 1u;
        const Turned y = magnitude(exact(i >> 3, i & 7));
        if (below(top[i >> 3], y)) top[i >> 3] = y;
      }
      __syncwarp();
    }
    for (int e = 0; e < 2; ++e) {
      auto swap = [](TwoFloats a) {
        return TwoFloats{__shfl_xor_sync(0xffffffffu, a.h, 1), __shfl_xor_sync(0xffffffffu, a.l, 1)};
      };
      const Turned other = IL ? top[1 - e] : Turned{swap(top[e].near), swap(top[e].rest)};
      if (below(top[e], other)) top[e] = other;
    }
    for (int e = 0; e < 2; ++e) {
      if (!part->open_scale[e]) continue;
      uint32_t at = part->scale[e];
      for (; at > 1; --at) {  // the border to the scale before, six times and by the factor
        const TwoFloats border = product_of(3.f * (q4_scale_value(at - 1) + q4_scale_value(at)), factor);
        if (!misses(top[e], border, at)) break;
      }
      part->scale[e] = at;
      const Q4Recip by(q4_scale_value(at), factor);
      part->code[e] = codes_within<IL>(part->y[e], e, part->off, part->most, by, &part->open[e]);
    }
  }
  uint32_t left = 0;
  for (int i = 0; i < 16; ++i)
    if (part->open[i >> 3] >> (4 * (i & 7)) & 15u) left |= 1u << i;
  while (__any_sync(0xffffffffu, left != 0u)) {
    if (left) {
      const int i = __ffs(left) - 1, e = i >> 3, shift = 4 * (i & 7);
      left &= left - 1u;
      const Turned y = exact(e, i & 7), size = magnitude(y);
      const float scale = q4_scale_value(part->scale[e]);
      uint32_t code = 7;
      for (; code > 0; --code) {
        const float middle = code < 5 ? 0.5f * code - 0.25f : (code < 7 ? code - 2.5f : 5.f);
        if (!misses(size, product_of(middle * scale, factor), code)) break;
      }
      const uint32_t sign = y.sign_of_less({0.f, 0.f}) < 0.f ? 8u : 0u;
      part->code[e] = (part->code[e] & ~(15u << shift)) | (code | sign) << shift;
    }
    __syncwarp();
  }
}

// A token's units in order: the keys and values of the first kAhead tokens; then by
// fours of tokens keys and values kAhead tokens ahead, and queries; the last queries.
// Measured at 2,096 tokens of 12 + 2 heads with norms and 8,616 of 28 + 4, in bf16, and
// the latter in fp32: kAhead 0: 8.4, 32.2 and 45.5 us; 1,216: 7.0, 30.7, 44.9; 2,432: 6.7,
// 31.1, 46.0; all: 6.7, 33.1, 49.6.  (Each token's units together: 2 us more than with 2,432.)
constexpr int kAhead = 2432;
// Divides numbers below 2^31 by d: the product with 2^shift / d, rounded up, is off by
// less than a quotient's step (Granlund and Montgomery, 1994).  Three instructions for
// some thirty, of a warp's 500: 0.8 us of 8,616 tokens'.
struct Divisor {
  uint32_t mul;
  int shift, d;
  explicit Divisor(int by) : shift(31), d(by) {
    while ((1LL << (shift - 31)) < d) ++shift;
    mul = (uint32_t)(((1ULL << shift) + d - 1) / d);
  }
  __device__ __forceinline__ int of(int x) const { return (int)((uint64_t)(uint32_t)x * mul >> shift); }
};
struct Order {
  int q_segs, first, rest;  // first: units of the keys and values that come first; rest: other tokens, in fours
  Divisor ahead, four, q;   // four: units of four tokens
  Order(int n, int q_segs, int segs)
      : q_segs(q_segs), ahead(n < kAhead ? n : kAhead), four(4 * segs), q(q_segs) {
    first = (segs - q_segs) * ahead.d;
    rest = (n - ahead.d + 3) / 4 * 4;
  }
};
struct Unit {
  int t, seg;
};
__device__ __forceinline__ Unit unit_of(int u, const Order& o) {
  if (u < o.first) {
    const int seg = o.ahead.of(u);
    return {u - seg * o.ahead.d, o.q_segs + seg};
  }
  u -= o.first;
  const int fours = o.four.of(u);
  if (4 * fours < o.rest) {
    const int i = u - fours * o.four.d, seg = (o.four.d >> 2) - 1 - (i >> 2);
    return {4 * fours + (i & 3) + (seg < o.q_segs ? 0 : o.ahead.d), seg};
  }
  u -= (o.rest >> 2) * o.four.d;
  const int t = o.q.of(u);
  return {o.rest + t, u - t * o.q.d};
}

// Registers for eight CTAs an SM, seven of fp32 (few are spilled): 8,616 tokens of bf16 take 31.3 / 31.1 / 30.2 us
// with seven / eight / nine, one 2.3 / 2.3 / 2.5, 64 3.9 / 3.9 / 4.0; 8,616 of fp32 with norms 49.7 / 49.1 / 53.2 with
// six / seven / eight.
template <typename T, int NB, bool IL>
__global__ void __launch_bounds__(kRotThreads, sizeof(T) == 2 ? 8 : 7)
    k_append_q4(const __grid_constant__ TokenView x, const __grid_constant__ RopeView rope,
                const __grid_constant__ PageView pg, const __grid_constant__ Q4View q4, T* q_out, int base, int extra,
                const __grid_constant__ Order order) {
  __shared__ uint64_t turn[kD / 2];
  __shared__ float4 cs[kRotWarps][2][8], sn[kRotWarps][2][8];  // as in k_rotate
  if (threadIdx.x < kD / 2) turn[threadIdx.x] = rope.turn[threadIdx.x];
  __syncthreads();
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane >> 3, c = lane & 7;
  const Unit unit = unit_of(blockIdx.x * kRotWarps + warp, order);
  const int t = unit.t, seg = unit.seg, q_segs = order.q_segs;
  if (t >= x.n) return;
  const int off0 = IL ? 16 * c : 8 * c, off1 = IL ? 16 * c + 8 : kD / 2 + 8 * c;
  const int end = pg.cu ? pg.cu[pg.n_seqs] : x.n;
  float a[8], b[8];
  if (seg < q_segs) {
    const int g0 = seg * base + min(seg, extra), g1 = g0 + base + (seg < extra);
    Vec8<T> va[NB], vb[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int head = kRotHeads * (g0 + i) + sub;
      if (g0 + i >= g1 || head >= x.hq) continue;
      const T* src = static_cast<const T*>(x.q) + t * x.q_stride + head * kD;
      va[i].load(src + off0);
      vb[i].load(src + off1);
    }
    form_sines(x, rope, turn, t, cs[warp], sn[warp]);
    if (t >= end) return;  // padding behind the last sequence
    __syncwarp();
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int head = kRotHeads * (g0 + i) + sub;
      const bool live = head < x.hq;
      if (g0 + i >= g1) break;  // the same for the whole warp
      if (live) {
        va[i].get(a);
        vb[i].get(b);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) a[j] = b[j] = 0.f;
      }
      if (x.q_norm) norm_head<T>(a, b, static_cast<const T*>(x.q_norm), off0, off1, x.eps);
      turn_pairs<IL>(a, b, cs[warp], sn[warp], c);
      va[i].set(a);
      vb[i].set(b);
      if (live) {
        T* dst = q_out + ((size_t)t * x.hq + head) * kD;
        va[i].store(dst + off0);
        vb[i].store(dst + off1);
      }
    }
    return;
  }
  // four of the key heads and, behind them, the value heads
  const int first = kRotHeads * (seg - q_segs), head = first + sub;
  const bool keys = first < x.hkv, is_v = head >= x.hkv;  // keys: some of the four are
  const int h = min(is_v ? head - x.hkv : head, x.hkv - 1);
  bool live = head < 2 * x.hkv;
  Vec8<T> va, vb;
  if (live) {
    const T* src = is_v ? static_cast<const T*>(x.v) + t * x.v_stride : static_cast<const T*>(x.k) + t * x.k_stride;
    va.load(src + h * kD + off0);
    vb.load(src + h * kD + off1);
  }
  if (keys) form_sines(x, rope, turn, t, cs[warp], sn[warp]);
  if (t >= end) return;
  const Place at = token_place(pg, t);
  live = live && at.page >= 0;
  __syncwarp();
  if (live) {
    va.get(a);
    vb.get(b);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) a[j] = b[j] = 0.f;
    va.set(a);
    vb.set(b);
  }
  const float* factor = is_v ? q4.v_factor : q4.k_factor;
  const float f = factor ? factor[h] : 1.f;
  Q4Factor by = {f, false};  // keys' borders are settled below, with the factor as it is
  if (q4.v_factor) {
    const Q4Factor moved = q4_factor<T, 8>(f);
    if (is_v) by = moved;
  }
  // How far a rotated key's elements may be off, 8 half steps of the magnitudes
  // of their pair (its angle and sines 2.6, products and sum 2.4, the ends of what
  // it may be and their quotients 3), 24 with a norm (16 more: 19 additions halved
  // by the root, 2 ulp of the root, two products).
  float off[8], most = 0.f;
  if (keys) {
    if (x.k_norm) norm_head<T>(a, b, is_v ? nullptr : static_cast<const T*>(x.k_norm), off0, off1, x.eps);
    const float part = x.k_norm ? 24.f * 0x1p-24f : 8.f * 0x1p-24f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float p = IL ? (j < 4 ? a[2 * (j & 3)] : b[2 * (j & 3)]) : a[j];
      const float q = IL ? (j < 4 ? a[2 * (j & 3) + 1] : b[2 * (j & 3) + 1]) : b[j];
      off[j] = (fabsf(p) + fabsf(q)) * part;
      most = fmaxf(most, off[j]);
    }
    if (!is_v) turn_pairs<IL>(a, b, cs[warp], sn[warp], c);
  }
  uint32_t top[2] = {q4_top(a), q4_top(b)};
  if (IL) {  // a and b are one group
    top[0] = top[1] = max(top[0], top[1]);
  } else {
#pragma unroll
    for (int e = 0; e < 2; ++e) top[e] = max(top[e], __shfl_xor_sync(0xffffffffu, top[e], 1));
    most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
  }
  const Q4Recip by_six(6.f, by.f);
  const Q4Scale sa(top[0], by_six, by), sb(top[1], by_six, by);
  uint32_t code[2], scale[2] = {sa.byte, sb.byte}, open[2] = {0u, 0u};
  bool open_a = false, open_b = false;
  if (is_v) {
    code[0] = q4_word(a, sa, by);
    code[1] = q4_word(b, sb, by);
  } else {
    code[0] = codes_within<IL>(a, 0, off, most, sa.by, &open[0]);
    code[1] = codes_within<IL>(b, 1, off, most, sb.by, &open[1]);
    if (sa.byte == kQ4NaN) code[0] = open[0] = 0u;
    if (sb.byte == kQ4NaN) code[1] = open[1] = 0u;
    open_a = open_scale(top[0], most, by_six, &scale[0]);
    open_b = open_scale(top[1], most, by_six, &scale[1]);
  }
  if (keys && __any_sync(0xffffffffu, open[0] || open[1] || open_a || open_b)) {
    KeyPart part;
    Vec8<T> w[2];
    va.get(part.x[0]);
    vb.get(part.x[1]);
    if (x.k_norm) {
      w[0].load(static_cast<const T*>(x.k_norm) + off0);
      w[1].load(static_cast<const T*>(x.k_norm) + off1);
      w[0].get(part.w[0]);
      w[1].get(part.w[1]);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      part.off[j] = off[j];
      part.y[0][j] = a[j];
      part.y[1][j] = b[j];
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      part.code[e] = code[e];
      part.scale[e] = scale[e];
      part.open[e] = open[e];
    }
    part.most = most;
    part.open_scale[0] = open_a;
    part.open_scale[1] = open_b;
    settle_keys<IL>(&part, x.k_norm != nullptr, x.eps, x.pos, x.n, t, rope.end0, rope.end1, turn, f);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      code[e] = part.code[e];
      scale[e] = part.scale[e];
    }
  }
  if (!live) return;
  const size_t row = q4_row(pg, at.page, at.row, h, x.hkv);
  uint8_t* codes = (is_v ? q4.v : q4.k) + row * kQ4Row;
  uint8_t* scales = (is_v ? q4.v_scale : q4.k_scale) + row * kQ4Scales;
  *reinterpret_cast<uint32_t*>(codes + off0 / 2) = code[0];
  *reinterpret_cast<uint32_t*>(codes + off1 / 2) = code[1];
  if (IL || !(c & 1)) scales[off0 / kQ4Group] = (uint8_t)scale[0];
  if (!IL && !(c & 1)) scales[off1 / kQ4Group] = (uint8_t)scale[1];
}

cudaError_t launch_append_q4(DType dt, const TokenView& x, const RopeView& rope, const PageView& pages,
                             const Q4View& pools, void* q_out, cudaStream_t st) {
  const RotateShare s = rotate_share(x.n, (x.hq + kRotHeads - 1) / kRotHeads);
  const int segs = s.segs + (2 * x.hkv + kRotHeads - 1) / kRotHeads;
  // (with what fills the last four tokens)
  const dim3 grid((unsigned)(((long long)(x.n + 3) * segs + kRotWarps - 1) / kRotWarps));
  TimingScope ts("paged_append_q4", st);
  cudaError_t e = cudaSuccess;
  with_rotate_type(dt, s, [&](auto zero, auto nb) {
    typedef decltype(zero) T;
    constexpr int NB = decltype(nb)::value;
    auto kern = rope.interleaved ? k_append_q4<T, NB, true> : k_append_q4<T, NB, false>;
    e = launch_after(kern, grid, kRotThreads, 0, st, x, rope, pages, pools, static_cast<T*>(q_out), s.base, s.extra,
                     Order(x.n, s.segs, segs));
  });
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace stl
