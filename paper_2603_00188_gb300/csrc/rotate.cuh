// A token's rotation, of the kernels that write it to rows, pages and 4-bit pages.
#pragma once

#include <type_traits>

#include "kernels.cuh"
#include "paged.cuh"

namespace stl {

constexpr int kRotThreads = 128, kRotWarps = kRotThreads / 32;
constexpr int kRotHeads = 4;   // heads of a group

// How a token's groups of heads are dealt to warps: `segs` segments of `base` groups, `extra` of one more.
constexpr int kRotMost = 3;  // groups of a warp
struct RotateShare {
  int base, extra, segs;
};
static RotateShare rotate_share(int n, int groups) {
  // kRotMost, fewer where there are few tokens: 32 warps for each of the chip's 152 SMs (the grid's
  // shape alone depends on it)
  long long segs = (152 * 32 + n - 1) / n;
  if (segs < (groups + kRotMost - 1) / kRotMost) segs = (groups + kRotMost - 1) / kRotMost;
  if (segs > groups) segs = groups;
  return {(int)(groups / segs), (int)(groups % segs), (int)segs};
}
template <typename F>
static void with_rotate_type(DType dt, const RotateShare& s, const F& run) {
  const int each = s.base + (s.extra > 0);
  auto pick = [&](auto zero) {
    if (each <= 1)
      run(zero, std::integral_constant<int, 1>());
    else if (each <= 2)
      run(zero, std::integral_constant<int, 2>());
    else
      run(zero, std::integral_constant<int, kRotMost>());
  };
  if (dt == kBF16)
    pick(__nv_bfloat16());
  else
    pick(float());
}

// k_rotate's steps.  (It holds them itself: through these its 8,616 tokens took 26.8 us, not 26.3.)
//
// The 64 sines and cosines of token t, two to a lane, where the lanes find them.
__device__ __forceinline__ void form_sines(const TokenView& x, const RopeView& rope, const uint64_t* turn, int t,
                                           float4 (&cs)[2][8], float4 (&sn)[2][8]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int pair = lane + 32 * e, axis = pair < rope.end0 ? 0 : (pair < rope.end1 ? 1 : 2);
    const uint64_t angle = (uint64_t)(int64_t)x.pos[(size_t)axis * x.n + t] * turn[pair];
    const int at = (pair & 4) * 8 + (pair >> 3) * 4 + (pair & 3);
    sincospif((float)(int32_t)(angle >> 32) * 0x1p-31f, reinterpret_cast<float*>(sn) + at,
              reinterpret_cast<float*>(cs) + at);
  }
}

// The lane's elements of a head under its norm (null: none).  Eight lanes a head, whole warp.
template <typename T>
__device__ __forceinline__ void norm_head(float (&a)[8], float (&b)[8], const T* norm, int off0, int off1, float eps) {
  float ss = 0.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) ss = fmaf(a[j], a[j], fmaf(b[j], b[j], ss));
#pragma unroll
  for (int o = 1; o < 8; o <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
  if (!norm) return;
  const float r = rsqrtf(ss * (1.f / kD) + eps);
  Vec8<T> n0, n1;
  float wa[8], wb[8];
  n0.load(norm + off0);
  n1.load(norm + off1);
  n0.get(wa);
  n1.get(wb);
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    a[j] = a[j] * r * wa[j];
    b[j] = b[j] * r * wb[j];
  }
}

// The lane's pairs turned: pair j is (a[j], b[j]), or interleaved within a, then b.
template <bool IL>
__device__ __forceinline__ void turn_pairs(float (&a)[8], float (&b)[8], const float4 (&cs)[2][8],
                                           const float4 (&sn)[2][8], int c) {
#pragma unroll
  for (int g = 0; g < 2; ++g) {
    const float4 c4 = cs[g][c], s4 = sn[g][c];
    const float cv[4] = {c4.x, c4.y, c4.z, c4.w}, sv[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float& p = IL ? (g == 0 ? a[2 * j] : b[2 * j]) : a[4 * g + j];
      float& q = IL ? (g == 0 ? a[2 * j + 1] : b[2 * j + 1]) : b[4 * g + j];
      const float y0 = p * cv[j] - q * sv[j], y1 = q * cv[j] + p * sv[j];
      p = y0;
      q = y1;
    }
  }
}

}  // namespace stl
