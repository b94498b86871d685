// Rows into 4-bit pages (the compaction's, see k_rotate for a step's tokens)
// and out of them.
#include "kernels.cuh"
#include "paged.cuh"
#include "q4.cuh"

namespace stl {

// ---------------------------------------------------------------- compaction
// k_gather_paged with the kept rows put into 4 bits on the way.  16 lanes hold a
// row of a head, 8 elements each, two lanes a group; a CTA takes 16 rows of one
// head, whose codes are one piece of their page.
template <typename T>
__global__ void __launch_bounds__(256) k_gather_q4(const __grid_constant__ Q4Layers io,
                                                   const __grid_constant__ PageView pg, int seq, int n, int hkv,
                                                   int budget) {
  pdl_trigger();
  pdl_wait();
  const int l = blockIdx.z, h = blockIdx.y, c = threadIdx.x & 15, r = blockIdx.x * 16 + (threadIdx.x >> 4);
  int src = -1;
  Place at = {-1, 0};
  if (r < budget) {
    src = io.idx[l][(size_t)h * budget + r];
    at = page_place(pg, seq, r);
  }
  const bool live = at.page >= 0 && src >= 0 && src < n;
  const Q4View& to = io.pools[l];
  Vec8<T> x[2];
  float f[2] = {1.f, 1.f};
  if (live) {
    const size_t from = ((size_t)src * hkv + h) * kD + 8 * c;
    x[0].load(static_cast<const T*>(io.k[l]) + from);
    x[1].load(static_cast<const T*>(io.v[l]) + from);
    if (to.k_factor) f[0] = to.k_factor[h];
    if (to.v_factor) f[1] = to.v_factor[h];
  }
  const size_t row = live ? q4_row(pg, at.page, at.row, h, hkv) : 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float y[8] = {};
    if (live) x[i].get(y);
    uint32_t top = q4_top(y);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    const Q4Scale s = q4_scale(top, f[i]);
    const uint32_t w = q4_word(y, s);
    if (live) {
      *reinterpret_cast<uint32_t*>((i ? to.v : to.k) + row * kQ4Row + 4 * c) = w;
      if (!(c & 1)) (i ? to.v_scale : to.k_scale)[row * kQ4Scales + (c >> 1)] = (uint8_t)s.byte;
    }
  }
}

cudaError_t launch_gather_q4(const Problem& p, const Q4Layers& io, int budget, const PageView& pages, int seq,
                             cudaStream_t st) {
  TimingScope ts("gather_q4", st);
  const dim3 grid((budget + 15) / 16, p.hkv, p.L);
  const cudaError_t e = launch_after(p.dtype == kBF16 ? k_gather_q4<__nv_bfloat16> : k_gather_q4<float>, grid, 256, 0,
                                     st, io, pages, seq, p.n, p.hkv, budget);
  return e != cudaSuccess ? e : cudaGetLastError();
}

// --------------------------------------------------------------------- fetch
// Rows as values: a warp takes a token's heads, a group of 16 elements to a
// lane, in every layer of its share.
template <typename T>
__global__ void __launch_bounds__(128) k_fetch_q4(const __grid_constant__ Q4Layers io,
                                                  const __grid_constant__ PageView pg, int n, int hkv, int layers) {
  pdl_trigger();
  pdl_wait();
  const int lane = threadIdx.x & 31, t = blockIdx.x * 4 + (threadIdx.x >> 5);
  if (t >= (pg.cu ? min(n, pg.cu[pg.n_seqs]) : n)) return;
  const Place at = token_place(pg, t);
  if (at.page < 0) return;
  for (int l = blockIdx.y; l < layers; l += gridDim.y) {
    const Q4View& from = io.pools[l];
    for (int e = lane; e < 2 * hkv * kQ4Scales; e += 32) {
      const int g = e & (kQ4Scales - 1), kh = e / kQ4Scales, is_v = kh >= hkv, h = is_v ? kh - hkv : kh;
      const size_t row = q4_row(pg, at.page, at.row, h, hkv);
      const uint2 w = *reinterpret_cast<const uint2*>((is_v ? from.v : from.k) + row * kQ4Row + 8 * g);
      const uint32_t b = (is_v ? from.v_scale : from.k_scale)[row * kQ4Scales + g], s = q4_scales(b | b << 8);
      const float* factor = is_v ? from.v_factor : from.k_factor;
      const float f = factor ? factor[h] : 1.f;
      T* dst = static_cast<T*>(const_cast<void*>(is_v ? io.v[l] : io.k[l])) + ((size_t)t * hkv + h) * kD + kQ4Group * g;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint32_t p[4];
        float y[8];
        q4_codes(i ? w.y : w.x, p);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t v = mul_f16x2(p[j], s);
          const float2 z = __half22float2(*reinterpret_cast<const __half2*>(&v));
          y[2 * j] = z.x * f;
          y[2 * j + 1] = z.y * f;
        }
        Vec8<T> o;
        o.set(y);
        o.store(dst + 8 * i);
      }
    }
  }
}

cudaError_t launch_fetch_q4(DType dt, const Q4Layers& io, int layers, int n, int hkv, const PageView& pages,
                            cudaStream_t st) {
  TimingScope ts("paged_fetch_q4", st);
  const int blocks = (n + 3) / 4;
  int share = 152 * 16 / blocks;  // CTAs to a token's layers, where there are few tokens
  share = share < 1 ? 1 : (share > layers ? layers : share);
  const cudaError_t e = launch_after(dt == kBF16 ? k_fetch_q4<__nv_bfloat16> : k_fetch_q4<float>, dim3(blocks, share),
                                     128, 0, st, io, pages, n, hkv, layers);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace stl
