// Rows into 4-bit pages (the compaction's; a step's tokens: k_append_q4) and out of
// them.
#include "kernels.cuh"
#include "paged.cuh"
#include "q4.cuh"

namespace stl {

// A group of sixteen elements as they are in memory.
template <typename T>
struct Group16 {
  Vec8<T> x[2];
  __device__ __forceinline__ void load(const T* p) {
    x[0].load(p);
    x[1].load(p + 8);
  }
  __device__ __forceinline__ void zero() {
    const float y[8] = {};
    x[0].set(y);
    x[1].set(y);
  }
  // The bits of its largest magnitude, as Q4Scale takes them.
  __device__ __forceinline__ uint32_t top() const;
};
template <>
__device__ __forceinline__ uint32_t Group16<float>::top() const {
  float y[2][8];
  x[0].get(y[0]);
  x[1].get(y[1]);
  return max(q4_top(y[0]), q4_top(y[1]));
}
// Two at a time, the sign of what comes out being of no account.
template <>
__device__ __forceinline__ uint32_t Group16<__nv_bfloat16>::top() const {
  const uint4 &a = x[0].u, &b = x[1].u;
  const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  uint32_t most = w[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) asm("max.NaN.xorsign.abs.bf16x2 %0, %0, %1;" : "+r"(most) : "r"(w[i]));
  return max(most << 16 & 0x7fff0000u, most & 0x7fff0000u);
}

// ---------------------------------------------------------------- compaction
// k_gather_paged with the kept rows put into 4 bits on the way.  A lane takes a
// group of 16 elements, eight lanes a row of a head, and a CTA 32 rows of one
// head, whose codes are one piece of each of their pages.  28 layers of 10,720
// rows: 115 us, a plain copy's rate for the bytes (a lane to 8 elements, whose
// scales two lanes then form, and a division for each element: some 200).  HBM
// bounds it, with the integer pipe half busy.
template <typename T>
__global__ void __launch_bounds__(256) k_gather_q4(const __grid_constant__ Q4Layers io,
                                                   const __grid_constant__ PageView pg, int seq, int n, int hkv,
                                                   int budget) {
  pdl_trigger();
  pdl_wait();
  const int l = blockIdx.z, h = blockIdx.y, c = threadIdx.x & 7, r = blockIdx.x * 32 + (threadIdx.x >> 3);
  const Q4View& to = io.pools[l];
  const float fk = to.k_factor ? to.k_factor[h] : 1.f, fv = to.v_factor ? to.v_factor[h] : 1.f;
  Q4Factor factors[2] = {{fk, sizeof(T) == 4 && q4_long(fk)}, {fv, sizeof(T) == 4 && q4_long(fv)}};
  if (sizeof(T) == 2 && (q4_long(fk) || q4_long(fv))) {  // the same for the whole CTA
    __shared__ float moved[2];
    const int warp = threadIdx.x >> 5;
    if (warp < 2) {
      const float f = q4_factor<T, 32>(warp ? fv : fk).f;
      if ((threadIdx.x & 31) == 0) moved[warp] = f;
    }
    __syncthreads();
    factors[0].f = moved[0];
    factors[1].f = moved[1];
  }
  if (r >= budget) return;
  const int src = io.idx[l][(size_t)h * budget + r];
  const Place at = page_place(pg, seq, r);
  if (at.page < 0 || src < 0 || src >= n) return;
  const size_t from = ((size_t)src * hkv + h) * kD + kQ4Group * c, row = q4_row(pg, at.page, at.row, h, hkv);
  Group16<T> x[2];
  x[0].load(static_cast<const T*>(io.k[l]) + from);
  x[1].load(static_cast<const T*>(io.v[l]) + from);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const Q4Factor f = factors[i];
    const Q4Scale s(x[i].top(), Q4Recip(6.f, f.f), f);
    float y[2][8];
    x[i].x[0].get(y[0]);
    x[i].x[1].get(y[1]);
    const uint2 w = make_uint2(q4_word(y[0], s, f), q4_word(y[1], s, f));
    *reinterpret_cast<uint2*>((i ? to.v : to.k) + row * kQ4Row + 8 * c) = w;
    (i ? to.v_scale : to.k_scale)[row * kQ4Scales + c] = (uint8_t)s.byte;
  }
}

cudaError_t launch_gather_q4(const Problem& p, const Q4Layers& io, int budget, const PageView& pages, int seq,
                             cudaStream_t st) {
  TimingScope ts("gather_q4", st);
  const dim3 grid((budget + 31) / 32, p.hkv, p.L);
  const cudaError_t e = launch_after(p.dtype == kBF16 ? k_gather_q4<__nv_bfloat16> : k_gather_q4<float>, grid, 256, 0,
                                     st, io, pages, seq, p.n, p.hkv, budget);
  return e != cudaSuccess ? e : cudaGetLastError();
}

// --------------------------------------------------------------------- fetch
// Rows as values.  A CTA's first warp finds the places of 32 tokens; then, for
// every head of its share of the layers' keys and values, a lane takes elements
// 8 g .. and 64 + 8 g .. of a row, so that what eight lanes write at a time lies
// together.  24 sessions, 65,000 rows of 12 layers: 324 us, 0.96 of a copy's rate
// (a warp to a token, its place found by the whole warp and a group of 16
// elements to a lane: 403).  Four heads are taken at once, of layers apart: three
// take 355 us, two 331, six 335, neighbours 362.
constexpr int kFetchTokens = 32, kFetchAtOnce = 4;
template <typename T>
__global__ void __launch_bounds__(256) k_fetch_q4(const __grid_constant__ Q4Layers io,
                                                  const __grid_constant__ PageView pg, int n, int hkv, int units) {
  __shared__ Place places[kFetchTokens];
  pdl_trigger();
  pdl_wait();
  const int t0 = blockIdx.x * kFetchTokens;
  if (threadIdx.x < kFetchTokens) {
    Place at = {-1, 0};
    if (t0 + (int)threadIdx.x < (pg.cu ? min(n, pg.cu[pg.n_seqs]) : n)) at = thread_token_place(pg, t0 + threadIdx.x);
    places[threadIdx.x] = at;
  }
  __syncthreads();
  const int g = threadIdx.x & 7, t = t0 + (threadIdx.x >> 3);
  const Place at = places[threadIdx.x >> 3];
  if (at.page < 0) return;
  // units: layers * 2 (keys, values) * heads
  for (int u0 = blockIdx.y; u0 < units; u0 += gridDim.y * kFetchAtOnce) {
    uint32_t w[kFetchAtOnce][2], b[kFetchAtOnce][2];
    float f[kFetchAtOnce];
    T* dst[kFetchAtOnce];
#pragma unroll
    for (int i = 0; i < kFetchAtOnce; ++i) {
      const int u = u0 + i * gridDim.y;
      if (u >= units) break;
      const int x = u / hkv, h = u - x * hkv, l = x >> 1;
      const bool is_v = x & 1;
      const Q4View& from = io.pools[l];
      const size_t row = q4_row(pg, at.page, at.row, h, hkv);
      const uint8_t *codes = (is_v ? from.v : from.k) + row * kQ4Row + 4 * g;
      const uint8_t* scales = (is_v ? from.v_scale : from.k_scale) + row * kQ4Scales + (g >> 1);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        w[i][k] = *reinterpret_cast<const uint32_t*>(codes + 32 * k);
        b[i][k] = scales[4 * k];
      }
      const float* factor = is_v ? from.v_factor : from.k_factor;
      f[i] = factor ? factor[h] : 1.f;
      dst[i] = static_cast<T*>(const_cast<void*>(is_v ? io.v[l] : io.k[l])) + ((size_t)t * hkv + h) * kD + 8 * g;
    }
#pragma unroll
    for (int i = 0; i < kFetchAtOnce; ++i) {
      if (u0 + i * (int)gridDim.y >= units) break;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const __half2 s2 = as_half2(q4_scales(b[i][k] | b[i][k] << 8));
        uint32_t p[4];
        float y[8];
        q4_codes(w[i][k], p);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 z = __half22float2(as_half2(mul_half2(p[j], s2)));
          y[2 * j] = z.x * f[i];
          y[2 * j + 1] = z.y * f[i];
        }
        Vec8<T> o;
        o.set(y);
        o.store(dst[i] + kD / 2 * k);
      }
    }
  }
}

cudaError_t launch_fetch_q4(DType dt, const Q4Layers& io, int layers, int n, int hkv, const PageView& pages,
                            cudaStream_t st) {
  TimingScope ts("paged_fetch_q4", st);
  const int blocks = (n + kFetchTokens - 1) / kFetchTokens, units = layers * 2 * hkv;
  // CTAs to the units of a block's tokens: one to those that it takes at once (24 sessions, 12 layers: 324 us; one to
  // all of them 337, one to two 331), and eight to each of the chip's 152 SMs in all where there are few tokens
  int share = (units + kFetchAtOnce - 1) / kFetchAtOnce;
  const int few = (152 * 8 + blocks - 1) / blocks;
  share = few > share ? few : share;
  share = share > units ? units : share;
  share = share > 65535 ? 65535 : share;
  const cudaError_t e = launch_after(dt == kBF16 ? k_fetch_q4<__nv_bfloat16> : k_fetch_q4<float>, dim3(blocks, share),
                                     256, 0, st, io, pages, n, hkv, units);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace stl
