// Attention of a serving step's new tokens over paged caches:
//   out[t][g] = sum_j softmax_j(q_{t,g} . k_{j,h} / sqrt(d)) v_{j,h}, h = g / G,
// over the rows j < len - (n - 1 - i) of the session, t its i-th of n new
// tokens.
#include <type_traits>

#include "kernels.cuh"

namespace stl {

constexpr int kPatThreads = 256;
constexpr int kPatWarps = kPatThreads / 32;
constexpr int kPatRows = 16;  // query rows of a CTA: (new token, query head) pairs of one KV head
constexpr float kPatLog2e = 1.4426950408889634f;

__device__ __forceinline__ float pat_weight(float a, float m) { return a == -CUDART_INF_F ? 0.f : exp2f(a - m); }
__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_f(float x, float* y) { *y = x; }
__device__ __forceinline__ void from_f(float x, __nv_bfloat16* y) { *y = __float2bfloat16_rn(x); }

// One CTA per (session, KV head, 16 query rows); a warp takes every eighth row
// of the cache, a lane four dimensions.
template <typename T>
__global__ void __launch_bounds__(kPatThreads) k_paged_attention(const __grid_constant__ PageView pg, const T* q,
                                                                 const T* k, const T* v, T* out, int n, int hq,
                                                                 int hkv, uint32_t* err) {
  __shared__ float wo[kPatWarps][kD];
  __shared__ float2 wml[kPatWarps];
  pdl_trigger();
  pdl_wait();
  const int s = blockIdx.x, h = blockIdx.y, r0 = blockIdx.z * kPatRows, G = hq / hkv;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int first = pg.cu ? pg.cu[s] : s * pg.w, fresh = pg.cu ? pg.cu[s + 1] - first : pg.w;
  const int cap = pg.max_pages * pg.page_rows, asked = pg.len[s], len = max(0, min(asked, cap));
  if (asked != len && threadIdx.x == 0) record_error(err, kErrInput);
  const float scale = kPatLog2e * rsqrtf((float)kD);
  for (int rr = r0; rr < min(r0 + kPatRows, min(fresh, pg.w) * G); ++rr) {
    const int i = rr / G, g = h * G + rr % G, t = first + i;
    if (t < 0 || t >= n) break;
    float qf[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -CUDART_INF_F, l = 0.f;
    for (int e = 0; e < 4; ++e) qf[e] = to_f(q[((size_t)t * hq + g) * kD + 4 * lane + e]) * scale;
    const int sees = len - (fresh - 1 - i);
    for (int j = warp; j < sees; j += kPatWarps) {
      const int p = j / pg.page_rows, page = pg.table[(size_t)s * pg.max_pages + p];
      if (page < 0 || page >= pg.n_pages) {
        if (lane == 0) record_error(err, kErrInput);
        continue;
      }
      const size_t at = (((size_t)page * pg.page_rows + (j - p * pg.page_rows)) * hkv + h) * kD + 4 * lane;
      float x = 0.f;
      for (int e = 0; e < 4; ++e) x = fmaf(qf[e], to_f(k[at + e]), x);
      x = warp_sum(x);
      const float mn = fmaxf(m, x), a = pat_weight(m, mn), w = pat_weight(x, mn);
      l = l * a + w;
      m = mn;
      for (int e = 0; e < 4; ++e) o[e] = fmaf(o[e], a, w * to_f(v[at + e]));
    }
    for (int e = 0; e < 4; ++e) wo[warp][4 * lane + e] = o[e];
    if (lane == 0) wml[warp] = make_float2(m, l);
    __syncthreads();
    if (threadIdx.x < kD) {
      float M = -CUDART_INF_F, L = 0.f, O = 0.f;
      for (int w = 0; w < kPatWarps; ++w) M = fmaxf(M, wml[w].x);
      for (int w = 0; w < kPatWarps; ++w) {
        const float a = pat_weight(wml[w].x, M);
        L = fmaf(wml[w].y, a, L);
        O = fmaf(wo[w][threadIdx.x], a, O);
      }
      from_f(L == 0.f ? 0.f : O / L, out + ((size_t)t * hq + g) * kD + threadIdx.x);
    }
    __syncthreads();
  }
}

size_t paged_workspace_bytes(DType, const PageView&, int, int) { return 256; }

cudaError_t launch_paged_attention(DType dt, const PageView& pages, const void* q, const void* k, const void* v,
                                   void* out, int n, int hq, int hkv, void* ws, cudaStream_t st) {
  const int chunks = (pages.w * (hq / hkv) + kPatRows - 1) / kPatRows;
  uint32_t* err = static_cast<uint32_t*>(ws);
  TimingScope ts("paged_attention", st);
  cudaError_t e = cudaSuccess;
  auto run = [&](auto zero) {
    typedef decltype(zero) T;
    e = launch_after(k_paged_attention<T>, dim3(pages.n_seqs, hkv, chunks), kPatThreads, 0, st, pages,
                     static_cast<const T*>(q), static_cast<const T*>(k), static_cast<const T*>(v),
                     static_cast<T*>(out), n, hq, hkv, err);
  };
  if (dt == kBF16)
    run(__nv_bfloat16());
  else
    run(float());
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace stl
