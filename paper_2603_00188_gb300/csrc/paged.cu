// Paged caches: new tokens' heads normed, rotated and written (packed, or keys
// and values into pages), and the compaction's rows moved into pages.
#include "kernels.cuh"

namespace stl {

// ------------------------------------------------------------------ rotation
// y = x / sqrt(mean(x^2) + eps) * norm, then pair (a, b) -> (a cos - b sin,
// b cos + a sin) by the token's position, all in fp32 and rounded once.
//
// The angle is formed in whole numbers: position times the pair's turn, a
// 64-bit fraction of a full turn, whose overflow drops the whole turns.  Its
// upper 32 bits are the angle within the turn to 2^-33 of one, exact for any
// position, where fp32 angles lose a bit with every doubling of the position.
//
// Eight lanes hold a head, each eight pairs (two 16-byte vectors of bf16); a
// warp holds four heads of one token at a time and walks the token's heads
// with its sines and cosines in registers.

constexpr int kRotThreads = 256;
constexpr int kRotHeads = 4;   // heads of a warp at a time
constexpr int kRotPairs = 8;   // pairs of a lane

__device__ __forceinline__ void load_vec(const __nv_bfloat16* p, float (&f)[8]) {
  const uint4 u = *reinterpret_cast<const uint4*>(p);
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load_vec(const float* p, float (&f)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
  f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
__device__ __forceinline__ void store_vec(__nv_bfloat16* p, const float (&f)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store_vec(float* p, const float (&f)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1], f[2], f[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(f[4], f[5], f[6], f[7]);
}

// Slot (page * page_rows + row of the page) of row r of sequence s, or -1.
__device__ __forceinline__ int page_slot(const PageView& pg, int s, int r) {
  if (r < 0 || r >= pg.max_pages * pg.page_rows) return -1;
  const int i = pg.page_shift >= 0 ? r >> pg.page_shift : r / pg.page_rows, page = pg.table[(size_t)s * pg.max_pages + i];
  return page >= 0 && page < pg.n_pages ? page * pg.page_rows + (r - i * pg.page_rows) : -1;
}

// Sequence of packed new token t, or -1 for padding behind the last one.
__device__ __forceinline__ int find_seq(const PageView& pg, int t) {
  if (!pg.cu) {
    const int s = t / pg.w;
    return s < pg.n_seqs ? s : -1;
  }
  if (t >= pg.cu[pg.n_seqs]) return -1;
  int lo = 0, hi = pg.n_seqs;  // cu[lo] <= t < cu[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (pg.cu[mid] <= t)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// One warp per unit: segment `u % segs` of the head groups of token u / segs.
template <typename T, bool IL, bool PAGED>
__global__ void __launch_bounds__(kRotThreads) k_rotate(const __grid_constant__ TokenView x,
                                                        const __grid_constant__ RopeView rope,
                                                        const __grid_constant__ PageView pg, T* q_out, T* k_out,
                                                        T* v_out, int groups, int segs) {
  __shared__ uint64_t turn[kD / 2];
  if (threadIdx.x < kD / 2) turn[threadIdx.x] = rope.turn[threadIdx.x];
  __syncthreads();
  pdl_trigger();
  pdl_wait();
  const long long u = (long long)blockIdx.x * (kRotThreads / 32) + (threadIdx.x >> 5);
  const int t = (int)(u / segs), seg = (int)(u % segs);
  if (t >= x.n) return;
  const int lane = threadIdx.x & 31, sub = lane >> 3, c = lane & 7;
  int slot = -1;
  if (PAGED) {
    const int s = find_seq(pg, t);
    if (s < 0) return;
    const int next = pg.cu ? pg.cu[s + 1] : (s + 1) * pg.w;
    slot = page_slot(pg, s, pg.len[s] - (next - t));
  }
  float cs[kRotPairs], sn[kRotPairs];
  {
    const bool axes = rope.end0 < kD / 2;
    const int p0 = x.pos[t], p1 = axes ? x.pos[x.n + t] : 0, p2 = axes ? x.pos[2 * (size_t)x.n + t] : 0;
#pragma unroll
    for (int i = 0; i < kRotPairs; ++i) {
      const int pair = kRotPairs * c + i;
      const int p = pair < rope.end0 ? p0 : (pair < rope.end1 ? p1 : p2);
      const uint64_t a = (uint64_t)(int64_t)p * turn[pair];
      sincospif((float)(int32_t)(a >> 32) * 0x1p-31f, &sn[i], &cs[i]);
    }
  }
  const int total = x.hq + (PAGED ? 2 : 1) * x.hkv;
  const int g0 = (int)((long long)groups * seg / segs), g1 = (int)((long long)groups * (seg + 1) / segs);
  const int off0 = IL ? 16 * c : 8 * c, off1 = IL ? 16 * c + 8 : kD / 2 + 8 * c;
  for (int g = g0; g < g1; ++g) {
    const int head = kRotHeads * g + sub;
    const bool is_q = head < x.hq, is_k = !is_q && head < x.hq + x.hkv;
    const T *src = nullptr, *norm = nullptr;
    T* dst = nullptr;
    if (is_q) {
      src = static_cast<const T*>(x.q) + t * x.q_stride + head * kD;
      norm = static_cast<const T*>(x.q_norm);
      dst = q_out + ((size_t)t * x.hq + head) * kD;
    } else if (head < total) {
      const int h = head - x.hq - (is_k ? 0 : x.hkv);
      src = (is_k ? static_cast<const T*>(x.k) + t * x.k_stride : static_cast<const T*>(x.v) + t * x.v_stride) + h * kD;
      norm = is_k ? static_cast<const T*>(x.k_norm) : nullptr;
      if (!PAGED)
        dst = k_out + ((size_t)t * x.hkv + h) * kD;
      else if (slot >= 0)
        dst = (is_k ? k_out : v_out) + ((size_t)slot * x.hkv + h) * kD;
    }
    float a[8], b[8];  // the lane's elements: pair i is (a[i], b[i]), or interleaved within a, then b
    if (src) {
      load_vec(src + off0, a);
      load_vec(src + off1, b);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] = b[i] = 0.f;
    }
    if (x.q_norm || x.k_norm) {
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(a[i], a[i], fmaf(b[i], b[i], ss));
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      if (norm) {
        const float r = rsqrtf(ss * (1.f / kD) + x.eps);
        float wa[8], wb[8];
        load_vec(norm + off0, wa);
        load_vec(norm + off1, wb);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          a[i] = a[i] * r * wa[i];
          b[i] = b[i] * r * wb[i];
        }
      }
    }
    if (is_q || is_k) {
#pragma unroll
      for (int i = 0; i < kRotPairs; ++i) {
        float& p = IL ? (i < 4 ? a[2 * i] : b[2 * i - 8]) : a[i];
        float& q = IL ? (i < 4 ? a[2 * i + 1] : b[2 * i - 7]) : b[i];
        const float y0 = p * cs[i] - q * sn[i], y1 = q * cs[i] + p * sn[i];
        p = y0;
        q = y1;
      }
    }
    if (dst) {
      store_vec(dst + off0, a);
      store_vec(dst + off1, b);
    }
  }
}

cudaError_t launch_rotate(DType dt, const TokenView& x, const RopeView& rope, const PageView* pages, void* q_out,
                          void* k_out, void* v_out, cudaStream_t st) {
  const int groups = (x.hq + (pages ? 2 : 1) * x.hkv + kRotHeads - 1) / kRotHeads;
  // enough warps for the GPU's SMs where there are few tokens
  long long segs = (152 * 16 + x.n - 1) / x.n;
  if (segs > groups) segs = groups;
  const long long warps = (long long)x.n * segs, per = kRotThreads / 32;
  const dim3 grid((unsigned)((warps + per - 1) / per));
  const PageView pg = pages ? *pages : PageView{};
  TimingScope ts(pages ? "paged_append" : "rotate_qk", st);
  cudaError_t e = cudaSuccess;
  auto run = [&](auto zero) {
    typedef decltype(zero) T;
    T *qo = static_cast<T*>(q_out), *ko = static_cast<T*>(k_out), *vo = static_cast<T*>(v_out);
    auto kern = rope.interleaved ? (pages ? k_rotate<T, true, true> : k_rotate<T, true, false>)
                                 : (pages ? k_rotate<T, false, true> : k_rotate<T, false, false>);
    e = launch_after(kern, grid, kRotThreads, 0, st, x, rope, pg, qo, ko, vo, groups, (int)segs);
  };
  if (dt == kBF16)
    run(__nv_bfloat16());
  else
    run(float());
  return e != cudaSuccess ? e : cudaGetLastError();
}

// ---------------------------------------------------------------- compaction
// k_gather with the kept rows going to a sequence's pages: a thread moves one
// 16-byte chunk of a key and of a value, CPR of them to a head's row, so that
// consecutive threads write consecutive chunks.  The bytes moved bound it: at
// 28 layers of 10,720 rows it copies at 0.94 of the rate of a plain copy (194
// us; four chunks to a thread, all loads first, 208; the same in a loop over a
// grid of eight CTAs per SM 234: such threads all read, then all write).
template <int CPR>
__global__ void __launch_bounds__(256) k_gather_paged(const __grid_constant__ LayerPtrs io,
                                                      const __grid_constant__ PageView pg, int seq, int n, int hkv) {
  pdl_trigger();
  pdl_wait();
  const int l = blockIdx.y, budget = io.budget[l];
  const int c = threadIdx.x % CPR, rh = blockIdx.x * (256 / CPR) + threadIdx.x / CPR;
  const int r = rh / hkv, h = rh - r * hkv;
  if (r >= budget) return;
  const int src = io.idx[l][(size_t)h * budget + r], slot = page_slot(pg, seq, r);
  if (src < 0 || src >= n || slot < 0) return;
  const size_t from = ((size_t)src * hkv + h) * CPR + c, to = ((size_t)slot * hkv + h) * CPR + c;
  const uint4 k = static_cast<const uint4*>(io.k[l])[from], v = static_cast<const uint4*>(io.v[l])[from];
  static_cast<uint4*>(io.k_out[l])[to] = k;
  static_cast<uint4*>(io.v_out[l])[to] = v;
}

cudaError_t launch_gather_paged(const Problem& p, const LayerPtrs& io, const PageView& pages, int seq,
                                cudaStream_t st) {
  const int cpr = p.dtype == kBF16 ? kD * 2 / 16 : kD * 4 / 16;
  long long most = 1;
  for (int l = 0; l < p.L; ++l) most = io.budget[l] > most ? io.budget[l] : most;
  const int rows = 256 / cpr;  // of heads, a CTA's
  TimingScope ts("gather_paged", st);
  const dim3 grid((unsigned)((most * p.hkv + rows - 1) / rows), p.L);
  const cudaError_t e = launch_after(cpr == 16 ? k_gather_paged<16> : k_gather_paged<32>, grid, 256, 0, st, io, pages,
                                     seq, p.n, p.hkv);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace stl
