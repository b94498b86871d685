// Paged caches: new tokens' heads normed, rotated and written (packed, or keys
// and values into pages), and the compaction's rows moved into pages.
#include "kernels.cuh"
#include "paged.cuh"
#include "rotate.cuh"

namespace stl {

// ------------------------------------------------------------------ rotation
// y = x / sqrt(mean(x^2) + eps) * norm, then pair (a, b) -> (a cos - b sin,
// b cos + a sin) by the token's position, all in fp32 and rounded once.
//
// The angle is formed in whole numbers: position times the pair's turn, a
// 64-bit fraction of a full turn, whose overflow drops the whole turns, so that
// no position costs precision (fp32 angles lose a bit with every doubling of
// it).  Its upper 32 bits, cut off to 2^-32 of a turn, are rounded to fp32, half
// turns: the angle within (-pi, pi) to 2^-24 of itself, as the fp32 sine and
// cosine of any angle start from.  That is some 1.2 times as far from 64 bits in
// the result as angles of 64 bits would be (1,152 fp32 tokens: 5.0e-8 relative
// against 4.1e-8); sines of a wider angle would cost the issue slots that
// already are 60 % taken.
//
// Eight lanes hold a head, each eight pairs (two 16-byte vectors of bf16), so
// that a warp holds four heads.  A warp takes up to NB such groups of a token's
// heads, all loaded before anything else, and meanwhile forms the token's 64
// sines and cosines, two to a lane, exchanged through shared memory.  The bytes
// moved bound it: 8,576 tokens of 28 + 4 bf16 heads take 22.3 us (6.3 TB/s, 0.93
// of a plain copy's rate; groups of a loop without loading ahead 27.1, eight
// groups ahead 22.8, a CTA to 32 heads with shared sines 29.8), 8,616 tokens
// with 4 value heads into pages 26.0 (eight groups 34.0, four 27.2, two 28.0).
// One warp per unit: segment `u % segs` of the head groups of token u / segs, `base` of them or, in the first
// `extra` segments, one more.
template <typename T, int NB, bool IL, bool PAGED>
__global__ void __launch_bounds__(kRotThreads) k_rotate(const __grid_constant__ TokenView x,
                                                        const __grid_constant__ RopeView rope,
                                                        const __grid_constant__ PageView pg, T* q_out, T* k_out,
                                                        T* v_out, int base, int extra, int segs) {
  __shared__ uint64_t turn[kD / 2];
  // [warp][four of a lane's eight pairs][lane][pair], so that eight lanes' vectors are adjacent
  __shared__ float4 cs[kRotWarps][2][8], sn[kRotWarps][2][8];
  if (threadIdx.x < kD / 2) turn[threadIdx.x] = rope.turn[threadIdx.x];
  __syncthreads();
  pdl_trigger();
  pdl_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane >> 3, c = lane & 7;
  const int u = blockIdx.x * kRotWarps + warp, t = u / segs, seg = u - t * segs;
  if (t >= x.n) return;
  const int total = x.hq + (PAGED ? 2 : 1) * x.hkv;
  const int g0 = seg * base + min(seg, extra), g1 = g0 + base + (seg < extra);
  const int off0 = IL ? 16 * c : 8 * c, off1 = IL ? 16 * c + 8 : kD / 2 + 8 * c;
  const int end = PAGED && pg.cu ? pg.cu[pg.n_seqs] : x.n;
  Vec8<T> va[NB], vb[NB];
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    const int head = kRotHeads * (g0 + i) + sub;
    if (g0 + i >= g1 || head >= total) continue;
    const T* src = static_cast<const T*>(x.q) + t * x.q_stride + head * kD;
    if (head >= x.hq) src = static_cast<const T*>(x.k) + t * x.k_stride + (head - x.hq) * kD;
    if (PAGED && head >= x.hq + x.hkv) src = static_cast<const T*>(x.v) + t * x.v_stride + (head - x.hq - x.hkv) * kD;
    va[i].load(src + off0);
    vb[i].load(src + off1);
  }
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int pair = lane + 32 * e, axis = pair < rope.end0 ? 0 : (pair < rope.end1 ? 1 : 2);
    const uint64_t angle = (uint64_t)(int64_t)x.pos[(size_t)axis * x.n + t] * turn[pair];
    const int at = (pair & 4) * 8 + (pair >> 3) * 4 + (pair & 3);
    sincospif((float)(int32_t)(angle >> 32) * 0x1p-31f, reinterpret_cast<float*>(sn[warp]) + at,
              reinterpret_cast<float*>(cs[warp]) + at);
  }
  if (t >= end) return;  // padding behind the last sequence
  int slot = -1;
  if (PAGED && kRotHeads * g1 > x.hq) slot = token_slot(pg, t);  // keys or values among the segment's heads
  __syncwarp();
#pragma unroll
  for (int i = 0; i < NB; ++i) {
    const int head = kRotHeads * (g0 + i) + sub;
    const bool live = g0 + i < g1 && head < total, is_q = head < x.hq, is_v = PAGED && head >= x.hq + x.hkv;
    if (g0 + i >= g1) break;  // the same for the whole warp
    float a[8], b[8];  // the lane's elements: pair j is (a[j], b[j]), or interleaved within a, then b
    if (live) {
      va[i].get(a);
      vb[i].get(b);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) a[j] = b[j] = 0.f;
    }
    if (x.q_norm || x.k_norm) {
      float ss = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) ss = fmaf(a[j], a[j], fmaf(b[j], b[j], ss));
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      const T* norm = static_cast<const T*>(is_v ? nullptr : (is_q ? x.q_norm : x.k_norm));
      if (norm) {
        const float r = rsqrtf(ss * (1.f / kD) + x.eps);
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
    }
    if (!is_v) {
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const float4 c4 = cs[warp][g][c], s4 = sn[warp][g][c];
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
      va[i].set(a);
      vb[i].set(b);
    }
    T* dst = q_out + ((size_t)t * x.hq + head) * kD;
    if (!is_q) {
      const int h = head - x.hq - (is_v ? x.hkv : 0);
      dst = (is_v ? v_out : k_out) + ((size_t)(PAGED ? slot : t) * x.hkv + h) * kD;
    }
    if (live && (is_q || !PAGED || slot >= 0)) {
      va[i].store(dst + off0);
      vb[i].store(dst + off1);
    }
  }
}

cudaError_t launch_rotate(DType dt, const TokenView& x, const RopeView& rope, const PageView* pages, void* q_out,
                          void* k_out, void* v_out, cudaStream_t st) {
  const RotateShare s = rotate_share(x.n, (x.hq + (pages ? 2 : 1) * x.hkv + kRotHeads - 1) / kRotHeads);
  const dim3 grid((unsigned)(((long long)x.n * s.segs + kRotWarps - 1) / kRotWarps));
  const PageView pg = pages ? *pages : PageView{};
  TimingScope ts(pages ? "paged_append" : "rotate_qk", st);
  cudaError_t e = cudaSuccess;
  with_rotate_type(dt, s, [&](auto zero, auto nb) {
    typedef decltype(zero) T;
    constexpr int NB = decltype(nb)::value;
    T *qo = static_cast<T*>(q_out), *ko = static_cast<T*>(k_out), *vo = static_cast<T*>(v_out);
    auto kern = rope.interleaved ? (pages ? k_rotate<T, NB, true, true> : k_rotate<T, NB, true, false>)
                                 : (pages ? k_rotate<T, NB, false, true> : k_rotate<T, NB, false, false>);
    e = launch_after(kern, grid, kRotThreads, 0, st, x, rope, pg, qo, ko, vo, s.base, s.extra, s.segs);
  });
  return e != cudaSuccess ? e : cudaGetLastError();
}

// ---------------------------------------------------------------- compaction
// k_gather with the kept rows going to a sequence's pages: a thread moves one
// 16-byte chunk of a key and of a value, CPR of them to a head's row, so that
// consecutive threads write consecutive chunks.  The bytes moved bound it: at
// 28 layers of 10,720 rows it copies at 0.98 of the rate of a plain copy (186
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
