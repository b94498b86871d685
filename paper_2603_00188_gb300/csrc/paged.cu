// Paged caches: new tokens' heads normed, rotated and written (packed, or keys
// and values into pages of 16 or 32 bits or of 4), and the compaction's rows
// moved into pages.
#include <type_traits>

#include "kernels.cuh"
#include "paged.cuh"
#include "q4.cuh"

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
//
// Into 4-bit pages keys and values go as they are here, in fp32, before they
// would be rounded: two neighbouring lanes share a group of 16 elements (one
// lane has it where pairs are interleaved).
constexpr int kRotThreads = 128, kRotWarps = kRotThreads / 32;
constexpr int kRotHeads = 4;   // heads of a group

// One warp per unit: segment `u % segs` of the head groups of token u / segs, `base` of them or, in the first
// `extra` segments, one more.
// To packed rows, to pages, or to pages in 4 bits.
enum RotateTo { kToRows = 0, kToPages = 1, kToQ4 = 2 };

template <typename T, int NB, bool IL, int TO>
__global__ void __launch_bounds__(kRotThreads) k_rotate(const __grid_constant__ TokenView x,
                                                        const __grid_constant__ RopeView rope,
                                                        const __grid_constant__ PageView pg,
                                                        const __grid_constant__ Q4View q4, T* q_out, T* k_out,
                                                        T* v_out, int base, int extra, int segs) {
  constexpr bool PAGED = TO != kToRows;
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
  Place at = {-1, 0};
  if (PAGED && kRotHeads * g1 > x.hq) at = token_place(pg, t);  // keys or values among the segment's heads
  const int slot = at.page >= 0 ? at.page * pg.page_rows + at.row : -1;
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
    if (TO == kToQ4 && kRotHeads * (g0 + i + 1) > x.hq) {  // a key or value in the group
      const int h = min(max(head - x.hq - (is_v ? x.hkv : 0), 0), x.hkv - 1);
      const float* factor = is_v ? q4.v_factor : q4.k_factor;
      const float f = factor ? factor[h] : 1.f;
      uint32_t top_a = q4_top(a), top_b = q4_top(b);
      if (IL) {  // a and b are one group
        top_a = top_b = max(top_a, top_b);
      } else {
        top_a = max(top_a, __shfl_xor_sync(0xffffffffu, top_a, 1));
        top_b = max(top_b, __shfl_xor_sync(0xffffffffu, top_b, 1));
      }
      const Q4Recip by_six(6.f * f);
      const Q4Scale sa(top_a, by_six, f), sb(top_b, by_six, f);
      if (live && !is_q && at.page >= 0) {
        const size_t row = q4_row(pg, at.page, at.row, h, x.hkv);
        uint8_t* codes = (is_v ? q4.v : q4.k) + row * kQ4Row;
        uint8_t* scales = (is_v ? q4.v_scale : q4.k_scale) + row * kQ4Scales;
        *reinterpret_cast<uint32_t*>(codes + off0 / 2) = q4_word(a, sa);
        *reinterpret_cast<uint32_t*>(codes + off1 / 2) = q4_word(b, sb);
        if (IL || !(c & 1)) scales[off0 / kQ4Group] = (uint8_t)sa.byte;
        if (!IL && !(c & 1)) scales[off1 / kQ4Group] = (uint8_t)sb.byte;
      }
    }
    if (TO == kToQ4 && !is_q) continue;
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

static cudaError_t run_rotate(DType dt, const TokenView& x, const RopeView& rope, RotateTo to, const PageView& pg,
                              const Q4View& q4, void* q_out, void* k_out, void* v_out, cudaStream_t st) {
  const int groups = (x.hq + (to != kToRows ? 2 : 1) * x.hkv + kRotHeads - 1) / kRotHeads;
  // groups of a warp: three, fewer where there are few tokens: 32 warps for each of the chip's 152 SMs (the grid's
  // shape alone depends on it)
  constexpr int most = 3;
  long long segs = (152 * 32 + x.n - 1) / x.n;
  if (segs < (groups + most - 1) / most) segs = (groups + most - 1) / most;
  if (segs > groups) segs = groups;
  const int base = (int)(groups / segs), extra = (int)(groups % segs), each = base + (extra > 0);
  const dim3 grid((unsigned)((x.n * segs + kRotWarps - 1) / kRotWarps));
  TimingScope ts(to == kToRows ? "rotate_qk" : (to == kToPages ? "paged_append" : "paged_append_q4"), st);
  cudaError_t e = cudaSuccess;
  auto run = [&](auto zero, auto nb) {
    typedef decltype(zero) T;
    constexpr int NB = decltype(nb)::value;
    T *qo = static_cast<T*>(q_out), *ko = static_cast<T*>(k_out), *vo = static_cast<T*>(v_out);
    auto pick = [&](auto il) {
      constexpr bool IL = decltype(il)::value;
      auto kern = to == kToRows ? k_rotate<T, NB, IL, kToRows>
                                : (to == kToPages ? k_rotate<T, NB, IL, kToPages> : k_rotate<T, NB, IL, kToQ4>);
      e = launch_after(kern, grid, kRotThreads, 0, st, x, rope, pg, q4, qo, ko, vo, base, extra, (int)segs);
    };
    if (rope.interleaved)
      pick(std::true_type());
    else
      pick(std::false_type());
  };
  auto pick = [&](auto zero) {
    if (each <= 1)
      run(zero, std::integral_constant<int, 1>());
    else if (each <= 2)
      run(zero, std::integral_constant<int, 2>());
    else
      run(zero, std::integral_constant<int, most>());
  };
  if (dt == kBF16)
    pick(__nv_bfloat16());
  else
    pick(float());
  return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t launch_rotate(DType dt, const TokenView& x, const RopeView& rope, const PageView* pages, void* q_out,
                          void* k_out, void* v_out, cudaStream_t st) {
  return run_rotate(dt, x, rope, pages ? kToPages : kToRows, pages ? *pages : PageView{}, Q4View{}, q_out, k_out, v_out,
                    st);
}

cudaError_t launch_append_q4(DType dt, const TokenView& x, const RopeView& rope, const PageView& pages,
                             const Q4View& pools, void* q_out, cudaStream_t st) {
  return run_rotate(dt, x, rope, kToQ4, pages, pools, q_out, nullptr, nullptr, st);
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
