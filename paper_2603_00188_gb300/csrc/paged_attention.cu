// Attention of a serving step's new tokens over paged caches:
//   out[t][g] = sum_j softmax_j(q_{t,g} . k_{j,h} / sqrt(d)) v_{j,h}, h = g / G,
// over the rows j < len - (n - 1 - i) of the session, t its i-th of n new
// tokens.  Every cached row is read once per row chunk: the bytes of K and V
// bound it.
#include <type_traits>

#include "paged_split.cuh"

namespace stl {

constexpr int kPmWarps = 4, kPmThreads = 32 * kPmWarps;
constexpr int kPmCtas = 2;  // per SM
constexpr int kPatBlock = 16, kPatBlockShift = 4;  // cached rows of a block

// ---------------------------------------------------------------------- bf16
// Each warp streams its own blocks (every kPmWarps-th of the range) through its
// own ring of stages in shared memory: 16 rows of keys and of values by
// asynchronous 16-byte copies (any page size: a lane looks up its row's page
// one block ahead; rows that do not count are filled with zeros and masked).
// No warp waits for another until an item ends.  Both products run on the
// warp's tensor cores (m16n8k16, fp32 accumulation):
//   S (16 rows x 8 queries) = K Q^T,
//   O^T (128 dims x 8 queries) += V^T P^T, P transposed in registers by
//   movmatrix and taken as P = hi + lo, two bf16 parts (16 bits of it: with one
//   part the weights' rounding would be as large as the result's).
// That way the products of up to 21 query rows take less time than the bytes
// (rates below), and a warp passes from one product to the next in registers.
// From 28 rows on the products bound it; tcgen05 tiles with the cached rows, then
// the dimensions, as M and the queries as N would be the form for those.
// A value that is an infinity or a NaN does not go through these products: a
// weight of 0 (a row that only newer tokens see), a part lo of 0 or one of the
// other sign would make a NaN of it.  A warp whose sums are not finite at an
// item's end takes its blocks again and adds such rows apart, by fp32 products
// of the whole weight, to the queries that see them.
// NT: groups of eight queries that share one read of the cache: 1 or 2 with
// their fragments in registers, 3 or 4 with them read from shared memory.
// Measured: 32 sessions of 1,000 to 53,600 rows, 7 queries to a KV head, 146 to
// 153 us (6.2 to 6.5 TB/s with start and merge; the copies without the products
// take the same time, so HBM bounds it; four warps and two CTAs per SM 155 where
// eight and one take 160); one session of 10,757 rows 10.2 us, all latency.  16
// sessions of 25,000 rows: 6.4 TB/s with 7 or 14 queries, 6.1 with 21, 5.2 with
// 28, bound by the products' latency at two warps per scheduler.
constexpr int kPmHalf = kPatBlock * kD * 2;         // keys, or values, of a block
constexpr int kPmPitch = kD + 4;                    // floats from row to row of the merge buffer
__host__ __device__ constexpr int pm_stages(int nt) { return nt == 1 ? 3 : 2; }
__host__ __device__ constexpr int pm_ring(int nt) { return kPmWarps * pm_stages(nt) * 2 * kPmHalf; }
__host__ __device__ constexpr int pm_queries(int nt) { return nt > 2 ? 8 * nt * kD * 2 : 0; }
__host__ __device__ constexpr int pm_pass(int nt) { return nt > 2 ? 2 : nt; }  // groups merged at a time
__host__ __device__ constexpr int pm_factors(int nt) {
  return 8 * nt * 4 * (1 + kPmWarps) > (int)sizeof(RangeScratch<kPmThreads>) ? 8 * nt * 4 * (1 + kPmWarps)
                                                                            : (int)sizeof(RangeScratch<kPmThreads>);
}
__host__ __device__ constexpr int pm_smem(int nt) {
  return pm_ring(nt) + pm_queries(nt) + kPmWarps * 8 * (pm_pass(nt) * kPmPitch * 4 + nt * 8) + pm_factors(nt);
}
static_assert(fits_sm(pm_smem(1), kPmCtas) && fits_sm(pm_smem(2), kPmCtas) && fits_sm(pm_smem(3), kPmCtas) &&
                  fits_sm(pm_smem(4), kPmCtas), "kPmCtas per SM");

__device__ __forceinline__ void pm_ldsm_x4(uint32_t addr, uint32_t (&a)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(a[0]), "=r"(a[1]), "=r"(a[2]), "=r"(a[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void pm_ldsm_x4_trans(uint32_t addr, uint32_t (&a)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(a[0]), "=r"(a[1]), "=r"(a[2]), "=r"(a[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void pm_mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Whether either of two bf16 is an infinity or a NaN.
__device__ __forceinline__ bool has_odd_bf16(uint32_t x) {
  return (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u;
}

// Byte of the 16-byte chunk c of row r of a half stage, swizzled so that eight
// rows' chunks lie in eight different bank groups.
__device__ __forceinline__ uint32_t pm_off(int r, int c) { return (uint32_t)(r * 256 + ((c ^ (r & 7)) << 4)); }

template <int NT>
__global__ void __launch_bounds__(kPmThreads, kPmCtas)
    k_paged_mma(const __grid_constant__ PageView pg, const __nv_bfloat16* q, const __nv_bfloat16* k,
                const __nv_bfloat16* v, __nv_bfloat16* out, int n, int hq, int hkv, int mode, int split, int chunks,
                int chunk_rows, PartDesc* desc, float2* part_ml, float* part_o, uint32_t* err) {
  constexpr int kStages = pm_stages(NT), kRows = 8 * NT, kPass = pm_pass(NT);
  extern __shared__ uint4 pat_smem[];
  uint8_t* sm = reinterpret_cast<uint8_t*>(pat_smem);
  float* wo = reinterpret_cast<float*>(sm + pm_ring(NT) + pm_queries(NT));
  float2* wml = reinterpret_cast<float2*>(wo + kPmWarps * 8 * kPass * kPmPitch);
  RangeScratch<kPmThreads>* scratch = reinterpret_cast<RangeScratch<kPmThreads>*>(wml + kPmWarps * kRows);
  // once an item has ended (the range was found long before): 1 / sum of each
  // query, and the warps' factors
  float* inv = reinterpret_cast<float*>(scratch);  // [kRows]
  float* factor = inv + kRows;                     // [warps][kRows]
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g8 = lane >> 2, t4 = lane & 3;
  const int G = hq / hkv, cta = blockIdx.x;
  const uint32_t ring = smem_u32(sm) + warp * kStages * 2 * kPmHalf;
  pdl_trigger();
  pdl_wait();
  const Range rg = find_range<kPmThreads>(pg, G, chunk_rows, hkv, kPmWarps, split, err, scratch);
  const bool describes = tid == kPmThreads - 32;  // the thread that writes the CTA's descriptor
  if (mode == kDescByCta && describes) desc[cta].item = -1;
  if (cta >= rg.ctas) return;

  RowFinder<kPmWarps, kPatBlock> finder(rg);
  uint64_t counts = 0;  // 16 bits per stage: which rows of its block count
  const int fc = lane & 15, fr = lane >> 4;
  const __nv_bfloat16 *kf = k + 8 * fc, *vf = v + 8 * fc;
  const uint32_t f_off = fr * 256 + ((fc ^ fr) << 4);
  auto fetch = [&](int stage, int row) {
    if (row != -2) {
      const uint64_t ok = __ballot_sync(0xffffffffu, row >= 0) & 0xffffu;
      counts = (counts & ~(0xffffull << (16 * stage))) | ok << (16 * stage);
      const uint32_t dst = ring + stage * 2 * kPmHalf;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = __shfl_sync(0xffffffffu, row, 2 * i + fr);
        const size_t at = (size_t)max(r, 0) * kD;
        const uint32_t to = dst + 512 * i + (f_off ^ ((2 * i & 6) << 4));
        cp_async16_fill(to, kf + at, r >= 0);
        cp_async16_fill(to + kPmHalf, vf + at, r >= 0);
      }
    }
    cp_async_commit();
  };
  auto fill = [&]() {
    int first[kStages];  // all table entries on their way before the first copies
#pragma unroll
    for (int st = 0; st < kStages; ++st) first[st] = finder.next(pg, warp, G, chunk_rows, hkv, err);
#pragma unroll
    for (int st = 0; st < kStages; ++st) fetch(st, first[st]);
  };
  fill();

  const float scale = kPatLog2e * rsqrtf((float)kD);
  const uint32_t k_off = (lane & 15) * 256 + (((lane >> 4) ^ (lane & 7)) << 4);
  const uint32_t v_off = ((lane & 7) + 8 * (lane >> 4)) * 256 + ((((lane >> 3) & 1) ^ (lane & 7)) << 4);
  const uint32_t q_smem = smem_u32(sm) + pm_ring(NT);
  Cursor cur = rg.at;
  int stage = 0;
  for (int seg = rg.b0; seg < rg.b1;) {
    // the part of one item that lies in the range: blocks part0 .. seg_end
    advance(cur, seg, pg, G, chunk_rows, hkv);
    const Item item = item_at(cur, seg);
    const int h = item.h, chunk = item.chunk, part0 = max(seg, item.f0), seg_end = min(item.i1, rg.b1);
    const int row0 = chunk * chunk_rows, rows = min(chunk_rows, min(cur.w.fresh, pg.w) * G - row0);
    const bool owns = part0 == item.f0, whole = owns && seg_end == item.i1;  // has the first block, has them all
    if (cur.w.blocks == 0 || part0 >= seg_end) {
      if (cur.w.blocks == 0 && seg == item.i0) {  // an empty session, begun in this range
        if (mode == kDescByItem && describes) desc[(cur.s * hkv + h) * chunks + chunk].item = -1;
        zero_rows<kPmThreads>(out, cur.w.first, n, hq, h * G, G, row0, rows);
      }
      seg = seg_end;
      continue;
    }
    if (describes && owns && mode != kWholeItems) {
      const int id = (cur.s * hkv + h) * chunks + chunk;
      const PartDesc d = {whole ? -1 : id, cta, whole ? cta : rg.cta_of(item.i1 - 1), 0};
      if (mode == kDescByItem)
        desc[id] = d;
      else if (!whole)
        desc[cta] = d;
    }

    // query fragments: dimensions 16 ks + 2 t4 + {0, 1} and + 8 of query 8 nt + g8
    uint32_t qb[NT > 2 ? 1 : 8][NT > 2 ? 1 : NT][2];
    if constexpr (NT <= 2) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int r = row0 + 8 * nt + g8, t = cur.w.first + r / G;
        const bool ok = 8 * nt + g8 < rows && t >= 0 && t < n;
        const uint32_t* qr = reinterpret_cast<const uint32_t*>(q + ((size_t)(ok ? t : 0) * hq + h * G + r % G) * kD);
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
          qb[ks][nt][0] = ok ? qr[8 * ks + t4] : 0u;
          qb[ks][nt][1] = ok ? qr[8 * ks + 4 + t4] : 0u;
        }
      }
    } else {
      uint4 y[NT];  // a thread's chunks of the chunk's queries, loaded together
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const int x = 8 * i + (tid >> 4), r = row0 + x, t = cur.w.first + r / G;
        y[i] = make_uint4(0, 0, 0, 0);
        if (x < rows && t >= 0 && t < n)
          y[i] = reinterpret_cast<const uint4*>(q + ((size_t)t * hq + h * G + r % G) * kD)[tid & 15];
      }
#pragma unroll
      for (int i = 0; i < NT; ++i)
        *reinterpret_cast<uint4*>(sm + pm_ring(NT) + pm_off(8 * i + (tid >> 4), tid & 15)) = y[i];
      __syncthreads();
    }
    // Running state: raw maximum and the lane's part of the sum of queries
    // 8 nt + 2 t4 + e; o[mt][nt][j] is dimension 16 mt + g8 + 8 (j >> 1) of
    // query 8 nt + 2 t4 + (j & 1).
    float m[NT][2], l[NT][2], o[8][NT][4];
    const int all_see = cur.w.len - (cur.w.fresh - 1 - row0 / G);  // rows that every query sees
    // The warp's blocks of the part; look: for values that are no numbers.
    auto take = [&](auto look) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        m[nt][0] = m[nt][1] = -CUDART_INF_F;
        l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
        for (int mt = 0; mt < 8; ++mt) o[mt][nt][0] = o[mt][nt][1] = o[mt][nt][2] = o[mt][nt][3] = 0.f;
      }
      for (int u = warps_first<kPmWarps>(part0, warp); u < seg_end; u += kPmWarps) {
        cp_async_wait<kStages - 1>();
        __syncwarp();
        const int next = finder.next(pg, warp, G, chunk_rows, hkv, err);  // the block that will take this stage
        const uint32_t kt = ring + stage * 2 * kPmHalf + k_off, vt = ring + stage * 2 * kPmHalf + kPmHalf + v_off;
        const int base = (u - item.f0) * kPatBlock;
        constexpr int kChains = NT == 1 ? 2 : 1;  // independent accumulations
        float c[kChains][NT][4];
#pragma unroll
        for (int i = 0; i < kChains; ++i)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) c[i][nt][0] = c[i][nt][1] = c[i][nt][2] = c[i][nt][3] = 0.f;
        if constexpr (NT <= 2) {
#pragma unroll
          for (int ks = 0; ks < 8; ++ks) {
            uint32_t a[4];
            pm_ldsm_x4(kt - k_off + (k_off ^ (ks << 5)), a);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) pm_mma(c[ks % kChains][nt], a, qb[ks][nt][0], qb[ks][nt][1]);
          }
        } else {
#pragma unroll
          for (int kp = 0; kp < 4; ++kp) {
            uint32_t a[4], a2[4];
            pm_ldsm_x4(kt - k_off + (k_off ^ (kp << 6)), a);
            pm_ldsm_x4(kt - k_off + (k_off ^ (kp << 6 | 32)), a2);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              uint32_t f[4];
              pm_ldsm_x4(q_smem + pm_off(8 * nt + (lane & 7), 4 * kp + (lane >> 3)), f);
              pm_mma(c[0][nt], a, f[0], f[1]);
              pm_mma(c[0][nt], a2, f[2], f[3]);
            }
          }
        }
        if constexpr (kChains == 2) {
#pragma unroll
          for (int j = 0; j < 4; ++j) c[0][0][j] += c[1][0][j];
        }
        const uint32_t ok = (uint32_t)(counts >> (16 * stage)) & 0xffffu;
        if (ok != 0xffffu || base + kPatBlock > all_see) {  // some rows do not count for some queries
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int r = g8 + 8 * (j >> 1), x = 8 * nt + 2 * t4 + (j & 1);
              const int sees = cur.w.len - (cur.w.fresh - 1 - (row0 + x) / G);
              if (!(ok >> r & 1u) || base + r >= sees) c[0][nt][j] = -CUDART_INF_F;
            }
        }
        float ms[NT][2];  // the new maxima, scaled
        bool moved = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float mx = fmaxf(c[0][nt][e], c[0][nt][2 + e]);
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
            mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
            mx = fmaxf(m[nt][e], mx);
            ms[nt][e] = mx == -CUDART_INF_F ? 0.f : mx * scale;
            moved |= mx != m[nt][e];
          }
        if (__any_sync(0xffffffffu, moved)) {  // rare once the maxima have settled
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float mx = max3(m[nt][e], c[0][nt][e], c[0][nt][2 + e]);
              float all = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
              all = fmaxf(all, __shfl_xor_sync(0xffffffffu, all, 8));
              all = fmaxf(all, __shfl_xor_sync(0xffffffffu, all, 16));
              const float alpha = ex2_approx(fmaf(m[nt][e], scale, -ms[nt][e]));
              l[nt][e] *= alpha;
              m[nt][e] = all;
#pragma unroll
              for (int mt = 0; mt < 8; ++mt) {
                o[mt][nt][e] *= alpha;
                o[mt][nt][2 + e] *= alpha;
              }
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int j = 0; j < 4; ++j) {  // scores become probabilities
            c[0][nt][j] = ex2_approx(fmaf(c[0][nt][j], scale, -ms[nt][j & 1]));
            l[nt][j & 1] += c[0][nt][j];
          }
        if constexpr (decltype(look)::value) {
          uint8_t* values = sm + (warp * kStages + stage) * 2 * kPmHalf + kPmHalf;
          bool odd = false;
          if (ok >> (lane & 15) & 1u) {
#pragma unroll 1
            for (int i = 0; i < 8; ++i) {
              const uint4 y = *reinterpret_cast<const uint4*>(values + pm_off(lane & 15, 8 * (lane >> 4) + i));
              odd |= has_odd_bf16(y.x) || has_odd_bf16(y.y) || has_odd_bf16(y.z) || has_odd_bf16(y.w);
            }
          }
          const uint32_t halves = __ballot_sync(0xffffffffu, odd), apart = (halves | halves >> 16) & 0xffffu;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
            for (uint32_t left = apart; left != 0u; left &= left - 1u) {
              const int r = __ffs(left) - 1, from = (r & 7) * 4 + t4;
              float w[2];
              bool seen[2];
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const float y0 = __shfl_sync(0xffffffffu, c[0][nt][e], from);
                const float y1 = __shfl_sync(0xffffffffu, c[0][nt][2 + e], from);
                const int sees = cur.w.len - (cur.w.fresh - 1 - (row0 + 8 * nt + 2 * t4 + e) / G);
                w[e] = r < 8 ? y0 : y1;
                seen[e] = base + r < sees;
              }
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const int dim = 8 * i + g8;
                const float y = __bfloat162float(
                    *reinterpret_cast<const __nv_bfloat16*>(values + pm_off(r, i) + 2 * (dim & 7)));
#pragma unroll
                for (int e = 0; e < 2; ++e)
                  if (seen[e]) o[i >> 1][nt][2 * (i & 1) + e] = fmaf(w[e], y, o[i >> 1][nt][2 * (i & 1) + e]);
              }
            }
          __syncwarp();  // added: they count no more
          if (apart >> (lane & 15) & 1u)
            for (int i = 0; i < 8; ++i)
              *reinterpret_cast<uint4*>(values + pm_off(lane & 15, 8 * (lane >> 4) + i)) = make_uint4(0, 0, 0, 0);
          __syncwarp();
        }
        uint32_t ph[NT][2], pl[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const float p0 = c[0][nt][2 * x], p1 = c[0][nt][2 * x + 1];
            const uint32_t hi = pack_bf16(p0, p1);
            ph[nt][x] = transpose8x8(hi);
            pl[nt][x] = transpose8x8(pack_bf16(p0 - __uint_as_float(hi << 16), p1 - __uint_as_float(hi & 0xffff0000u)));
          }
#pragma unroll
        for (int mt = 0; mt < 8; ++mt) {
          uint32_t a[4];
          pm_ldsm_x4_trans(vt - v_off + (v_off ^ (mt << 5)), a);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            pm_mma(o[mt][nt], a, ph[nt][0], ph[nt][1]);
            pm_mma(o[mt][nt], a, pl[nt][0], pl[nt][1]);
          }
        }
        __syncwarp();
        fetch(stage, next);
        stage = stage + 1 == kStages ? 0 : stage + 1;
      }
    };
    take(std::false_type());
    float none = 0.f;  // or a NaN, where a sum is not finite
#pragma unroll
    for (int mt = 0; mt < 8; ++mt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 4; ++j) none = fmaf(o[mt][nt][j], 0.f, none);
    if (__any_sync(0xffffffffu, none != 0.f)) {
      cp_async_wait<0>();  // no copy is on its way to the stages
      __syncwarp();
      finder.start(cur, part0);
      fill();
      stage = 0;
      take(std::true_type());
    }
    // The warps' states of this item, merged in shared memory, kPass groups of
    // queries at a time.
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float s = l[nt][e];
        s += __shfl_xor_sync(0xffffffffu, s, 4);
        s += __shfl_xor_sync(0xffffffffu, s, 8);
        s += __shfl_xor_sync(0xffffffffu, s, 16);
        if (g8 == 0) wml[warp * kRows + 8 * nt + 2 * t4 + e] = make_float2(m[nt][e] * scale, s);
      }
    __syncthreads();
    const int part = 2 * cta + (owns ? 1 : 0);
    // a thread for each warp's query: its factor, and, from the first warp's
    // thread, the query's maximum and sum over the warps
    for (int e = tid; e < kPmWarps * kRows; e += kPmThreads) {
      const int x = e % kRows;
      float M = -CUDART_INF_F;
#pragma unroll
      for (int w = 0; w < kPmWarps; ++w) M = fmaxf(M, wml[w * kRows + x].x);
      factor[e] = pat_weight(wml[e].x, M);
      if (e < rows) {
        float L = 0.f;
#pragma unroll
        for (int w = 0; w < kPmWarps; ++w) L = fmaf(wml[w * kRows + x].y, pat_weight(wml[w * kRows + x].x, M), L);
        if (whole)
          inv[x] = L == 0.f ? 0.f : 1.f / L;
        else
          part_ml[part * kRows + x] = make_float2(M, L);
      }
    }
    __syncthreads();
#pragma unroll
    for (int n0 = 0; n0 < NT; n0 += kPass) {
      if (n0 > 0) __syncthreads();  // the buffer is free again
#pragma unroll
      for (int i = 0; i < kPass; ++i)
#pragma unroll
        for (int e = 0; e < 2 && n0 + i < NT; ++e) {
          const int x = 8 * i + 2 * t4 + e;
          const float a = factor[warp * kRows + 8 * n0 + x];
          float* w = wo + (warp * 8 * kPass + x) * kPmPitch + g8;
#pragma unroll
          for (int mt = 0; mt < 8; ++mt) {
            w[16 * mt] = o[mt][n0 + i][e] * a;
            w[16 * mt + 8] = o[mt][n0 + i][2 + e] * a;
          }
        }
      __syncthreads();
#pragma unroll 2
      for (int y = warp; y < min(8 * kPass, rows - 8 * n0); y += kPmWarps) {
        const int x = 8 * n0 + y;
        float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kPmWarps; ++w) {
          const float4 z = *reinterpret_cast<const float4*>(wo + (w * 8 * kPass + y) * kPmPitch + 4 * lane);
          O.x += z.x;
          O.y += z.y;
          O.z += z.z;
          O.w += z.w;
        }
        if (whole) {
          const int r = row0 + x, t = cur.w.first + r / G;
          const float f = inv[x];
          if (t >= 0 && t < n)
            store4(out + ((size_t)t * hq + h * G + r % G) * kD + 4 * lane, O.x * f, O.y * f, O.z * f, O.w * f);
        } else {
          store4(part_o + ((size_t)part * kRows + x) * kD + 4 * lane, O.x, O.y, O.z, O.w);
        }
      }
    }
    seg = seg_end;
    if (seg < rg.b1) __syncthreads();  // the merge buffer (and the queries) are free again
  }
  cp_async_wait<0>();
}

// ---------------------------------------------------------------------- fp32
// The same split and rings with fp32 products, two to an instruction
// (fma.rn.f32x2).  A block's keys and its values are a slot each, three to a
// warp.  Shared-memory reads bound the products, so a lane holds four rows of
// the keys against each chunk of a query that it reads:
//   scores: lane (r, c), r = 0 .. 3, c = 0 .. 7, sums rows r, r + 4, r + 8 and
//     r + 12 over every eighth 16-byte chunk from c on; the eight lanes' sums of
//     eight queries are added in 28 shuffles that leave lane c with query c's;
//   softmax: each lane its own query;
//   values: a lane owns four dimensions of every query, the probabilities come
//     back through shared memory.
// GM: queries of a chunk (4, or one or two times eight).
// Measured: 8 sessions of 25,000 rows, 7 queries to a KV head, 128 to 137 us (6.0
// to 6.4 TB/s; with two rows to a lane and every lane's exponentials of all queries
// 178), 14 queries 196 (30 TFLOP/s), bound by the reads of the products from
// shared memory; k_paged_fma<16> also spills (255 registers, 120 bytes).
constexpr int kPfSlots = 3;
constexpr int kPfHalf = kPatBlock * kD * 4;  // keys, or values, of a block
constexpr int kPfPass = 4;                   // queries merged at a time
__host__ __device__ constexpr int pf_ring() { return kPmWarps * kPfSlots * kPfHalf; }
// a warp's floats: probabilities of a block [gm][16] and rescaling factors [gm]
__host__ __device__ constexpr int pf_probs(int gm) { return gm * (kPatBlock + 1); }
// these, and, once an item has ended, the merge buffer
__host__ __device__ constexpr int pf_shared(int gm) {
  return kPmWarps * 4 * (pf_probs(gm) > kPfPass * kPmPitch ? pf_probs(gm) : kPfPass * kPmPitch);
}
__host__ __device__ constexpr int pf_smem(int gm) {
  return pf_ring() + gm * kD * 4 + pf_shared(gm) + kPmWarps * gm * 8 + (int)sizeof(RangeScratch<kPmThreads>);
}
static_assert(fits_sm(pf_smem(4), kPmCtas) && fits_sm(pf_smem(8), kPmCtas) && fits_sm(pf_smem(16), kPmCtas), "kPmCtas per SM");

// The sums over eight neighbouring lanes of s[row][query]: lane c of them is
// left with query c % Q's, rows 0 .. 3 for Q = 8, rows 2 (c / 4) + 0, 1 for Q = 4.
__device__ __forceinline__ void lane_sums(const float (&s)[4][8], int c, float (&out)[4]) {
  float a[4][4], b[4][2];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
#pragma unroll
    for (int x = 0; x < 4; ++x)
      a[j][x] = (c & 4 ? s[j][x + 4] : s[j][x]) + __shfl_xor_sync(0xffffffffu, c & 4 ? s[j][x] : s[j][x + 4], 4);
#pragma unroll
    for (int x = 0; x < 2; ++x)
      b[j][x] = (c & 2 ? a[j][x + 2] : a[j][x]) + __shfl_xor_sync(0xffffffffu, c & 2 ? a[j][x] : a[j][x + 2], 2);
    out[j] = (c & 1 ? b[j][1] : b[j][0]) + __shfl_xor_sync(0xffffffffu, c & 1 ? b[j][0] : b[j][1], 1);
  }
}
__device__ __forceinline__ void lane_sums(const float (&s)[4][4], int c, float (&out)[2]) {
  float a[2][4], b[2][2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
#pragma unroll
    for (int x = 0; x < 4; ++x)
      a[j][x] = (c & 4 ? s[j + 2][x] : s[j][x]) + __shfl_xor_sync(0xffffffffu, c & 4 ? s[j][x] : s[j + 2][x], 4);
#pragma unroll
    for (int x = 0; x < 2; ++x)
      b[j][x] = (c & 2 ? a[j][x + 2] : a[j][x]) + __shfl_xor_sync(0xffffffffu, c & 2 ? a[j][x] : a[j][x + 2], 2);
    out[j] = (c & 1 ? b[j][1] : b[j][0]) + __shfl_xor_sync(0xffffffffu, c & 1 ? b[j][0] : b[j][1], 1);
  }
}

template <int GM>
__global__ void __launch_bounds__(kPmThreads, kPmCtas)
    k_paged_fma(const __grid_constant__ PageView pg, const float* q, const float* k, const float* v, float* out, int n,
                int hq, int hkv, int mode, int split, int chunks, int chunk_rows, PartDesc* desc, float2* part_ml,
                float* part_o, uint32_t* err) {
  extern __shared__ uint4 pat_smem[];
  uint8_t* sm = reinterpret_cast<uint8_t*>(pat_smem);
  float* qs = reinterpret_cast<float*>(sm + pf_ring());  // [GM][128]
  float* shared = qs + GM * kD;
  float2* wml = reinterpret_cast<float2*>(sm + pf_ring() + GM * kD * 4 + pf_shared(GM));  // [warps][GM]
  RangeScratch<kPmThreads>* scratch = reinterpret_cast<RangeScratch<kPmThreads>*>(wml + kPmWarps * GM);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int G = hq / hkv, cta = blockIdx.x;
  uint8_t* ring = sm + warp * kPfSlots * kPfHalf;
  float* ps = shared + warp * pf_probs(GM);  // [GM][16]
  float* rescale = ps + GM * kPatBlock;      // [GM]
  pdl_trigger();
  pdl_wait();
  const Range rg = find_range<kPmThreads>(pg, G, chunk_rows, hkv, kPmWarps, split, err, scratch);
  const bool describes = tid == kPmThreads - 32;  // the thread that writes the CTA's descriptor
  if (mode == kDescByCta && describes) desc[cta].item = -1;
  if (cta >= rg.ctas) return;

  RowFinder<kPmWarps, kPatBlock> finder(rg);
  auto fetch = [&](int slot, int row, const float* from) {
    if (row != -2) {
      const uint32_t dst = smem_u32(ring) + slot * kPfHalf;
#pragma unroll
      for (int r = 0; r < kPatBlock; ++r) {
        const int x = __shfl_sync(0xffffffffu, row, r);
        cp_async16_fill(dst + 512 * r + 16 * lane, from + (size_t)max(x, 0) * kD + 4 * lane, x >= 0);
      }
    }
    cp_async_commit();
  };
  // keys and values alternate through the slots; the block after the current
  // one has its keys on the way
  int now = finder.next(pg, warp, G, chunk_rows, hkv, err), after = finder.next(pg, warp, G, chunk_rows, hkv, err);
  fetch(0, now, k);
  fetch(1, now, v);
  fetch(2, after, k);
  int slot = 0;

  const float scale = kPatLog2e * rsqrtf((float)kD);
  constexpr int Q = GM < 8 ? GM : 8, kSets = GM / Q, kLaneRows = Q == 8 ? 4 : 2;
  const int r4 = lane >> 3, c8 = lane & 7, mine = c8 & (Q - 1);  // the lane's query of each set
  const int lane_row = r4 + (Q == 8 ? 0 : 8 * (c8 >> 2));        // its rows: lane_row, + 4, ...
  Cursor cur = rg.at;
  for (int seg = rg.b0; seg < rg.b1;) {
    // the part of one item that lies in the range: blocks part0 .. seg_end
    advance(cur, seg, pg, G, chunk_rows, hkv);
    const Item item = item_at(cur, seg);
    const int h = item.h, chunk = item.chunk, part0 = max(seg, item.f0), seg_end = min(item.i1, rg.b1);
    const int row0 = chunk * chunk_rows, rows = min(chunk_rows, min(cur.w.fresh, pg.w) * G - row0);
    const bool owns = part0 == item.f0, whole = owns && seg_end == item.i1;  // has the first block, has them all
    if (cur.w.blocks == 0 || part0 >= seg_end) {
      if (cur.w.blocks == 0 && seg == item.i0) {  // an empty session, begun in this range
        if (mode == kDescByItem && describes) desc[(cur.s * hkv + h) * chunks + chunk].item = -1;
        zero_rows<kPmThreads>(out, cur.w.first, n, hq, h * G, G, row0, rows);
      }
      seg = seg_end;
      continue;
    }
    if (describes && owns && mode != kWholeItems) {
      const int id = (cur.s * hkv + h) * chunks + chunk;
      const PartDesc d = {whole ? -1 : id, cta, whole ? cta : rg.cta_of(item.i1 - 1), 0};
      if (mode == kDescByItem)
        desc[id] = d;
      else if (!whole)
        desc[cta] = d;
    }
    {
      float4 y[GM / 4];
#pragma unroll
      for (int i = 0; i < GM / 4; ++i) {
        const int x = 4 * i + warp, r = row0 + x, t = cur.w.first + r / G;
        y[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (x < rows && t >= 0 && t < n)
          y[i] = reinterpret_cast<const float4*>(q + ((size_t)t * hq + h * G + r % G) * kD)[lane];
      }
#pragma unroll
      for (int i = 0; i < GM / 4; ++i) reinterpret_cast<float4*>(qs + (4 * i + warp) * kD)[lane] = y[i];
    }
    __syncthreads();
    float m[kSets], l[kSets], o[GM][4];  // raw maximum and the lane's part of the sum of its queries
#pragma unroll
    for (int u = 0; u < kSets; ++u) {
      m[u] = -CUDART_INF_F;
      l[u] = 0.f;
    }
#pragma unroll
    for (int x = 0; x < GM; ++x) o[x][0] = o[x][1] = o[x][2] = o[x][3] = 0.f;
    const int all_see = cur.w.len - (cur.w.fresh - 1 - row0 / G);  // rows that every query sees
    for (int u = warps_first<kPmWarps>(part0, warp); u < seg_end; u += kPmWarps) {
      cp_async_wait<kPfSlots - 1>();
      __syncwarp();
      const int then = finder.next(pg, warp, G, chunk_rows, hkv, err);
      const uint32_t ok = __ballot_sync(0xffffffffu, now >= 0) & 0xffffu;
      const int base = (u - item.f0) * kPatBlock;
      const uint8_t* kt = ring + slot * kPfHalf + 512 * r4 + 16 * c8;
      float s[kSets][kLaneRows];
#pragma unroll
      for (int y = 0; y < kSets; ++y) {
        float lo[4][Q], hi[4][Q];  // even and odd dimensions
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int x = 0; x < Q; ++x) lo[j][x] = hi[j][x] = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float4 kk[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) kk[j] = *reinterpret_cast<const float4*>(kt + 2048 * j + 128 * i);
#pragma unroll
          for (int x = 0; x < Q; ++x) {
            const float4 z = *reinterpret_cast<const float4*>(qs + (Q * y + x) * kD + 32 * i + 4 * c8);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              fma2(kk[j].x, kk[j].y, z.x, z.y, lo[j][x], hi[j][x], lo[j][x], hi[j][x]);
              fma2(kk[j].z, kk[j].w, z.z, z.w, lo[j][x], hi[j][x], lo[j][x], hi[j][x]);
            }
          }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int x = 0; x < Q; ++x) lo[j][x] += hi[j][x];
        lane_sums(lo, c8, s[y]);
      }
      __syncwarp();
      fetch(slot, after, v);
      slot = slot + 1 == kPfSlots ? 0 : slot + 1;
      if (ok != 0xffffu || base + kPatBlock > all_see) {  // some rows do not count for some queries
#pragma unroll
        for (int y = 0; y < kSets; ++y) {
          const int sees = cur.w.len - (cur.w.fresh - 1 - (row0 + Q * y + mine) / G);
#pragma unroll
          for (int j = 0; j < kLaneRows; ++j)
            if (!(ok >> (lane_row + 4 * j) & 1u) || base + lane_row + 4 * j >= sees) s[y][j] = -CUDART_INF_F;
        }
      }
      bool moved = false;
#pragma unroll
      for (int y = 0; y < kSets; ++y) {
        float mx = s[y][0];
#pragma unroll
        for (int j = 1; j < kLaneRows; ++j) mx = fmaxf(mx, s[y][j]);
        if (Q == 4) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
        const float mn = fmaxf(m[y], mx), ms = mn == -CUDART_INF_F ? 0.f : mn;
        const float a = exp2f((m[y] - ms) * scale);  // 1 where the maximum stays
        moved |= mn != m[y];
        m[y] = mn;
        l[y] *= a;
        if (lane < Q) rescale[Q * y + mine] = a;
#pragma unroll
        for (int j = 0; j < kLaneRows; ++j) {
          const float e = exp2f((s[y][j] - ms) * scale);
          l[y] += e;
          ps[(Q * y + mine) * kPatBlock + lane_row + 4 * j] = e;
        }
      }
      moved = __any_sync(0xffffffffu, moved);
      cp_async_wait<kPfSlots - 1>();
      __syncwarp();
      if (moved) {  // rare once the maxima have settled
#pragma unroll
        for (int x = 0; x < GM; ++x) {
          const float a = rescale[x];
#pragma unroll
          for (int e = 0; e < 4; ++e) o[x][e] *= a;
        }
      }
      uint8_t* vt = ring + slot * kPfHalf + 16 * lane;
      if (cur.w.fresh > 1 && base + kPatBlock > all_see) {
        // Rows that only the newer tokens see: a weight of 0 times a value that
        // is no number would reach the older ones.  If there is one, these
        // rows are added here and count no more.
        const uint32_t rows_apart = ok & ~((1u << max(0, all_see - base)) - 1u);
        bool odd = false;
        for (uint32_t left = rows_apart; left != 0u; left &= left - 1u) {
          const float4 y = *reinterpret_cast<const float4*>(vt + 512 * (__ffs(left) - 1));
          odd |= !(isfinite(y.x) && isfinite(y.y) && isfinite(y.z) && isfinite(y.w));
        }
        if (__any_sync(0xffffffffu, odd))
          for (uint32_t left = rows_apart; left != 0u; left &= left - 1u) {
            const int r = __ffs(left) - 1;
            const float4 y = *reinterpret_cast<const float4*>(vt + 512 * r);
            *reinterpret_cast<float4*>(vt + 512 * r) = make_float4(0.f, 0.f, 0.f, 0.f);  // the lane's own dimensions
#pragma unroll
            for (int x = 0; x < GM; ++x) {
              const float w = ps[x * kPatBlock + r];
              if (base + r >= cur.w.len - (cur.w.fresh - 1 - (row0 + x) / G)) continue;
              o[x][0] = fmaf(w, y.x, o[x][0]);
              o[x][1] = fmaf(w, y.y, o[x][1]);
              o[x][2] = fmaf(w, y.z, o[x][2]);
              o[x][3] = fmaf(w, y.w, o[x][3]);
            }
          }
      }
#pragma unroll 2
      for (int r0 = 0; r0 < kPatBlock; r0 += 4) {
        float4 y[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = *reinterpret_cast<const float4*>(vt + 512 * (r0 + j));
#pragma unroll
        for (int x = 0; x < GM; ++x) {
          const float4 p4 = *reinterpret_cast<const float4*>(ps + x * kPatBlock + r0);
          const float p[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            fma2(p[j], p[j], y[j].x, y[j].y, o[x][0], o[x][1], o[x][0], o[x][1]);
            fma2(p[j], p[j], y[j].z, y[j].w, o[x][2], o[x][3], o[x][2], o[x][3]);
          }
        }
      }
      __syncwarp();
      now = after;
      after = then;
      fetch(slot, after, k);
      slot = slot + 1 == kPfSlots ? 0 : slot + 1;
    }
    // the warps' states of this item, merged in shared memory
#pragma unroll
    for (int y = 0; y < kSets; ++y) {
      float sum = l[y];
      if (Q == 4) sum += __shfl_xor_sync(0xffffffffu, sum, 4);
      sum += __shfl_xor_sync(0xffffffffu, sum, 8);
      sum += __shfl_xor_sync(0xffffffffu, sum, 16);
      if (lane < Q) wml[warp * GM + Q * y + mine] = make_float2(m[y] * scale, sum);
    }
    const int part = 2 * cta + (owns ? 1 : 0);
#pragma unroll
    for (int x0 = 0; x0 < GM; x0 += kPfPass) {
      __syncthreads();  // the probabilities, or the last pass, are done with
#pragma unroll
      for (int i = 0; i < kPfPass; ++i)
        *reinterpret_cast<float4*>(shared + (warp * kPfPass + i) * kPmPitch + 4 * lane) =
            make_float4(o[x0 + i][0], o[x0 + i][1], o[x0 + i][2], o[x0 + i][3]);
      __syncthreads();
      const int x = x0 + warp;  // a query for each warp
      if (x < rows) {
        float M = -CUDART_INF_F, L = 0.f;
#pragma unroll
        for (int w = 0; w < kPmWarps; ++w) M = fmaxf(M, wml[w * GM + x].x);
        float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kPmWarps; ++w) {
          const float2 ml = wml[w * GM + x];
          const float a = pat_weight(ml.x, M);
          L = fmaf(ml.y, a, L);
          const float4 z = *reinterpret_cast<const float4*>(shared + (w * kPfPass + warp) * kPmPitch + 4 * lane);
          O.x = fmaf(z.x, a, O.x);
          O.y = fmaf(z.y, a, O.y);
          O.z = fmaf(z.z, a, O.z);
          O.w = fmaf(z.w, a, O.w);
        }
        const int r = row0 + x, t = cur.w.first + r / G;
        if (whole) {
          const float inv = L == 0.f ? 0.f : 1.f / L;
          if (t >= 0 && t < n)
            store4(out + ((size_t)t * hq + h * G + r % G) * kD + 4 * lane, O.x * inv, O.y * inv, O.z * inv, O.w * inv);
        } else {
          *reinterpret_cast<float4*>(part_o + ((size_t)part * GM + x) * kD + 4 * lane) = O;
          if (lane == 0) part_ml[part * GM + x] = make_float2(M, L);
        }
      }
    }
    seg = seg_end;
    if (seg < rg.b1) __syncthreads();  // the merge buffer and the queries are free again
  }
  cp_async_wait<0>();
}

// --------------------------------------------------------------------- merge
// out of the items that several CTAs had parts of.  grid (descriptors, rows):
// each warp takes its share of the parts, a lane four dimensions; the parts'
// weights are formed in shared memory while the first partials are on their
// way, ten to a warp.  Eight warps take the 76 parts of one session on the whole
// GPU in one latency (10.3 us for 10,757 rows; four warps 12.1, four with twenty
// at once 11.4); where there are many CTAs the parts are few, and four warps
// launch faster (32 sessions: 150 us, eight warps 153).
constexpr int kMrgAtOnce = 10;
template <typename T, int kMrgThreads>
__global__ void __launch_bounds__(kMrgThreads) k_paged_merge(const __grid_constant__ PageView pg, T* out, int n,
                                                             int hq, int hkv, int chunks, int chunk_rows,
                                                             int part_rows, int by_item, const PartDesc* desc,
                                                             const float2* part_ml, const float* part_o) {
  constexpr int kMrgSlices = kMrgThreads / 32;
  __shared__ float wts[kPatMaxCtas];
  __shared__ float red[2][kMrgSlices];
  __shared__ float4 acc[kMrgSlices - 1][32];
  pdl_trigger();
  pdl_wait();
  const PartDesc d = desc[blockIdx.x];
  const int G = hq / hkv;
  if (by_item) {  // items of sessions with fewer rows have no entry
    const int per = hkv * chunks, s = blockIdx.x / per;
    if ((int)(blockIdx.x - s * per) % chunks >= seq_work(pg, s, 0, G, chunk_rows).chunks) return;
  }
  if (d.item < 0) return;
  const int hs = d.item / chunks, chunk = d.item - hs * chunks, s = hs / hkv, h = hs - s * hkv;
  const int x = blockIdx.y, r = chunk * chunk_rows + x, parts = d.c1 - d.c0 + 1;
  const int tid = threadIdx.x, slice = tid >> 5, lane = tid & 31;
  auto at = [&](int p) { return (p == 0 ? 2 * d.c0 + 1 : 2 * (d.c0 + p)) * part_rows + x; };
  float4 y[kMrgAtOnce];
  auto load = [&](int p0) {
#pragma unroll
    for (int u = 0; u < kMrgAtOnce; ++u) {
      const int p = p0 + slice + kMrgSlices * u;
      if (p < parts) y[u] = reinterpret_cast<const float4*>(part_o + (size_t)at(p) * kD)[lane];
    }
  };
  load(0);
  const float2 none = make_float2(-CUDART_INF_F, 0.f);
  const float2 ml0 = tid < parts ? part_ml[at(tid)] : none;
  const SeqWork w = seq_work(pg, s, 0, G, chunk_rows);
  float M = ml0.x;
  for (int p = tid + kMrgThreads; p < parts; p += kMrgThreads) M = fmaxf(M, part_ml[at(p)].x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
  if (lane == 0) red[0][slice] = M;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kMrgSlices; ++i) M = fmaxf(M, red[0][i]);
  float L = 0.f;
  for (int p = tid; p < parts; p += kMrgThreads) {
    const float2 ml = p == tid ? ml0 : part_ml[at(p)];
    const float a = pat_weight(ml.x, M);
    wts[p] = a;
    L = fmaf(ml.y, a, L);
  }
  L = warp_sum(L);
  if (lane == 0) red[1][slice] = L;
  __syncthreads();
  L = 0.f;
#pragma unroll
  for (int i = 0; i < kMrgSlices; ++i) L += red[1][i];
  float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int p0 = 0;;) {
#pragma unroll
    for (int u = 0; u < kMrgAtOnce; ++u) {
      const int p = p0 + slice + kMrgSlices * u;
      if (p < parts) {
        const float a = wts[p];
        O.x = fmaf(y[u].x, a, O.x);
        O.y = fmaf(y[u].y, a, O.y);
        O.z = fmaf(y[u].z, a, O.z);
        O.w = fmaf(y[u].w, a, O.w);
      }
    }
    p0 += kMrgSlices * kMrgAtOnce;
    if (p0 >= parts) break;
    load(p0);
  }
  if (slice > 0) acc[slice - 1][lane] = O;
  __syncthreads();
  if (slice > 0) return;
#pragma unroll
  for (int i = 0; i < kMrgSlices - 1; ++i) {
    O.x += acc[i][lane].x;
    O.y += acc[i][lane].y;
    O.z += acc[i][lane].z;
    O.w += acc[i][lane].w;
  }
  const int t = w.first + r / G;
  if (r >= min(w.fresh, pg.w) * G || t < 0 || t >= n) return;
  const float inv = L == 0.f ? 0.f : 1.f / L;
  store4(out + ((size_t)t * hq + h * G + r % G) * kD + 4 * lane, O.x * inv, O.y * inv, O.z * inv, O.w * inv);
}

cudaError_t launch_paged_merge(DType dt, const PageView& pages, void* out, int n, int hq, int hkv, int chunks,
                               int chunk_rows, int part_rows, bool by_item, int descs, const PartDesc* desc,
                               const float2* part_ml, const float* part_o, cudaStream_t st) {
  TimingScope ts("paged_merge", st);
  const dim3 grid(descs, chunk_rows);
  const bool few = descs * chunk_rows <= 304;  // two CTAs for each of the chip's SMs
  auto run = [&](auto zero) {
    typedef decltype(zero) T;
    auto kern = few ? k_paged_merge<T, 256> : k_paged_merge<T, 128>;
    return launch_after(kern, grid, few ? 256 : 128, 0, st, pages, static_cast<T*>(out), n, hq, hkv, chunks, chunk_rows,
                        part_rows, by_item, desc, part_ml, part_o);
  };
  return dt == kF32 ? run(float()) : run(__nv_bfloat16());
}

// -------------------------------------------------------------------- launch
static int paged_ctas() {
  int dev = 0, sms = 152;
  if (cudaGetDevice(&dev) == cudaSuccess) cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return kPmCtas * sms < kPatMaxCtas ? kPmCtas * sms : kPatMaxCtas;
}

// Query rows of a CTA's part, which share one read of the cache.
static int paged_part_rows(DType dt, const PageView& pages, int G) {
  const int rows = pages.w * G, most = dt == kF32 ? 16 : 32;
  const int chunks = (rows + most - 1) / most, each = (rows + chunks - 1) / chunks;
  if (dt == kF32) return each <= 4 ? 4 : (each <= 8 ? 8 : 16);
  return (each + 7) / 8 * 8;
}

// Workspace: the error word, the descriptors (16 KB), then two parts of each
// CTA: (max, sum) of its query rows, and their weighted values.
constexpr size_t kPatHead = 256, kPatDescs = kPatMaxCtas * sizeof(PartDesc);
size_t paged_workspace_bytes(DType dt, const PageView& pages, int hq, int hkv) {
  return kPatHead + kPatDescs +
         (size_t)2 * paged_ctas() * paged_part_rows(dt, pages, hq / hkv) * (sizeof(float2) + kD * sizeof(float));
}

cudaError_t launch_paged_attention(DType dt, const PageView& view, const void* q, const void* k, const void* v,
                                   void* out, int n, int hq, int hkv, void* ws, cudaStream_t st) {
  PageView pages = view;
  uint32_t* err = static_cast<uint32_t*>(ws);
  const int rows = pages.w * (hq / hkv), part_rows = paged_part_rows(dt, pages, hq / hkv);
  const int most = dt == kF32 ? 16 : 32, chunks = (rows + most - 1) / most, chunk_rows = (rows + chunks - 1) / chunks;
  const int ctas = paged_ctas();
  const long long items = (long long)pages.n_seqs * hkv * chunks;
  // An item's own costs, and what a split costs, in units: a block of up to 16
  // bf16 queries takes 0.2 us of a CTA's, one of more queries or of fp32 0.4.
  // (12 for the first: one session of 10,757 rows 0.6 us slower; 6 for the
  // others: five drafted tokens of eight sessions 1.8 us slower.)
  const bool light = dt == kBF16 && part_rows <= 16;
  pages.item_units = light ? 6 : 12;
  pages.block_shift = kPatBlockShift;
  int split = light ? 24 : 14;
  // Sessions that cannot be longer than a split and a little are never split,
  // which saves the second launch (one session of 256 rows: 7.0 us, split 6.9,
  // and 2 us less on the host; 64 sessions 8.4 and 14.8).
  const long long longest = ((long long)pages.max_pages * pages.page_rows + kPatBlock - 1) / kPatBlock;
  const int mode = longest <= (light ? 16 : 6) ? kWholeItems : (items <= ctas ? kDescByItem : kDescByCta);
  if (mode == kWholeItems) split = 1 << 30;
  const int descs = items <= ctas ? (int)items : ctas;
  uint8_t* at = static_cast<uint8_t*>(ws) + kPatHead;
  PartDesc* desc = reinterpret_cast<PartDesc*>(at);
  float2* part_ml = reinterpret_cast<float2*>(at + kPatDescs);
  float* part_o = reinterpret_cast<float*>(part_ml + (size_t)2 * ctas * part_rows);
  cudaError_t e = cudaSuccess;
  auto run = [&](auto zero, auto width) {
    typedef decltype(zero) T;
    constexpr int kWidth = decltype(width)::value;
    {
      TimingScope ts("paged_attention", st);
      auto go = [&](auto kern, int smem) {
        e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return;
        e = launch_after(kern, dim3(ctas), kPmThreads, smem, st, pages, static_cast<const T*>(q),
                         static_cast<const T*>(k), static_cast<const T*>(v), static_cast<T*>(out), n, hq, hkv, mode, split,
                         chunks, chunk_rows, desc, part_ml, part_o, err);
      };
      if constexpr (std::is_same<T, float>::value) {
        auto kern = k_paged_fma<kWidth>;
        go(kern, pf_smem(kWidth));
      } else {
        auto kern = k_paged_mma<kWidth>;
        go(kern, pm_smem(kWidth));
      }
      if (e != cudaSuccess || (e = cudaGetLastError()) != cudaSuccess || mode == kWholeItems) return;
    }
    e = launch_paged_merge(dt, pages, out, n, hq, hkv, chunks, chunk_rows, part_rows, mode == kDescByItem, descs, desc,
                           part_ml, part_o, st);
  };
  std::integral_constant<int, 1> w1;
  std::integral_constant<int, 2> w2;
  std::integral_constant<int, 3> w3;
  std::integral_constant<int, 4> w4;
  std::integral_constant<int, 8> w8;
  std::integral_constant<int, 16> w16;
  if (dt == kF32)
    part_rows == 4 ? run(float(), w4) : (part_rows == 8 ? run(float(), w8) : run(float(), w16));
  else
    part_rows <= 16 ? (part_rows == 8 ? run(__nv_bfloat16(), w1) : run(__nv_bfloat16(), w2))
                    : (part_rows == 24 ? run(__nv_bfloat16(), w3) : run(__nv_bfloat16(), w4));
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace stl
