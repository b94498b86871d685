// Attention of a serving step's new tokens over paged caches in 4 bits:
//   out[t][g] = sum_j softmax_j(q_{t,g} . K_j / sqrt(d)) V_j,
//   K = code * scale * factor (q4.cuh), and V the same,
// over the rows that paged_attention.cu says, divided among CTAs as there
// (paged_split.cuh).
//
// Each warp streams its own blocks of 32 rows through its own ring in shared
// memory and decodes them in registers, as operands of its tensor cores'
// m16n8k16 products of fp16 with fp32 sums:
//   S (16 rows x 8 queries) = K Q^T: a lane takes 32 neighbouring elements of a
//     row (one 16-byte read; four codes a step, the sum's order is free),
//   O^T (128 dims x 8 queries) += V^T P^T: a lane takes one group of 16 elements
//     of each of four rows, whose codes it pairs by rows (the sum runs over
//     them) before they are decoded.
// code * scale is exact in fp16. What is rounded: queries, scaled by a power of
// two so that the largest element of each is in [1, 2), to fp16, which holds
// bf16 ones exactly down to 2^-17 of the largest and loses less than 2^-25 of
// it below; and weights, to fp16's 11 bits (2^-12, an eighth of the bf16 result's
// own rounding: 32 sessions of 1,000 to 53,600 rows are off from 64 bits by 1.685e-3
// of the result where that rounding alone makes 1.673e-3; with weights in two parts,
// also 1.673e-3, they take 61.7 us and not 55.9, 28 queries to a head 130 and not
// 100).  fp32 queries and their weights are taken as hi + lo, two parts of 11 bits,
// which is twice the products (off by 4.6e-7, as fp32 throughout).
//
// Weights are 2^(x - m), m the largest score so far less 10, moved only when one
// exceeds it by more than 14: no maximum is formed for blocks that do not.  So they
// are at most 2^14 (fp16 goes to 2^16).  Scores of 2^27 and more, whose difference
// to m fp32 cannot hold within that, have the largest itself as m.
//
// What bounds it.  16 sessions of 25,000 rows, one token of 7 queries to a KV
// head, take 48 to 51 us with start (4 us) and merge, 4.8 TB/s, 0.70 of a copy's
// rate (with the copies alone 44, with the decoding and the products alone 47):
// of some 300 instructions to 16 rows 64 convert codes, 64 multiply by scales, 16
// are products and 30 copy; conversions and integer instructions share a pipe
// that takes one every two cycles and is busy half of the time, no scheduler has
// more than three warps, and branches in a block cost more than their
// instructions (looking for bad pages and bad scales at the end: 61 -> 56 us for
// 32 sessions of 1,000 to 53,600 rows; the mask's branch apart from the block, or
// the next table entries asked for after it: 60).  14 queries take 60 us, 21 75,
// 28 100: the products then.  fp32: half as many sessions 33 us.
#include <type_traits>

#include "paged_split.cuh"
#include "q4.cuh"

namespace stl {

constexpr int kQaBlock = 32, kQaBlockShift = 5;  // cached rows of a block
constexpr int kQaStages = 2;  // of a warp's ring
constexpr int kQaCodes = kQaBlock * kQ4Row, kQaScales = kQaBlock * kQ4Scales;  // of keys, or of values, of a block
constexpr int kQaStage = 2 * (kQaCodes + kQaScales);
constexpr int kQaPitch = kD + 4;      // floats from row to row of the merge buffer
constexpr float kQaLift = 10.f;       // weights are 2^(x - m), m their reference less this
constexpr float kQaSlack = 4.f;       // how far a score may exceed the reference
constexpr int kQaWarps = 4, kQaThreads = 32 * kQaWarps;
// CTAs per SM.  12 warps of one group of queries keep their state in 168
// registers (16 in 128: 61 us where 12 take 56), eight of more in 255.
__host__ __device__ constexpr int qa_ctas(int nt) { return nt == 1 ? 3 : 2; }
// Bytes of shared memory for queries; none where they are in registers.
__host__ __device__ constexpr int qa_queries(int nt, int parts) { return nt * parts > 1 ? 8 * nt * parts * kD * 2 : 0; }
constexpr int kQaRing = kQaWarps * kQaStages * kQaStage;
// Once an item has ended: 1 / sum of each query, and the warps' factors; the split's scratch before.
__host__ __device__ constexpr int qa_factors(int nt) {
  return 8 * nt * 4 * (1 + kQaWarps) > (int)sizeof(RangeScratch<kQaThreads>) ? 8 * nt * 4 * (1 + kQaWarps)
                                                                            : (int)sizeof(RangeScratch<kQaThreads>);
}
__host__ __device__ constexpr int qa_smem(int nt, int parts) {
  const int merge = kQaWarps * 8 * nt * (kQaPitch * 4 + 8);  // the warps' sums, maxima and weights
  const int need = kQaRing + qa_queries(nt, parts) + merge + qa_factors(nt) + 8 * nt * 4;
  // No more CTAs share an SM than are dealt to it: otherwise those of a launch
  // that starts while another ends gather on the SMs that are free first (16
  // sessions of 25,000 rows: up to 75 us in place of 53).
  const int alone = (228 * 1024 / (qa_ctas(nt) + 1) - 1024) / 128 * 128 + 128;
  return need > alone ? need : alone;
}

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 unpack_f16(uint32_t x) { return __half22float2(as_half2(x)); }
__device__ __forceinline__ void cp_async8(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async8_fill(uint32_t dst, const void* src, bool valid) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(valid ? 8 : 0) : "memory");
}

// Reads of a ring's stage: after the wait for its copies and before the next copies to it.
template <int OFFSET>
__device__ __forceinline__ uint4 lds128(uint32_t at) {
  uint4 x;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4 + %5];"
               : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w)
               : "r"(at), "n"(OFFSET));
  return x;
}
template <int OFFSET>
__device__ __forceinline__ uint2 lds64(uint32_t at) {
  uint2 x;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2 + %3];" : "=r"(x.x), "=r"(x.y) : "r"(at), "n"(OFFSET));
  return x;
}
template <int OFFSET>
__device__ __forceinline__ uint32_t lds32(uint32_t at) {
  uint32_t x;
  asm volatile("ld.shared.b32 %0, [%1 + %2];" : "=r"(x) : "r"(at), "n"(OFFSET));
  return x;
}
template <int OFFSET>
__device__ __forceinline__ uint32_t lds16(uint32_t at) {
  uint16_t x;
  asm volatile("ld.shared.u16 %0, [%1 + %2];" : "=h"(x) : "r"(at), "n"(OFFSET));
  return x;
}

// Four neighbouring elements of a query, as they are in memory.
template <typename T>
struct Query4;
template <>
struct Query4<float> {
  float4 x;
  __device__ __forceinline__ float4 get() const { return x; }
};
template <>
struct Query4<__nv_bfloat16> {
  uint2 x;
  __device__ __forceinline__ float4 get() const {
    return make_float4(__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xffff0000u), __uint_as_float(x.y << 16),
                       __uint_as_float(x.y & 0xffff0000u));
  }
};

// Byte of the 16-byte chunk c of value row r in its block: eight rows' first
// chunks, which a read takes together, lie in different banks.
__device__ __forceinline__ uint32_t qa_value_off(int r, int c) {
  return (uint32_t)((r >> 1) * 128 + ((((r & 1) * 4 + c) ^ (((r >> 1) & 3) << 1)) << 4));
}

// NT: groups of eight queries that share one read of the cache.
template <typename T, int NT>
__global__ void __launch_bounds__(kQaThreads, qa_ctas(NT))
    k_paged_q4(const __grid_constant__ PageView pg, const __grid_constant__ Q4View pools, const T* q, T* out, int n,
               int hq, int hkv, int mode, int split, int chunks, int chunk_rows, PartDesc* desc, float2* part_ml,
               float* part_o, uint32_t* err) {
  constexpr int kParts = std::is_same<T, float>::value ? 2 : 1;  // of a query's elements and of a weight
  constexpr int kRows = 8 * NT;
  constexpr int kTiles = NT * kParts >= 4 ? 1 : 2;  // of 16 rows, whose scores are formed together
  constexpr bool kRegs = qa_queries(NT, kParts) == 0;  // queries in registers, else in shared memory
  extern __shared__ uint4 pat_smem[];
  uint8_t* sm = reinterpret_cast<uint8_t*>(pat_smem);
  uint2* qs = reinterpret_cast<uint2*>(sm + kQaRing);  // [part][NT][step][lane]
  float* wo = reinterpret_cast<float*>(sm + kQaRing + qa_queries(NT, kParts));
  float2* wml = reinterpret_cast<float2*>(wo + kQaWarps * kRows * kQaPitch);
  RangeScratch<kQaThreads>* scratch = reinterpret_cast<RangeScratch<kQaThreads>*>(wml + kQaWarps * kRows);
  // [kRows]: what each query's sums are multiplied by
  float* q_back = reinterpret_cast<float*>(sm + qa_smem(NT, kParts) - kRows * 4);
  float* inv = reinterpret_cast<float*>(scratch);  // [kRows]
  float* factor = inv + kRows;                     // [warps][kRows]
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g8 = lane >> 2, t4 = lane & 3;
  const int G = hq / hkv, cta = blockIdx.x;
  const uint32_t pick = (g8 & 3) | (4 + (g8 & 3)) << 4;  // the lane's group's byte of two words
  const uint32_t ring = smem_u32(sm) + warp * kQaStages * kQaStage;
  pdl_trigger();
  pdl_wait();
  const Range rg = find_range<kQaThreads>(pg, G, chunk_rows, hkv, kQaWarps, split, err, scratch);
  const bool describes = tid == kQaThreads - 32;  // the thread that writes the CTA's descriptor
  if (mode == kDescByCta && describes) desc[cta].item = -1;
  if (cta >= rg.ctas) return;

  // The warp's blocks, one after the other.  A block's table entries are asked for
  // while another block is worked on, and looked at when it is to be copied.
  struct {
    Cursor at;
    int u, f0, i1;  // the next block, and the first block and the end of the item that it is sought in
    const int32_t* entries;
    int head_row;   // of the item's head: its first row in a page
  } find;
  auto start = [&](const Cursor& c, int from) {
    find.at = c;
    find.u = find.f0 = find.i1 = from;
  };
  struct Entry {
    int page, row;  // the lane's row of the block: the page, and the row in it and the head; -1: no row of the session
  };
  auto look_up = [&](Entry& e) {  // false past the range
    while (find.u >= find.i1) {
      if (find.i1 >= rg.b1) return false;
      advance(find.at, find.i1, pg, G, chunk_rows, hkv);
      const Item x = item_at(find.at, find.i1);
      find.u = warps_first<kQaWarps>(max(find.i1, x.f0), warp);
      find.f0 = x.f0;
      find.i1 = x.i1;
      find.entries = pg.table + (size_t)find.at.s * pg.max_pages;
      find.head_row = x.h * pg.page_rows;
    }
    if (find.u >= rg.b1) return false;
    const int j = (find.u - find.f0) * kQaBlock + lane;
    find.u += kQaWarps;
    const int i = pg.page_shift >= 0 ? j >> pg.page_shift : j / pg.page_rows;
    e.row = find.head_row + j - i * pg.page_rows;
    if (j < find.at.w.len)
      e.page = find.entries[i];
    else
      e.row = -1;
    return true;
  };
  // A stage: keys' codes, values' codes, keys' scales, values' scales.  Of a row
  // that does not count only the scales are written, zeros: whatever codes lie in
  // its place are numbers.
  bool bad = false;              // a table entry was no page
  uint32_t ok = 0, ok_next = 0;  // rows that count of the block at hand, and of the one after it
  // where the lane reads in a stage: keys' codes and scales, values' even and odd rows and scales
  const uint32_t k_at = ring + 16 * lane, ks_at = ring + 2 * kQaCodes + kQ4Scales * g8 + 2 * t4;
  const uint32_t v_at = ring + kQaCodes + qa_value_off(2 * t4, g8 >> 1) + 8 * (g8 & 1);
  const uint32_t v_odd = ring + kQaCodes + qa_value_off(2 * t4 + 1, g8 >> 1) + 8 * (g8 & 1);
  const uint32_t vs_at = ring + 2 * kQaCodes + kQaScales + 2 * kQ4Scales * t4 + (g8 & 4);
  const uint8_t *k_from = pools.k + 16 * t4, *v_from = pools.v + 16 * t4;
  const uint32_t v_to = kQaCodes + qa_value_off(g8, t4);
  const int page_all = hkv * pg.page_rows;  // rows of all heads
  const bool whole_tiles = pg.page_rows % 16 == 0;
  // Known to be powers of two, these become shifts and additions on the pipe that
  // the conversions fill; as numbers they are multiplications on another.
  uint32_t code_bytes, scale_bytes, sixteen;
  asm volatile("mov.u32 %0, 64;\n\tmov.u32 %1, 8;\n\tmov.u32 %2, 16;"
               : "=r"(code_bytes), "=r"(scale_bytes), "=r"(sixteen));
  auto fetch = [&](uint32_t dst, bool any, const Entry& e) {
    ok = ok_next;
    ok_next = 0;
    if (any) {
      const bool good = e.row >= 0 && (uint32_t)e.page < (uint32_t)pg.n_pages;
      bad |= e.row >= 0 && !good;
      const int row = good ? e.page * page_all + e.row : -1;
      ok_next = __ballot_sync(0xffffffffu, good);
      const uint32_t k_to = dst + 16 * lane, v_at = dst + v_to, s_to = dst + 2 * kQaCodes + 8 * lane;
      if (whole_tiles && ok_next == 0xffffffffu) {  // 16 rows lie together
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const uint64_t at = (uint64_t)(uint32_t)(__shfl_sync(0xffffffffu, row, 16 * y) + g8) * code_bytes;
          const uint8_t *ks = k_from + at, *vs = v_from + at;
          asm volatile(
              "cp.async.cg.shared.global [%0], [%1], 16;\n\t"
              "cp.async.cg.shared.global [%0 + 512], [%1 + 512], 16;\n\t"
              "cp.async.cg.shared.global [%2], [%3], 16;\n\t"
              "cp.async.cg.shared.global [%2 + 512], [%3 + 512], 16;" ::"r"(k_to + 1024 * y),
              "l"(ks), "r"(v_at + 1024 * y), "l"(vs)
              : "memory");
        }
        const uint64_t at = (uint64_t)(uint32_t)row * scale_bytes;
        cp_async8(s_to, pools.k_scale + at);
        cp_async8(s_to + kQaScales, pools.v_scale + at);
      } else {
#pragma unroll
        for (int i = 0; i < kQaBlock / 8; ++i) {
          const int r = __shfl_sync(0xffffffffu, row, g8 + 8 * i);
          asm volatile(
              "{\n\t.reg .pred p;\n\tsetp.ge.s32 p, %4, 0;\n\t"
              "@p cp.async.cg.shared.global [%0], [%1], 16;\n\t"
              "@p cp.async.cg.shared.global [%2], [%3], 16;\n\t}" ::"r"(k_to + 512 * i),
              "l"(k_from + (uint64_t)(uint32_t)r * code_bytes), "r"(v_at + 512 * i),
              "l"(v_from + (uint64_t)(uint32_t)r * code_bytes), "r"(r)
              : "memory");
        }
        const uint64_t at = (uint64_t)(uint32_t)max(row, 0) * scale_bytes;
        cp_async8_fill(s_to, pools.k_scale + at, row >= 0);
        cp_async8_fill(s_to + kQaScales, pools.v_scale + at, row >= 0);
      }
    }
    cp_async_commit();
  };
  // Queries of an item: its lane takes elements 32 t4 .. of query g8 of group 0
  // (one group: every warp all of them) or of the warp's number.
  const int group = kRegs ? 0 : warp;
  Query4<T> raw[8];
  // Step ks of the products takes elements 32 t4 + 4 ks .. + 3 of query 8 nt + g8.
  // sc: what the sums of queries 8 nt + 2 t4 + e are multiplied by.
  uint2 qr[8];
  float sc[NT][2];
  auto load_queries = [&](const Cursor& c, const Item& x) {
    const int row0 = x.chunk * chunk_rows, rows = min(chunk_rows, min(c.w.fresh, pg.w) * G - row0);
    const int at = 8 * group + g8, r = row0 + at, t = c.w.first + r / G;
    const bool there = at < rows && t >= 0 && t < n;
    const T* from = q + ((size_t)(there ? t : 0) * hq + x.h * G + r % G) * kD + 32 * t4;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      raw[ks].x = {};
      if (there) raw[ks] = *reinterpret_cast<const Query4<T>*>(from + 4 * ks);
    }
  };
  auto take_queries = [&](int h) {
    if (!kRegs && warp >= NT) return;
    uint32_t top = 0;
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      const float4 y = raw[ks].get();
      const float x[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    }
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const int ex = min((int)(top >> 23), 253);
    float mul = __uint_as_float((uint32_t)(254 - ex) << 23);  // 2^-exponent
    // What the products, below 2^21 and multiples of 2^-34, become scores by.  Below 2^-100 every weight is 1, above
    // 2^100 the largest score's alone counts, whatever it is: held there, no score is an infinity, nor 0 times one.
    float back = kPatLog2e * rsqrtf((float)kD) * (pools.k_factor ? pools.k_factor[h] : 1.f) / mul;
    back = fminf(fmaxf(back, 0x1p-100f), 0x1p100f);
    if (top >= 0x7f800000u) mul = CUDART_NAN_F;  // not all are numbers: nor are its scores
    if constexpr (kRegs) {
      sc[0][0] = __shfl_sync(0xffffffffu, back, 8 * t4);
      sc[0][1] = __shfl_sync(0xffffffffu, back, 8 * t4 + 4);
    } else if (t4 == 0) {
      q_back[8 * warp + g8] = back;
    }
#pragma unroll
    for (int ks = 0; ks < 8; ++ks) {
      const float4 y = raw[ks].get(), z = make_float4(y.x * mul, y.y * mul, y.z * mul, y.w * mul);
      const uint2 hi = make_uint2(pack_f16(z.x, z.y), pack_f16(z.z, z.w));
      if constexpr (kRegs) {
        qr[ks] = hi;
      } else {
        qs[(warp * 8 + ks) * 32 + lane] = hi;
        if (kParts == 2) {
          const float2 a = unpack_f16(hi.x), b = unpack_f16(hi.y);
          qs[((NT + warp) * 8 + ks) * 32 + lane] =
              make_uint2(pack_f16(z.x - a.x, z.y - a.y), pack_f16(z.z - b.x, z.w - b.y));
        }
      }
    }
  };
  auto fill = [&](auto between) {
    Entry first[kQaStages];  // all table entries on their way before the first copies
    bool any[kQaStages];
#pragma unroll
    for (int st = 0; st < kQaStages; ++st) any[st] = look_up(first[st]);
    between();
#pragma unroll
    for (int st = 0; st < kQaStages; ++st) fetch(ring + st * kQaStage, any[st], first[st]);
  };
  start(rg.at, rg.b0);
  Cursor cur = rg.at;
  int ready = -1;  // the unit that the part begins at whose queries are taken: the first
  if (rg.b0 < rg.b1) {
    advance(cur, rg.b0, pg, G, chunk_rows, hkv);
    const Item x = item_at(cur, rg.b0);
    fill([&]() { load_queries(cur, x); });
    take_queries(x.h);
    ready = rg.b0;
  }

  int stage = 0;  // bytes to the stage at hand
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
        zero_rows<kQaThreads>(out, cur.w.first, n, hq, h * G, G, row0, rows);
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

    if (ready != seg) {
      load_queries(cur, item);
      take_queries(h);
    }
    if constexpr (!kRegs) {
      __syncthreads();
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) sc[nt][e] = q_back[8 * nt + 2 * t4 + e];
    }

    // Running state: reference and the lane's part of the sum of queries
    // 8 nt + 2 t4 + e; o[mt][nt][j] is dimension 16 g8 + 2 mt + (j >> 1) of
    // query 8 nt + 2 t4 + (j & 1).
    float m[NT][2], l[NT][2], o[8][NT][4];
    const int all_see = cur.w.len - (cur.w.fresh - 1 - row0 / G);  // rows that every query sees
    // The warp's blocks of the part.  A value's scale that is no number makes its
    // group's results so for the tokens that see its row, and a weight of 0 would
    // carry it to the others too: a warp whose sums are not numbers at the part's
    // end takes its blocks again and looks for them.
    auto take = [&](auto look) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        m[nt][0] = m[nt][1] = -3e38f;
        l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
        for (int mt = 0; mt < 8; ++mt) o[mt][nt][0] = o[mt][nt][1] = o[mt][nt][2] = o[mt][nt][3] = 0.f;
      }
      for (int u = warps_first<kQaWarps>(part0, warp); u < seg_end; u += kQaWarps) {
        cp_async_wait<kQaStages - 1>();
        __syncwarp();
        Entry next;  // of the block that will take this stage
        const bool any = look_up(next);
        const int base = (u - item.f0) * kQaBlock;
#pragma unroll 1
        for (int y0 = 0; y0 < 2; y0 += kTiles) {
          float c[kTiles][NT][4];
#pragma unroll
          for (int y = 0; y < kTiles; ++y)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) c[y][nt][0] = c[y][nt][1] = c[y][nt][2] = c[y][nt][3] = 0.f;
          {
            const uint32_t kt = k_at + stage + 16 * kQ4Row * y0, st = ks_at + stage + 16 * kQ4Scales * y0;
            uint4 w[2 * kTiles];      // rows g8, g8 + 8, ...
            __half2 s[2 * kTiles];
            w[0] = lds128<0>(kt);
            w[1] = lds128<8 * kQ4Row>(kt);
            s[0] = as_half2(q4_scales(lds16<0>(st)));
            s[1] = as_half2(q4_scales(lds16<8 * kQ4Scales>(st)));
            if constexpr (kTiles == 2) {
              w[2] = lds128<16 * kQ4Row>(kt);
              w[3] = lds128<24 * kQ4Row>(kt);
              s[2] = as_half2(q4_scales(lds16<16 * kQ4Scales>(st)));
              s[3] = as_half2(q4_scales(lds16<24 * kQ4Scales>(st)));
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              uint32_t p[2 * kTiles][4];
#pragma unroll
              for (int x = 0; x < 2 * kTiles; ++x) {
                q4_codes(i == 0 ? w[x].x : (i == 1 ? w[x].y : (i == 2 ? w[x].z : w[x].w)), p[x]);
                const __half2 f = i < 2 ? __low2half2(s[x]) : __high2half2(s[x]);
#pragma unroll
                for (int j = 0; j < 4; ++j) p[x][j] = mul_half2(p[x][j], f);
              }
#pragma unroll
              for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                  for (int part = 0; part < kParts; ++part) {
                    uint2 b;
                    if constexpr (kRegs)
                      b = qr[2 * i + j];
                    else
                      b = qs[((part * NT + nt) * 8 + 2 * i + j) * 32 + lane];
#pragma unroll
                    for (int y = 0; y < kTiles; ++y) {  // two sums that do not wait for one another
                      const uint32_t a[4] = {p[2 * y][2 * j], p[2 * y + 1][2 * j], p[2 * y][2 * j + 1],
                                             p[2 * y + 1][2 * j + 1]};
                      mma_f16(c[y][nt], a, b.x, b.y);
                    }
                  }
            }
          }
          if (ok != 0xffffffffu || base + kQaBlock > all_see) {  // some rows do not count for some queries
#pragma unroll
            for (int y = 0; y < kTiles; ++y)
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                  const int r = 16 * (y0 + y) + g8 + 8 * (j >> 1), x = 8 * nt + 2 * t4 + (j & 1);
                  const int sees = cur.w.len - (cur.w.fresh - 1 - (row0 + x) / G);
                  // times a factor of 2^-100 at least
                  if (!(ok >> r & 1u) || base + r >= sees) c[y][nt][j] = -CUDART_INF_F;
                }
          }
          // Scores over their references, in powers of two.  A product and a difference,
          // each rounded: fused, a huge score would exceed itself.
          float d[kTiles][NT][4];
          float most = -CUDART_INF_F;
#pragma unroll
          for (int y = 0; y < kTiles; ++y)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                c[y][nt][j] = __fmul_rn(c[y][nt][j], sc[nt][j & 1]);
                d[y][nt][j] = __fsub_rn(c[y][nt][j], m[nt][j & 1]);
              }
              most = max3(max3(most, d[y][nt][0], d[y][nt][1]), d[y][nt][2], d[y][nt][3]);
            }
          if (__any_sync(0xffffffffu, most > kQaLift + kQaSlack)) {  // rare once the references have settled
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                float mx = fmaxf(c[0][nt][e], c[0][nt][2 + e]);
#pragma unroll
                for (int y = 1; y < kTiles; ++y) mx = max3(mx, c[y][nt][e], c[y][nt][2 + e]);
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
                const float lifted = __fsub_rn(mx, kQaLift);  // 16 below where fp32's numbers are 16 apart
                mx = fmaxf(m[nt][e], __fsub_rn(mx, lifted) > kQaLift + kQaSlack ? mx : lifted);
                const float alpha = ex2_approx(m[nt][e] - mx);
                m[nt][e] = mx;
                l[nt][e] *= alpha;
#pragma unroll
                for (int y = 0; y < kTiles; ++y) {
                  d[y][nt][e] = __fsub_rn(c[y][nt][e], mx);
                  d[y][nt][2 + e] = __fsub_rn(c[y][nt][2 + e], mx);
                }
#pragma unroll
                for (int mt = 0; mt < 8; ++mt) {
                  o[mt][nt][e] *= alpha;
                  o[mt][nt][2 + e] *= alpha;
                }
              }
          }
#pragma unroll
          for (int y = 0; y < kTiles; ++y) {
            uint32_t p[kParts][NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              float z[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) {  // scores become weights
                z[j] = ex2_approx(d[y][nt][j]);
                l[nt][j & 1] += z[j];
              }
#pragma unroll
              for (int x = 0; x < 2; ++x) {
                const uint32_t hi = pack_f16(z[2 * x], z[2 * x + 1]);
                p[0][nt][x] = transpose8x8(hi);
                if (kParts == 2) {
                  const float2 t = unpack_f16(hi);
                  p[kParts - 1][nt][x] = transpose8x8(pack_f16(z[2 * x] - t.x, z[2 * x + 1] - t.y));
                }
              }
            }
            const uint32_t vt = v_at + stage + 16 * kQ4Row * (y0 + y), vo = v_odd + stage + 16 * kQ4Row * (y0 + y);
            const uint32_t st = vs_at + stage + 16 * kQ4Scales * (y0 + y);
            // scales of rows 2 t4, 2 t4 + 1 of the tile, and of those + 8
            uint32_t b[2] = {__byte_perm(lds32<0>(st), lds32<kQ4Scales>(st), pick),
                             __byte_perm(lds32<8 * kQ4Scales>(st), lds32<9 * kQ4Scales>(st), pick)};
            if constexpr (decltype(look)::value) {
              uint32_t which = 0;  // rows of the tile, of the lane's four
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if ((b[i >> 1] >> (8 * (i & 1)) & 0x7fu) == kQ4NaN) {
                  which |= 1u << (2 * t4 + 8 * (i >> 1) + (i & 1));
                  b[i >> 1] &= ~(0xffu << (8 * (i & 1)));
                }
              which |= __shfl_xor_sync(0xffffffffu, which, 1);
              which |= __shfl_xor_sync(0xffffffffu, which, 2);
              which &= ok >> (16 * (y0 + y));
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                  // of the tile's rows
                  const int sees = cur.w.len - (cur.w.fresh - 1 - (row0 + 8 * nt + 2 * t4 + e) / G) - base -
                                   16 * (y0 + y);
                  if (which & (sees >= 16 ? 0xffffu : (1u << max(sees, 0)) - 1u))
#pragma unroll
                    for (int mt = 0; mt < 8; ++mt) o[mt][nt][e] = o[mt][nt][2 + e] = CUDART_NAN_F;
                }
            }
            const __half2 f0 = as_half2(q4_scales(b[0])), f1 = as_half2(q4_scales(b[1]));
            const uint2 w[4] = {lds64<0>(vt), lds64<0>(vo), lds64<8 * kQ4Row>(vt), lds64<8 * kQ4Row>(vo)};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              // bytes of two rows' codes of one dimension: even dimensions, odd ones
              const uint32_t r0 = i ? w[0].y : w[0].x, r1 = i ? w[1].y : w[1].x, r2 = i ? w[2].y : w[2].x,
                             r3 = i ? w[3].y : w[3].x;
              uint32_t even0[4], odd0[4], even1[4], odd1[4];
              q4_codes((r0 & 0x0f0f0f0fu) | (r1 * sixteen & 0xf0f0f0f0u), even0);
              q4_codes((r0 >> 4 & 0x0f0f0f0fu) | (r1 & 0xf0f0f0f0u), odd0);
              q4_codes((r2 & 0x0f0f0f0fu) | (r3 * sixteen & 0xf0f0f0f0u), even1);
              q4_codes((r2 >> 4 & 0x0f0f0f0fu) | (r3 & 0xf0f0f0f0u), odd1);
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const uint32_t a[4] = {mul_half2(even0[j], f0), mul_half2(odd0[j], f0), mul_half2(even1[j], f1),
                                       mul_half2(odd1[j], f1)};
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                  for (int part = 0; part < kParts; ++part)
                    mma_f16(o[4 * i + j][nt], a, p[part][nt][0], p[part][nt][1]);
              }
            }
          }
        }
        __syncwarp();
        fetch(ring + stage, any, next);
        stage = kQaStage - stage;
      }
    };
    take(std::false_type());
    float none = 0.f;  // or a NaN, where a sum is one
#pragma unroll
    for (int mt = 0; mt < 8; ++mt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int j = 0; j < 4; ++j) none = fmaf(o[mt][nt][j], 0.f, none);
    if (__any_sync(0xffffffffu, none != 0.f)) {
      cp_async_wait<0>();  // no copy is on its way to the stages
      __syncwarp();
      start(cur, part0);
      stage = 0;
      fill([]() {});
      take(std::true_type());
    }
    // The warps' states of this item, merged in shared memory.
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float s = l[nt][e];
        s += __shfl_xor_sync(0xffffffffu, s, 4);
        s += __shfl_xor_sync(0xffffffffu, s, 8);
        s += __shfl_xor_sync(0xffffffffu, s, 16);
        if (g8 == 0) wml[warp * kRows + 8 * nt + 2 * t4 + e] = make_float2(m[nt][e], s);
      }
    __syncthreads();
    const int part = 2 * cta + (owns ? 1 : 0);
    const float vf = pools.v_factor ? pools.v_factor[h] : 1.f;
    // a thread for each warp's query: its factor, and, from the first warp's
    // thread, the query's maximum and sum over the warps
    for (int e = tid; e < kQaWarps * kRows; e += kQaThreads) {
      const int x = e % kRows;
      float M = -CUDART_INF_F;
#pragma unroll
      for (int w = 0; w < kQaWarps; ++w) M = fmaxf(M, wml[w * kRows + x].x);
      factor[e] = pat_weight(wml[e].x, M) * vf;
      if (e < rows) {
        float L = 0.f;
#pragma unroll
        for (int w = 0; w < kQaWarps; ++w) L = fmaf(wml[w * kRows + x].y, pat_weight(wml[w * kRows + x].x, M), L);
        if (whole)
          inv[x] = L == 0.f ? 0.f : 1.f / L;
        else
          part_ml[part * kRows + x] = make_float2(M, L);
      }
    }
    __syncthreads();
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int x = 8 * nt + 2 * t4 + e;
        const float a = factor[warp * kRows + x];
        float* w = wo + (warp * kRows + x) * kQaPitch + 16 * g8;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          store4(w + 4 * k, o[2 * k][nt][e] * a, o[2 * k][nt][2 + e] * a, o[2 * k + 1][nt][e] * a,
                 o[2 * k + 1][nt][2 + e] * a);
      }
    __syncthreads();
#pragma unroll 2
    for (int x = warp; x < rows; x += kQaWarps) {
      float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kQaWarps; ++w) {
        const float4 z = *reinterpret_cast<const float4*>(wo + (w * kRows + x) * kQaPitch + 4 * lane);
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
    seg = seg_end;
    if (seg < rg.b1) __syncthreads();  // the merge buffer (and the queries) are free again
  }
  cp_async_wait<0>();
  if (bad) record_error(err, kErrInput);
}

// -------------------------------------------------------------------- launch
static int q4_ctas(int part_rows) {
  int dev = 0, sms = 152;
  if (cudaGetDevice(&dev) == cudaSuccess) cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  const int ctas = qa_ctas(part_rows / 8) * sms;
  return ctas < kPatMaxCtas ? ctas : kPatMaxCtas;
}

// Query rows of a CTA's part, which share one read of the cache: at most 32, or
// 16 of fp32 (two parts of each).
static int q4_most_rows(DType dt) { return dt == kF32 ? 16 : 32; }
static int q4_part_rows(DType dt, const PageView& pages, int G) {
  const int rows = pages.w * G, most = q4_most_rows(dt), chunks = (rows + most - 1) / most;
  return ((rows + chunks - 1) / chunks + 7) / 8 * 8;
}

// Workspace: as paged_workspace_bytes says.
constexpr size_t kQaHead = 256, kQaDescs = kPatMaxCtas * sizeof(PartDesc);
size_t paged_q4_workspace_bytes(DType dt, const PageView& pages, int hq, int hkv) {
  const int rows = q4_part_rows(dt, pages, hq / hkv);
  return kQaHead + kQaDescs + (size_t)2 * q4_ctas(rows) * rows * (sizeof(float2) + kD * sizeof(float));
}

cudaError_t launch_paged_attention_q4(DType dt, const PageView& view, const void* q, const Q4View& pools, void* out,
                                      int n, int hq, int hkv, void* ws, cudaStream_t st) {
  PageView pages = view;
  uint32_t* err = static_cast<uint32_t*>(ws);
  const int rows = pages.w * (hq / hkv), part_rows = q4_part_rows(dt, pages, hq / hkv), most = q4_most_rows(dt);
  const int chunks = (rows + most - 1) / most, chunk_rows = (rows + chunks - 1) / chunks, ctas = q4_ctas(part_rows);
  const long long items = (long long)pages.n_seqs * hkv * chunks;
  pages.block_shift = kQaBlockShift;
  // Blocks that an item's own costs take: 6 / 12 / 18 / 24 make 58.4 / 55.7 / 54.7 / 55.5 us of 32 sessions of 1,000 to
  // 53,600 rows, 27.7 / 27.1 / 27.9 / 28.5 of 64 of 2,000, 15.7 / 15.6 / 15.6 / 16.7 of five tokens each of eight.
  pages.item_units = 12;
  // And those that splitting one takes: 0 and 10 as 20; 40 makes 11.9 us and not 8.3 of one session of 1,000 rows, 30.7
  // and not 27.2 of 64 of 2,000.
  int split = 20;
  // Tables of at most eight blocks: their items stay whole, which saves the second launch (64 sessions of 256 rows
  // 9.1 us, 11.2 split; up to 32 blocks one of 1,000 rows would: 11.2, 8.3 split).
  const long long longest = ((long long)pages.max_pages * pages.page_rows + kQaBlock - 1) / kQaBlock;
  const int mode = longest <= 8 ? kWholeItems : (items <= ctas ? kDescByItem : kDescByCta);
  if (mode == kWholeItems) split = 1 << 30;
  const int descs = items <= ctas ? (int)items : ctas;
  uint8_t* at = static_cast<uint8_t*>(ws) + kQaHead;
  PartDesc* desc = reinterpret_cast<PartDesc*>(at);
  float2* part_ml = reinterpret_cast<float2*>(at + kQaDescs);
  float* part_o = reinterpret_cast<float*>(part_ml + (size_t)2 * ctas * part_rows);
  cudaError_t e = cudaSuccess;
  auto run = [&](auto zero, auto width) {
    typedef decltype(zero) T;
    constexpr int NT = decltype(width)::value, kParts = std::is_same<T, float>::value ? 2 : 1;
    static_assert(fits_sm(qa_smem(NT, kParts), qa_ctas(NT)), "qa_ctas per SM");
    TimingScope ts("paged_attention_q4", st);
    auto kern = k_paged_q4<T, NT>;
    const int smem = qa_smem(NT, kParts);
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return;
    e = launch_after(kern, dim3(ctas), kQaThreads, smem, st, pages, pools, static_cast<const T*>(q),
                     static_cast<T*>(out), n, hq, hkv, mode, split, chunks, chunk_rows, desc, part_ml, part_o, err);
  };
  if (dt == kF32)
    part_rows == 8 ? run(float(), std::integral_constant<int, 1>()) : run(float(), std::integral_constant<int, 2>());
  else if (part_rows <= 16)
    part_rows == 8 ? run(__nv_bfloat16(), std::integral_constant<int, 1>())
                   : run(__nv_bfloat16(), std::integral_constant<int, 2>());
  else
    part_rows == 24 ? run(__nv_bfloat16(), std::integral_constant<int, 3>())
                    : run(__nv_bfloat16(), std::integral_constant<int, 4>());
  if (e != cudaSuccess || (e = cudaGetLastError()) != cudaSuccess) return e;
  if (mode == kWholeItems) return cudaSuccess;
  e = launch_paged_merge(dt, pages, out, n, hq, hkv, chunks, chunk_rows, part_rows, mode == kDescByItem, descs, desc,
                         part_ml, part_o, st);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace stl
