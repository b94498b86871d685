// What the kernels over paged caches share: rows' places, elements by eights.
#pragma once

#include "kernels.cuh"

namespace stl {

// Eight consecutive elements as they are in memory.
template <typename T>
struct Vec8;
template <>
struct Vec8<__nv_bfloat16> {
  uint4 u;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { u = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = u; }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ void set(const float (&f)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    u = make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <>
struct Vec8<float> {
  float4 x, y;
  __device__ __forceinline__ void load(const float* p) {
    x = reinterpret_cast<const float4*>(p)[0];
    y = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void store(float* p) const {
    reinterpret_cast<float4*>(p)[0] = x;
    reinterpret_cast<float4*>(p)[1] = y;
  }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    f[0] = x.x; f[1] = x.y; f[2] = x.z; f[3] = x.w;
    f[4] = y.x; f[5] = y.y; f[6] = y.z; f[7] = y.w;
  }
  __device__ __forceinline__ void set(const float (&f)[8]) {
    x = make_float4(f[0], f[1], f[2], f[3]);
    y = make_float4(f[4], f[5], f[6], f[7]);
  }
};

// Slot (page * page_rows + row of the page) of row r of sequence s, or -1.
__device__ __forceinline__ int page_slot(const PageView& pg, int s, int r) {
  if (r < 0 || r >= pg.max_pages * pg.page_rows) return -1;
  const int i = pg.page_shift >= 0 ? r >> pg.page_shift : r / pg.page_rows, page = pg.table[(size_t)s * pg.max_pages + i];
  return page >= 0 && page < pg.n_pages ? page * pg.page_rows + (r - i * pg.page_rows) : -1;
}

// The slot of packed new token t, which is not padding, or -1.  A whole warp
// calls it; 32 sequences are compared at a time, so that up to 32 take two
// memory latencies: their cu and len, then the table.
__device__ __forceinline__ int token_slot(const PageView& pg, int t) {
  if (!pg.cu) {
    const int s = t / pg.w;
    return s < pg.n_seqs ? page_slot(pg, s, pg.len[s] - ((s + 1) * pg.w - t)) : -1;
  }
  const int lane = threadIdx.x & 31;
  int lo = 0, count = pg.n_seqs;  // cu[lo] <= t, and the sequence is one of the `count` from lo on
  while (count > 32) {
    const int step = (count + 31) / 32, i = lane * step;
    const uint32_t le = __ballot_sync(0xffffffffu, i < count && pg.cu[lo + i] <= t);
    const int k = le ? 31 - __clz(le) : 0;
    lo += k * step;
    count = min(step, count - k * step);
  }
  const int mine = lo + min(lane, count - 1), first = pg.cu[mine], next = pg.cu[mine + 1], len = pg.len[mine];
  const uint32_t le = __ballot_sync(0xffffffffu, lane < count && first <= t);
  const int k = le ? 31 - __clz(le) : 0;
  const int row = __shfl_sync(0xffffffffu, len, k) - (__shfl_sync(0xffffffffu, next, k) - t);
  return page_slot(pg, lo + k, row);
}

// Page and row of the page of row r of sequence s; page -1 where there is none.
struct Place {
  int page, row;
};
__device__ __forceinline__ Place page_place(const PageView& pg, int s, int r) {
  if (r < 0 || r >= pg.max_pages * pg.page_rows) return {-1, 0};
  const int i = pg.page_shift >= 0 ? r >> pg.page_shift : r / pg.page_rows;
  const int page = pg.table[(size_t)s * pg.max_pages + i];
  return {page >= 0 && page < pg.n_pages ? page : -1, r - i * pg.page_rows};
}

// token_slot's page and row.
__device__ __forceinline__ Place token_place(const PageView& pg, int t) {
  const int slot = token_slot(pg, t);
  if (slot < 0) return {-1, 0};
  const int page = pg.page_shift >= 0 ? slot >> pg.page_shift : slot / pg.page_rows;
  return {page, slot - page * pg.page_rows};
}

// The same by a thread for itself: the sequence is found by halves.
__device__ __forceinline__ Place thread_token_place(const PageView& pg, int t) {
  if (!pg.cu) {
    const int s = t / pg.w;
    if (s >= pg.n_seqs) return {-1, 0};
    return page_place(pg, s, pg.len[s] - ((s + 1) * pg.w - t));
  }
  int lo = 0, hi = pg.n_seqs;  // cu[lo] <= t < cu[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (pg.cu[mid] <= t)
      lo = mid;
    else
      hi = mid;
  }
  return page_place(pg, lo, pg.len[lo] - (pg.cu[lo + 1] - t));
}

}  // namespace stl
