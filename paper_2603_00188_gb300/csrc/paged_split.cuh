// How attention over paged caches is divided among CTAs.
//
// Work is divided by what the sessions hold when the kernel runs.  An item is
// (session, KV head, chunk of query rows); its cache is cut into blocks of
// 16 (or 32) rows.  An item counts for its blocks and for some units before them that stand
// for its own costs (queries, merge: launch_paged_attention gives their number);
// the units of all items, laid end to end, are cut into equal ranges, one per CTA.  A CTA
// computes the parts of the few items that its range meets: an item whose
// blocks lie inside one range is finished there, the parts of others are merged
// by a second kernel.
#pragma once

#include <type_traits>

#include "kernels.cuh"
#include "ptx.cuh"

namespace stl {

constexpr float kPatLog2e = 1.4426950408889634f;

__device__ __forceinline__ float pat_weight(float a, float m) { return a == -CUDART_INF_F ? 0.f : exp2f(a - m); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// The 8 x 8 matrix of 16-bit values held two to a lane, transposed.
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ void store4(float* p, float x, float y, float z, float w) {
  *reinterpret_cast<float4*>(p) = make_float4(x, y, z, w);
}
__device__ __forceinline__ void store4(__nv_bfloat16* p, float x, float y, float z, float w) {
  *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(x, y), pack_bf16(z, w));
}

// ---------------------------------------------------------------- the split

// Whether any item can be split, and whether what is left for the second
// kernel is described by CTA or by item.
enum SplitMode { kWholeItems = 0, kDescByCta = 1, kDescByItem = 2 };

// What a session asks for.
struct SeqWork {
  int first, fresh;  // its packed tokens: first .. first + fresh
  int len;           // cached rows
  int blocks;        // blocks of one item; none: its output is zeros
  int units;         // what the item counts for: these after pg.item_units
  int chunks;        // items of one KV head
};
__device__ __forceinline__ SeqWork seq_work(const PageView& pg, int first, int fresh, int len, int G, int chunk_rows) {
  SeqWork w;
  w.first = first;
  w.fresh = fresh;
  w.len = max(0, min(len, pg.max_pages * pg.page_rows));
  w.blocks = (int)(((uint32_t)w.len + (1u << pg.block_shift) - 1u) >> pg.block_shift);  // len may be 2^31 - 1
  w.units = pg.item_units + w.blocks;
  const int rows = max(0, min(fresh, pg.w)) * G;
  w.chunks = rows <= chunk_rows ? (rows > 0 ? 1 : 0) : (rows + chunk_rows - 1) / chunk_rows;
  return w;
}
__device__ __forceinline__ SeqWork seq_work(const PageView& pg, int s, int len, int G, int chunk_rows) {
  const int first = pg.cu ? pg.cu[s] : s * pg.w;
  return seq_work(pg, first, pg.cu ? pg.cu[s + 1] - first : pg.w, len, G, chunk_rows);
}

// A position in the sequence of all units: session s begins at unit `base`.
// Unit numbers fit an int (the call's checks).
struct Cursor {
  int base, s;
  SeqWork w;
  __device__ __forceinline__ int cost(int hkv) const { return w.units * w.chunks * hkv; }
};

// A CTA's range of units and where it starts.  All units are dealt to `ctas`
// CTAs in ranges of `quota`, the first `extra` one more.
struct Range {
  int b0, b1;
  int quota, ctas, extra;
  Cursor at;
  __device__ __forceinline__ int start(int c) const { return c * quota + min(c, extra); }
  __device__ __forceinline__ int cta_of(int b) const {
    const int wide = extra * (quota + 1);
    return b < wide ? b / (quota + 1) : extra + (b - wide) / quota;
  }
};

// Moves on to the session of unit b.
__device__ __forceinline__ void advance(Cursor& c, int b, const PageView& pg, int G, int chunk_rows, int hkv) {
  while (b >= c.base + c.cost(hkv)) {
    c.base += c.cost(hkv);
    ++c.s;
    c.w = seq_work(pg, c.s, pg.len[c.s], G, chunk_rows);
  }
}

// An item that a range meets.
struct Item {
  int h, chunk;
  int i0, f0, i1;  // units: its first, its first block's, its end
};
__device__ __forceinline__ Item item_at(const Cursor& c, int u) {
  const int units = c.w.units, i = (u - c.base) / units;
  Item x;
  x.h = c.w.chunks == 1 ? i : i / c.w.chunks;
  x.chunk = i - x.h * c.w.chunks;
  x.i0 = c.base + i * units;
  x.i1 = x.i0 + units;
  x.f0 = x.i1 - c.w.blocks;
  return x;
}

// The costs are summed over the sessions, and the range's first session found
// by the thread that holds it.  Whole CTA; least: the fewest units that make a
// CTA's range.  split: the units that splitting an item costs beside its parts
// (writing them, a second part in the CTA, the merge).  Where CTAs with whole
// items, each the CTA's where its first unit falls, are sure to take no longer
// than the even ranges and this, the range's ends move on to the next item's
// start: of 16-bit rows, 64 sessions of 2,000 on 304 CTAs take 45 us so and 53
// split; 8 of 256 rows 7.8 and 8.2; 8 of 500 rows, a tenth of the CTAs, 11.2 and 9.0.
// (4-bit rows: see their launch.)
template <int THREADS>
struct RangeScratch {
  int warp_sum[THREADS / 32], warp_most[THREADS / 32], warp_least[THREADS / 32];
  Cursor at;
};
template <int THREADS>
__device__ Range find_range(const PageView& pg, int G, int chunk_rows, int hkv, int least, int split, uint32_t* err,
                            RangeScratch<THREADS>* scratch) {
  constexpr int kWarps = THREADS / 32, kAtOnce = 4;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per = (pg.n_seqs + THREADS - 1) / THREADS, s0 = min(pg.n_seqs, tid * per), s1 = min(pg.n_seqs, s0 + per);
  int mine = 0, longest = 0, shortest = 0x7fffffff;
  Cursor c;  // of the thread's last session, and its only one where there are no more than threads
  for (int s = s0; s < s1; s += kAtOnce) {
    int asked[kAtOnce], first[kAtOnce + 1];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) asked[i] = s + i < s1 ? pg.len[s + i] : 0;
#pragma unroll
    for (int i = 0; i <= kAtOnce; ++i) first[i] = pg.cu ? pg.cu[min(s + i, s1)] : (s + i) * pg.w;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      if (s + i >= s1) break;
      c.w = seq_work(pg, first[i], first[i + 1] - first[i], asked[i], G, chunk_rows);
      mine += c.cost(hkv);
      if (c.w.chunks > 0) {
        longest = max(longest, c.w.units);
        shortest = min(shortest, c.w.units);
      }
      if (blockIdx.x == 0 && c.w.len != asked[i]) record_error(err, kErrInput);
    }
  }
  int incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += x;
  }
  longest = __reduce_max_sync(0xffffffffu, longest);
  shortest = __reduce_min_sync(0xffffffffu, shortest);
  if (lane == 31) {
    scratch->warp_sum[warp] = incl;
    scratch->warp_most[warp] = longest;
    scratch->warp_least[warp] = shortest;
  }
  __syncthreads();
  int before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const int x = scratch->warp_sum[w];
    if (w < warp) before += x;
    total += x;
    longest = max(longest, scratch->warp_most[w]);
    shortest = min(shortest, scratch->warp_least[w]);
  }
  Range r;
  r.ctas = min((int)gridDim.x, total / least + (total % least != 0));
  if ((int)blockIdx.x >= r.ctas) return r;  // the same for every thread
  r.quota = total / r.ctas;
  r.extra = total - r.quota * r.ctas;
  r.b0 = r.start(blockIdx.x);
  r.b1 = r.start(blockIdx.x + 1);
  incl += before;
  if (mine > 0 && incl - mine <= r.b0 && r.b0 < incl) {
    c.base = incl - mine;
    c.s = s0;
    if (per > 1) {
      for (c.w = seq_work(pg, s0, pg.len[s0], G, chunk_rows); r.b0 >= c.base + c.cost(hkv);) {
        c.base += c.cost(hkv);
        ++c.s;
        c.w = seq_work(pg, c.s, pg.len[c.s], G, chunk_rows);
      }
    }
    scratch->at = c;
  }
  __syncthreads();
  r.at = scratch->at;
  // a range of `most` units holds at most most / shortest (rounded up) items' starts
  const int most = r.quota + (r.extra > 0);
  const long long whole = min((long long)most + longest, (long long)(most / shortest + (most % shortest != 0)) * longest);
  if (whole - r.quota <= split) {
    c = r.at;
    advance(c, r.b1 - 1, pg, G, chunk_rows, hkv);
    const Item first = item_at(r.at, r.b0);
    if (first.i0 < r.b0) r.b0 = first.i1;
    r.b1 = item_at(c, r.b1 - 1).i1;
  }
  return r;
}

// Which part of which item is left for the second kernel: `desc` has an entry
// for each item, or for each CTA where those are fewer, of the item that
// starts there.
struct PartDesc {
  int item;     // (session * hkv + head) * chunks of a full session + chunk; -1: nothing to merge
  int c0, c1;   // CTAs with a part: slot 2 c0 + 1, then slots 2 c for c = c0 + 1 .. c1
  int pad;
};

constexpr int kPatMaxCtas = 1024;

__device__ __forceinline__ void cp_async16_fill(uint32_t dst, const void* src, bool valid) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(valid ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Whether `ctas` CTAs of so much dynamic shared memory share an SM's 228 KB
// (1 KB of it each is reserved).
__host__ __device__ constexpr bool fits_sm(int smem, int ctas) {
  return ctas * ((smem + 127) / 128 * 128 + 1024) <= 228 * 1024;
}

// The rows of a warp's blocks, one block after the other.  The block of unit u
// is warp u % WARPS's.
template <int WARPS>
__device__ __forceinline__ int warps_first(int u, int warp) { return u + ((warp - u) & (WARPS - 1)); }
template <int WARPS, int BLOCK>
struct RowFinder {
  Cursor at;
  int end;         // of the CTA's range
  int u, f0, i1;   // the warp's next block, and the first block and the end of the item that it is sought in
  int head;

  __device__ __forceinline__ RowFinder(const Range& r) : end(r.b1), head(0) { start(r.at, r.b0); }

  // The next block is the first at or after unit `from`, of c's session or a later one.
  __device__ __forceinline__ void start(const Cursor& c, int from) {
    at = c;
    u = f0 = i1 = from;
  }

  // Moves on to the item of the warp's next block; false past the range.
  __device__ __forceinline__ bool seek(const PageView& pg, int warp, int G, int chunk_rows, int hkv) {
    while (u >= i1) {
      if (i1 >= end) return false;
      advance(at, i1, pg, G, chunk_rows, hkv);
      const Item x = item_at(at, i1);
      u = warps_first<WARPS>(max(i1, x.f0), warp);
      f0 = x.f0;
      i1 = x.i1;
      head = x.h;
    }
    return u < end;
  }

  // Lane % BLOCK's row of the warp's next block, as a row of 128 elements of the
  // pools seen as [rows][128]; -1 where it does not count, -2 past the range.
  __device__ __forceinline__ int next(const PageView& pg, int warp, int G, int chunk_rows, int hkv, uint32_t* err) {
    if (!seek(pg, warp, G, chunk_rows, hkv)) return -2;
    const int j = (u - f0) * BLOCK + (threadIdx.x & (BLOCK - 1));
    u += WARPS;
    if (j >= at.w.len) return -1;
    const int i = pg.page_shift >= 0 ? j >> pg.page_shift : j / pg.page_rows;
    const int page = pg.table[(size_t)at.s * pg.max_pages + i];
    if (page < 0 || page >= pg.n_pages) {
      record_error(err, kErrInput);
      return -1;
    }
    return (page * pg.page_rows + (j - i * pg.page_rows)) * hkv + head;
  }
};

// Query rows row0 .. row0 + rows of a session's KV head, whose first query head
// is g0, that see nothing.
template <int THREADS, typename T>
__device__ __forceinline__ void zero_rows(T* out, int first, int n, int hq, int g0, int G, int row0, int rows) {
  for (int e = threadIdx.x; e < rows * (kD / 4); e += THREADS) {
    const int r = row0 + e / (kD / 4), t = first + r / G;
    if (t >= 0 && t < n) store4(out + ((size_t)t * hq + g0 + r % G) * kD + 4 * (e % (kD / 4)), 0.f, 0.f, 0.f, 0.f);
  }
}

// The second kernel (k_paged_merge): `descs` descriptors, `chunk_rows` query
// rows each, of parts of part_rows.
cudaError_t launch_paged_merge(DType dt, const PageView& pages, void* out, int n, int hq, int hkv, int chunks,
                               int chunk_rows, int part_rows, bool by_item, int descs, const PartDesc* desc,
                               const float2* part_ml, const float* part_o, cudaStream_t st);

}  // namespace stl
