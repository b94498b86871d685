// Page tables, lengths and places of a serving step.
#include "kernels.cuh"

namespace stl {

// All of a step in one launch of one cluster.  Each CTA sums over all sessions
// for itself, kStepThreads of them at a time, a thread a session; the entries
// to move are then dealt out flat, to all threads of the cluster, which find
// an entry's session among the sums in shared memory.  Two waits of the whole
// cluster separate what reads the state before from what changes it: pages that
// go back are on the free list before any is taken, and lengths are written
// when no CTA reads the old ones.  Latency bounds it (lengths, table, free list,
// four sums, two waits): 64 sessions with five drafts each 4.8 us; CTAs of 512
// threads 6.1, of 1,024 10.3; four CTAs are as fast and take 17.7 for the 256
// sessions below.
constexpr int kStepThreads = 256, kStepCtas = 8;
// Places of more tokens than this are found by a second kernel on the whole
// chip: 226,000 tokens of 256 sessions and their 16,000 pages 10.7 us so, 34 in
// the cluster (0.1 us for each 1,000 of them).
constexpr int kStepSlots = 16384;

__device__ __forceinline__ void cluster_wait_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Two sums over the threads up to this one, and over all of them (*total).
// Sums stop at 2^31 - 1, so that they keep their order however much is asked
// for.  Whole CTA; calls take turns with two buffers.
struct Sums {
  int a, b;
};
__device__ __forceinline__ int add_most(int x, int y) { return (int)min((uint32_t)x + (uint32_t)y, 0x7fffffffu); }
__device__ __forceinline__ Sums scan(Sums x, Sums* warp_sums, Sums* total) {
  constexpr int kWarps = kStepThreads / 32;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int ya = __shfl_up_sync(0xffffffffu, x.a, o), yb = __shfl_up_sync(0xffffffffu, x.b, o);
    if (lane >= o) {
      x.a = add_most(x.a, ya);
      x.b = add_most(x.b, yb);
    }
  }
  if (lane == 31) warp_sums[warp] = x;
  __syncthreads();
  Sums before = {0, 0}, all = {0, 0};
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    const Sums y = warp_sums[w];
    if (w == warp) before = all;
    all.a = add_most(all.a, y.a);
    all.b = add_most(all.b, y.b);
  }
  *total = all;
  return {add_most(before.a, x.a), add_most(before.b, x.b)};
}

// The last of the kStepThreads sessions whose entries begin at or before j.
__device__ __forceinline__ int session_of(const int* start, int j) {
  int lo = 0;
#pragma unroll
  for (int step = kStepThreads / 2; step > 0; step >>= 1)
    if (start[lo + step] <= j) lo += step;
  return lo;
}

__global__ void __cluster_dims__(kStepCtas, 1, 1) __launch_bounds__(kStepThreads)
    k_pages_step(const __grid_constant__ StepView s) {
  __shared__ int start[kStepThreads], tok_start[kStepThreads], kept_of[kStepThreads], keep_of[kStepThreads];
  __shared__ Sums sums[2][kStepThreads / 32];
  pdl_trigger();
  pdl_wait();
  const int tid = threadIdx.x, rank = blockIdx.x, flat = rank * kStepThreads + tid;
  constexpr int kAll = kStepCtas * kStepThreads, kAtOnce = 4;  // entries that a thread moves at a time
  const int rows_max = s.max_pages * s.page_rows, pr = s.page_rows;
  const int n0 = max(0, min(*s.n_free, s.n_pages));
  int have = 0, keep = 0, fresh = 0, held = 0, kept = 0;
  auto load = [&](int s0) {
    have = keep = fresh = 0;
    const int i = s0 + tid;
    if (i < s.n_seqs) {
      have = max(0, min(s.len[i], rows_max));
      keep = s.keep ? max(0, min(s.keep[i], have)) : have;
      fresh = max(0, s.fresh[i]);
    }
    held = have / pr + (have % pr != 0);
    kept = keep / pr + (keep % pr != 0);
  };
  // Pages past the rows that stay go on top of the free ones.  The sums of pages
  // are below 2^31: a table's entries are.
  int back = 0;
  Sums total;
  for (int s0 = 0; s0 < s.n_seqs; s0 += kStepThreads) {
    load(s0);
    const int mine = held - kept;
    start[tid] = scan({mine, 0}, sums[0], &total).a - mine;
    kept_of[tid] = kept;
    __syncthreads();
    for (uint32_t j0 = flat; j0 < (uint32_t)total.a; j0 += kAtOnce * kAll) {
      int page[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const uint32_t j = j0 + i * kAll;
        if (j >= (uint32_t)total.a) break;
        const int b = session_of(start, j);
        page[i] = s.table[(size_t)(s0 + b) * s.max_pages + kept_of[b] + j - start[b]];
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const uint32_t j = j0 + i * kAll;
        const long long to = (long long)n0 + back + j;
        if (j < (uint32_t)total.a && to < s.n_pages) s.free_pages[to] = page[i];
      }
    }
    back += total.a;
    if (s0 + kStepThreads < s.n_seqs) __syncthreads();
  }
  cluster_wait_all();
  const int n_free = (int)min((long long)s.n_pages, (long long)n0 + back);

  // who is served, and what it gets
  Sums asked = {0, 0};       // pages and tokens asked for by the sessions before
  int taken = 0, given = 0;  // what those got
  int new_len = 0;
  if (rank == 0 && tid == 0) s.cu[0] = 0;
  for (int s0 = 0; s0 < s.n_seqs; s0 += kStepThreads) {
    if (s.n_seqs > kStepThreads) load(s0);
    const bool fits = fresh <= rows_max - keep;
    const int rows = fits ? keep + fresh : keep, want = rows / pr + (rows % pr != 0) - kept;
    const int pages_to = add_most(asked.a, scan({want, 0}, sums[1], &total).a);
    asked.a = add_most(asked.a, total.a);
    const bool may = fits && (want == 0 || pages_to <= n_free);
    const int tokens_to = add_most(asked.b, scan({0, may ? fresh : 0}, sums[0], &total).b);
    asked.b = add_most(asked.b, total.b);
    // a sum that stopped is too much for any step
    const bool served = may && (fresh == 0 || (tokens_to <= s.n_tokens && tokens_to < 0x7fffffff));
    const int pages = served ? want : 0, got = served ? fresh : 0;
    const Sums to = scan({pages, got}, sums[1], &total);
    const int my_pages = to.a - pages, my_tokens = to.b - got;
    start[tid] = my_pages;
    tok_start[tid] = my_tokens;
    kept_of[tid] = kept;
    keep_of[tid] = keep;
    new_len = keep + got;
    if (rank == 0 && s0 + tid < s.n_seqs) s.cu[s0 + tid + 1] = given + to.b;
    __syncthreads();
    const int top = n_free - 1 - taken;
    for (uint32_t j0 = flat; j0 < (uint32_t)total.a; j0 += kAtOnce * kAll) {
      int page[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i)
        if (j0 + i * kAll < (uint32_t)total.a) page[i] = s.free_pages[top - (int)(j0 + i * kAll)];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        const uint32_t j = j0 + i * kAll;
        if (j >= (uint32_t)total.a) break;
        const int b = session_of(start, j);
        s.table[(size_t)(s0 + b) * s.max_pages + kept_of[b] + j - start[b]] = page[i];
      }
    }
    if (s.slot)
      for (uint32_t j = flat; j < (uint32_t)total.b; j += kAll) {
        const int b = session_of(tok_start, j), row = keep_of[b] + j - tok_start[b], i = row / pr;
        const int page = i < kept_of[b] ? s.table[(size_t)(s0 + b) * s.max_pages + i]
                                        : s.free_pages[top - (start[b] + i - kept_of[b])];
        s.slot[given + j] = page >= 0 && page < s.n_pages ? page * pr + (row - i * pr) : -1;
      }
    taken += total.a;
    given += total.b;
    if (s0 + kStepThreads < s.n_seqs) __syncthreads();
  }
  if (s.slot)
    for (uint32_t j = given + flat; j < (uint32_t)s.n_tokens; j += kAll) s.slot[j] = -1;
  cluster_wait_all();
  if (rank > 0) return;
  if (tid == 0) *s.n_free = n_free - taken;
  const int last = (s.n_seqs - 1) / kStepThreads * kStepThreads;  // the sessions that the threads still hold
  for (int i = tid; i < last; i += kStepThreads) {
    const int was = max(0, min(s.len[i], rows_max)), stays = s.keep ? max(0, min(s.keep[i], was)) : was;
    s.len[i] = stays + (s.cu[i + 1] - s.cu[i]);
  }
  if (last + tid < s.n_seqs) s.len[last + tid] = new_len;
}

// The places of new tokens, as k_pages_step writes them: a token to a thread,
// its session found by halves in cu.
__global__ void __launch_bounds__(256) k_step_slots(const __grid_constant__ StepView s) {
  pdl_trigger();
  pdl_wait();
  if (blockIdx.x * 256u + threadIdx.x >= (uint32_t)s.n_tokens) return;
  const int t = blockIdx.x * 256 + threadIdx.x;
  int slot = -1;
  if (t < s.cu[s.n_seqs]) {
    int lo = 0, hi = s.n_seqs;  // cu[lo] <= t < cu[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s.cu[mid] <= t)
        lo = mid;
      else
        hi = mid;
    }
    const int row = s.len[lo] - (s.cu[lo + 1] - t), i = row / s.page_rows;
    const int page = s.table[(size_t)lo * s.max_pages + i];
    if (page >= 0 && page < s.n_pages) slot = page * s.page_rows + (row - i * s.page_rows);
  }
  s.slot[t] = slot;
}

cudaError_t launch_pages_step(const StepView& step, cudaStream_t st) {
  StepView s = step;
  const bool apart = s.slot && s.n_tokens > kStepSlots;
  cudaError_t e;
  {
    TimingScope ts("pages_step", st);
    if (apart) s.slot = nullptr;
    e = launch_after(k_pages_step, dim3(kStepCtas), kStepThreads, 0, st, s);
    if (e != cudaSuccess || (e = cudaGetLastError()) != cudaSuccess || !apart) return e;
  }
  TimingScope ts("step_slots", st);
  s.slot = step.slot;
  e = launch_after(k_step_slots, dim3(((unsigned)s.n_tokens + 255) / 256), 256, 0, st, s);
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace stl
