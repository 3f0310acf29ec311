// Pages of a cache pool: tables, reference counts and page copies (gfx950).
//
// The sequences that answer over one blended context keep the rows of their
// own in pages of a pool.  Slot s holds len[s] rows; row r is row r %
// page_rows of page table[s][r / page_rows]; ref[p] counts the table entries
// that hold page p, and a page nobody holds is free.  Only the entries below
// ceil(len / page_rows) mean anything.  What is decided (which page, which
// row) follows from the tables alone: free pages are taken from the lowest
// number up, slots in order, so equal inputs give equal tables; the counts
// are sums of integers, whose order does not matter.  All of it stays on the
// device, so a serving step needs no copy to the host and can be captured.
//
// Tables and counts are small (a pool of 64k pages has 256 KB of counts) and
// bound by latency: the steps that number pages run in one workgroup, whose
// barriers are cheaper than launches: rows for 12 slots in a pool of 256 pages
// 7.4 us, a pool of 2,048 pages renumbered in 5.7.  Page copies are bound by HBM.
#include "bf16_util.h"
#include "kvc_internal.h"

namespace kvc {
namespace {

__device__ __forceinline__ int rows_of(const PageTables& P, int s) {
  return min(max(P.len[s], 0), P.max_pages << P.page_shift);
}
__device__ __forceinline__ int pages_for(const PageTables& P, int rows) {
  return (int)(((unsigned)rows + ((1u << P.page_shift) - 1)) >> P.page_shift);
}
__device__ __forceinline__ bool is_page(const PageTables& P, int p) { return p >= 0 && p < P.n_pages; }
__device__ __forceinline__ int32_t* row_of(const PageTables& P, int s) {
  return P.table + (size_t)s * P.max_pages;
}

// One workgroup per slot.
constexpr int kTableThreads = 256;

__global__ __launch_bounds__(kTableThreads) void pages_trim_kernel(const PageTables P, const int32_t* __restrict__ keep) {
  const int s = blockIdx.x;
  const int have = rows_of(P, s), k = keep[s];
  if (k < 0 || k >= have) return;
  for (int c = pages_for(P, k) + threadIdx.x; c < pages_for(P, have); c += kTableThreads) {
    const int p = row_of(P, s)[c];
    if (is_page(P, p)) atomicSub(P.ref + p, 1);
  }
  __syncthreads();  // every thread has read the length
  if (threadIdx.x == 0) P.len[s] = k;
}

// What a slot continues is read before any table changes: the first launch
// lets go of the slots' own pages and puts their new tables aside (a length
// of -1: nothing to do), the second puts them in place.
__global__ __launch_bounds__(kTableThreads) void pages_fork_take_kernel(const PageTables P, const int32_t* __restrict__ src_of,
                                                                        int32_t* __restrict__ new_len,
                                                                        int32_t* __restrict__ new_table) {
  const int s = blockIdx.x, from = src_of[s];
  const bool fork = from >= 0 && from < P.n_slots && from != s;
  if (threadIdx.x == 0) new_len[s] = fork ? rows_of(P, from) : -1;
  if (!fork) return;
  for (int c = threadIdx.x; c < pages_for(P, rows_of(P, s)); c += kTableThreads) {
    const int p = row_of(P, s)[c];
    if (is_page(P, p)) atomicSub(P.ref + p, 1);
  }
  for (int c = threadIdx.x; c < pages_for(P, rows_of(P, from)); c += kTableThreads)
    new_table[(size_t)s * P.max_pages + c] = row_of(P, from)[c];
}
__global__ __launch_bounds__(kTableThreads) void pages_fork_put_kernel(const PageTables P, const int32_t* __restrict__ new_len,
                                                                       const int32_t* __restrict__ new_table) {
  const int s = blockIdx.x, n = new_len[s];
  if (n < 0) return;
  for (int c = threadIdx.x; c < pages_for(P, n); c += kTableThreads) {
    const int p = new_table[(size_t)s * P.max_pages + c];
    row_of(P, s)[c] = p;
    if (is_page(P, p)) atomicAdd(P.ref + p, 1);
  }
  if (threadIdx.x == 0) P.len[s] = n;
}

// ---- one workgroup that numbers pages and slots --------------------------------
constexpr int kOneThreads = 1024;
constexpr int kOneWaves = kOneThreads / 64;

// Sum of v over the threads before this one; *total: over all of them.
// Threads meet twice, so `part` may be used again after the call.
__device__ __forceinline__ int scan_before(int v, int* part, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int x = v;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const int y = __shfl_up(x, m, 64);
    if (lane >= m) x += y;
  }
  __syncthreads();
  if (lane == 63) part[wave] = x;
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kOneWaves; ++w) {
    const int y = part[w];
    if (w < wave) before += y;
    all += y;
  }
  *total = all;
  return before + x - v;
}

// Rows for the new tokens.  A slot that starts a row in a page it shares gets
// a copy of that page first; of several slots that share it, the last one in
// the call (in slot order) that would be left alone with it keeps it.
__global__ __launch_bounds__(kOneThreads) void pages_reserve_kernel(
    const PageTables P, const int32_t* __restrict__ n_new, int max_new, int32_t* __restrict__ rows,
    int32_t* __restrict__ copy_src, int32_t* __restrict__ copy_dst, int32_t* __restrict__ shortage,
    int32_t* __restrict__ first, int32_t* __restrict__ fresh, int32_t* __restrict__ free_list,
    int32_t* __restrict__ writers) {
  __shared__ int part[kOneWaves];
  __shared__ int lasts[kOneThreads];
  const int tid = threadIdx.x;
  const int page_mask = (1 << P.page_shift) - 1;
  auto wanted = [&](int s) { return min(max(n_new[s], 0), max_new); };

  // the pages that slots start to write in: how many writers came before
  for (int s = tid; s < P.n_slots; s += kOneThreads) {
    const int have = rows_of(P, s);
    if (wanted(s) > 0 && (have & page_mask)) {
      const int p = row_of(P, s)[have >> P.page_shift];
      if (is_page(P, p)) writers[p] = 0;
    }
  }
  __syncthreads();
  int total = 0, full = 0;
  for (int s0 = 0; s0 < P.n_slots; s0 += kOneThreads) {
    const int s = s0 + tid;
    int count = 0, last = -1, beyond = 0, holders = 0;
    if (s < P.n_slots) {
      const int have = rows_of(P, s), w = wanted(s);
      if (w > 0) {
        const long long end = (long long)have + w;  // may pass what the table holds
        const long long need = (end + page_mask) >> P.page_shift;
        count = (int)(need - pages_for(P, have));
        beyond = need > P.max_pages;
        if (have & page_mask) {
          const int p = row_of(P, s)[have >> P.page_shift];
          if (is_page(P, p)) {
            holders = P.ref[p];
            if (holders > 1) last = p;
          }
        }
      }
    }
    // writers of a shared page before this slot
    int copy = 0;
    if (__syncthreads_or(last >= 0)) {
      lasts[tid] = last;
      __syncthreads();
      if (last >= 0) {
        // past the L1, which the other slots' atomic additions went around
        int before = __hip_atomic_load(writers + last, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        for (int j = 0; j < tid; ++j) before += lasts[j] == last;
        copy = holders - before > 1;
      }
      __syncthreads();  // everyone has read the earlier writers
      if (last >= 0) atomicAdd(writers + last, 1);
      __syncthreads();
    }
    count += copy;
    int all;
    const int before = scan_before(count, part, &all);
    if (s < P.n_slots) {
      first[s] = total + before;
      fresh[s] = copy;
    }
    total += all;
    full += __syncthreads_count(beyond);
  }

  // the lowest free pages
  int found = 0;
  for (long long p0 = 0; p0 < P.n_pages && found < total; p0 += 4 * kOneThreads) {
    const long long p = p0 + 4 * tid;
    int is_free[4], mine = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      is_free[e] = p + e < P.n_pages && P.ref[p + e] <= 0;
      mine += is_free[e];
    }
    int all;
    int turn = found + scan_before(mine, part, &all);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (is_free[e]) {
        if (turn < total) free_list[turn] = (int)(p + e);
        ++turn;
      }
    found += all;
  }
  const int missing = max(total - found, 0);
  if (tid == 0) {
    shortage[0] = missing;
    shortage[1] = full;
  }
  const bool good = missing == 0 && full == 0;  // otherwise nothing changes
  __syncthreads();

  for (int s = tid; s < P.n_slots; s += kOneThreads) {
    const int w = good ? wanted(s) : 0;
    int from = -1, to = -1;
    if (w > 0) {
      const int have = rows_of(P, s), held = pages_for(P, have), need = pages_for(P, have + w);
      const int32_t* take = free_list + first[s];
      int32_t* row = row_of(P, s);
      if (fresh[s]) {
        from = row[held - 1];
        to = *take++;
        atomicSub(P.ref + from, 1);
        P.ref[to] = 1;
        row[held - 1] = to;
      }
      for (int c = held; c < need; ++c) {
        const int p = take[c - held];
        row[c] = p;
        P.ref[p] = 1;
      }
    }
    copy_src[s] = from;
    copy_dst[s] = to;
  }
  __syncthreads();
  const long long cells = (long long)P.n_slots * max_new;
  for (long long i = tid; i < cells; i += kOneThreads) {
    const int s = (int)(i / max_new), t = (int)(i - (long long)s * max_new);
    int r = -1;
    if (good && t < wanted(s)) {
      const int at = rows_of(P, s) + t;
      const int p = row_of(P, s)[at >> P.page_shift];
      if (is_page(P, p)) r = (p << P.page_shift) + (at & page_mask);
    }
    rows[i] = r;
  }
  __syncthreads();
  if (good)
    for (int s = tid; s < P.n_slots; s += kOneThreads)
      if (wanted(s) > 0) P.len[s] = rows_of(P, s) + wanted(s);
}

// Live pages above the number of live pages move into the holes below it, in
// ascending order on both sides.  to[p]: where page p >= live goes.
__global__ __launch_bounds__(kOneThreads) void pages_compact_kernel(const PageTables P, int32_t* __restrict__ move_src,
                                                                    int32_t* __restrict__ move_dst,
                                                                    int32_t* __restrict__ counts,
                                                                    int32_t* __restrict__ to) {
  __shared__ int part[kOneWaves];
  const int tid = threadIdx.x;
  int mine = 0;
  for (long long p = tid; p < P.n_pages; p += kOneThreads) mine += P.ref[p] > 0;
  int live;
  scan_before(mine, part, &live);
  int holes = 0, far = 0;
  for (long long p0 = 0; p0 < P.n_pages; p0 += 4 * kOneThreads) {
    const long long p = p0 + 4 * tid;
    int hole[4], up[4], h = 0, f = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool in = p + e < P.n_pages, used = in && P.ref[p + e] > 0;
      hole[e] = in && !used && p + e < live;
      up[e] = used && p + e >= live;
      h += hole[e];
      f += up[e];
    }
    int all_h, all_f;
    int at_h = holes + scan_before(h, part, &all_h), at_f = far + scan_before(f, part, &all_f);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (hole[e]) move_dst[at_h++] = (int)(p + e);
      if (up[e]) move_src[at_f++] = (int)(p + e);
      if (p + e < P.n_pages && p + e >= live) to[p + e] = (int)(p + e);
    }
    holes += all_h;
    far += all_f;
  }
  // as many holes as pages to move: both are what live pages and pages below
  // `live` do not have in common
  __syncthreads();
  for (int m = tid; m < P.n_pages / 2; m += kOneThreads) {
    if (m < far) {
      const int a = move_src[m], b = move_dst[m];
      to[a] = b;
      P.ref[b] = P.ref[a];
      P.ref[a] = 0;
    } else {
      move_src[m] = -1;
      move_dst[m] = -1;
    }
  }
  if (tid == 0) {
    counts[0] = live;
    counts[1] = far;
  }
}
__global__ __launch_bounds__(kTableThreads) void pages_renumber_kernel(const PageTables P, const int32_t* __restrict__ counts,
                                                                       const int32_t* __restrict__ to) {
  const int s = blockIdx.x, live = counts[0];
  for (int c = threadIdx.x; c < pages_for(P, rows_of(P, s)); c += kTableThreads) {
    const int p = row_of(P, s)[c];
    if (p >= live && p < P.n_pages) row_of(P, s)[c] = to[p];
  }
}

// ---- page copies ------------------------------------------------------------------
// A wave moves a piece of N KB at a time, all of it requested before the
// first store; consecutive waves take consecutive pieces of a page.  Many short
// waves did better than few long ones: 443 pages of 32 KB in 32 layers, K and
// V (1.86 GB moved), took 334 us (5.57 TB/s) with a 4 KB piece a wave, 339 with 8
// KB, 357 in a grid of 2,048 workgroups, 361 with ordinary loads and stores.
constexpr int kCopyThreads = 256;
constexpr int kCopyWaves = kCopyThreads / 64;

template <int N>
__global__ __launch_bounds__(kCopyThreads) void pages_copy_kernel(int n_pages, unsigned pieces, long long page_bytes,
                                                                  int n_layers, char* __restrict__ k, char* __restrict__ v,
                                                                  const int32_t* __restrict__ src,
                                                                  const int32_t* __restrict__ dst, long long n_pairs,
                                                                  const int32_t* __restrict__ count) {
  const int lane = threadIdx.x & 63;
  if (count) n_pairs = min(n_pairs, (long long)max(*count, 0));
  // (pair, layer and tensor, piece of the page), pieces fastest
  const unsigned per_pair = 2u * n_layers;
  const long long n = n_pairs * per_pair * pieces;
  for (long long i = (long long)blockIdx.x * kCopyWaves + (threadIdx.x >> 6); i < n;
       i += (long long)gridDim.x * kCopyWaves) {
    const long long page = i / pieces;
    const unsigned piece = (unsigned)(i - page * pieces);
    const long long pair = page / per_pair;
    const unsigned which = (unsigned)(page - pair * per_pair);
    const int a = src[pair], b = dst[pair];
    if (a < 0 || a >= n_pages || b < 0 || b >= n_pages) continue;
    char* pool = which & 1 ? v : k;
    const long long layer = (long long)(which >> 1) * n_pages;
    const char* from = pool + (layer + a) * page_bytes + (long long)piece * (N * 1024) + lane * 16;
    char* to = pool + (layer + b) * page_bytes + (long long)piece * (N * 1024) + lane * 16;
    uint4 x[N];
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = load_nt(from + j * 1024);
#pragma unroll
    for (int j = 0; j < N; ++j) store_nt(to + j * 1024, x[j]);
  }
}

}  // namespace

hipError_t launch_pages_trim(const PageTables& P, const int32_t* keep, hipStream_t s) {
  if (P.n_slots <= 0) return hipSuccess;
  hipLaunchKernelGGL(pages_trim_kernel, dim3(P.n_slots), dim3(kTableThreads), 0, s, P, keep);
  return hipGetLastError();
}

hipError_t launch_pages_fork(const PageTables& P, const int32_t* src_of, int32_t* ws, hipStream_t s) {
  if (P.n_slots <= 0) return hipSuccess;
  int32_t* new_table = ws + P.n_slots;
  hipLaunchKernelGGL(pages_fork_take_kernel, dim3(P.n_slots), dim3(kTableThreads), 0, s, P, src_of, ws, new_table);
  hipLaunchKernelGGL(pages_fork_put_kernel, dim3(P.n_slots), dim3(kTableThreads), 0, s, P, ws, new_table);
  return hipGetLastError();
}

hipError_t launch_pages_reserve(const PageTables& P, const int32_t* n_new, int32_t max_new, int32_t* rows,
                                int32_t* copy_src, int32_t* copy_dst, int32_t* shortage, int32_t* ws, hipStream_t s) {
  int32_t* first = ws;
  int32_t* fresh = first + P.n_slots;
  int32_t* free_list = fresh + P.n_slots;
  int32_t* writers = free_list + P.n_pages;
  hipLaunchKernelGGL(pages_reserve_kernel, dim3(1), dim3(kOneThreads), 0, s, P, n_new, max_new, rows, copy_src,
                     copy_dst, shortage, first, fresh, free_list, writers);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const PageTables& P, int32_t* move_src, int32_t* move_dst, int32_t* counts,
                                int32_t* ws, hipStream_t s) {
  hipLaunchKernelGGL(pages_compact_kernel, dim3(1), dim3(kOneThreads), 0, s, P, move_src, move_dst, counts, ws);
  if (P.n_slots > 0)
    hipLaunchKernelGGL(pages_renumber_kernel, dim3(P.n_slots), dim3(kTableThreads), 0, s, P, counts, ws);
  return hipGetLastError();
}

hipError_t launch_pages_copy(int32_t n_pages, int64_t page_bytes, int n_layers, uint16_t* k, uint16_t* v,
                             const int32_t* src, const int32_t* dst, int64_t n_pairs, const int32_t* count,
                             hipStream_t s) {
  if (n_pairs <= 0 || n_layers <= 0) return hipSuccess;
  const int kb = page_bytes % 4096 == 0 ? 4 : 2;
  const unsigned pieces = (unsigned)(page_bytes / (kb * 1024));
  const int64_t waves = n_pairs * n_layers * 2 * (int64_t)pieces;
  const dim3 grid((unsigned)std::min<int64_t>((waves + kCopyWaves - 1) / kCopyWaves, 65536)), block(kCopyThreads);
#define KVC_COPY(N)                                                                                             \
  hipLaunchKernelGGL(pages_copy_kernel<N>, grid, block, 0, s, n_pages, pieces, (long long)page_bytes, n_layers, \
                     reinterpret_cast<char*>(k), reinterpret_cast<char*>(v), src, dst, (long long)n_pairs, count)
  if (kb == 4) KVC_COPY(4);
  else KVC_COPY(2);
#undef KVC_COPY
  return hipGetLastError();
}

}  // namespace kvc
