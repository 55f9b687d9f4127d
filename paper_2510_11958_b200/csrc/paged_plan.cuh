// Pages and slots for a step's new tokens, on the GPU: dmtd_paged_plan.
//
// Request b holds ceil(len / page) pages and wants ceil((len + n) / page) after the step; page i of all the grants in turn is
// the i-th from the top of the stack of free pages.  Two prefix sums (rows, wanted pages) give every request its first row and its
// place in the stack; after that every row and every new page is independent: a binary search of the prefix sums finds its request.
//
// Bound: latency; a step of 8 requests moves 300 bytes, one of 4096 half a megabyte.  One launch of one block, or of one cluster
// of 8 where there is enough to write: every block works the prefix sums out for itself (a thread to up to eight requests in a
// row, then one scan of the threads' sums), so that the only barrier of the cluster is the one between reading what the call may overwrite
// (lengths and the count of free pages may be updated in place) and writing it.  The search of a row costs some 150 instructions, so that
// the rows of a large step (53 000 rows: 11 us on the cluster's 8 SMs) are left to a second launch that fills all SMs and reads
// the tables as the first has left them.  Measured: 8 requests 4.0 us, 300 with 6481 rows 8.8, 4096 with 53 518 rows 15.0.
#pragma once

#include "paged_common.cuh"

namespace dmtd {

constexpr int PLAN_THREADS = 1024;
constexpr int PLAN_CLUSTER = 8;              // blocks, where one is not enough
constexpr int PLAN_MAX_REQUESTS = 8192;
constexpr int PLAN_RUN = 4;                  // released pages that a thread works on at a time
constexpr int PLAN_WORDS = 40;               // shared memory in front of the arrays: a scan's warp totals, broadcast values
constexpr int PLAN_MOST = 0x3fffffff;        // prefix sums stay at this value once they have reached it

inline int plan_smem_bytes(int n_requests) { return (PLAN_WORDS + 3 * n_requests) * 4; }

struct PagedPlanParams {
  const int *lens, *n_new;
  int n_requests, lg_page;
  int *table;
  int table_stride;
  int *free_pages;
  int n_pages;
  const int *n_free;
  int n_rows;
  int *row_start, *position, *slot, *granted, *lens_out, *n_free_out;
  int fill_rows;                             // position and slot are written here, and not by paged_rows_of_plan_kernel
};

__device__ __forceinline__ int plan_add(int a, int b) { return min(a + b, PLAN_MOST); }   // of values in [0, PLAN_MOST]

// Sum over the threads in front of this one; `total`: over all of them.  Whole block.
__device__ __forceinline__ int plan_scan(int v, int *totals, int &total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int w = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v = plan_add(v, w);
  }
  __syncthreads();                           // the totals of the scan before have been read
  if (lane == 31) totals[warp] = v;
  __syncthreads();
  int t = lane < (int)(blockDim.x >> 5) ? totals[lane] : 0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int w = __shfl_up_sync(0xffffffffu, t, o);
    if (lane >= o) t = plan_add(t, w);
  }
  const int before = __shfl_sync(0xffffffffu, t, max(warp - 1, 0));
  total = __shfl_sync(0xffffffffu, t, 31);
  v = __shfl_up_sync(0xffffffffu, v, 1);
  return plan_add(lane ? v : 0, warp ? before : 0);
}

// For each x: the first of n entries of a rising sequence that is above it (n if none is).  The searches run side by side; `top`: the
// largest power of two that is not above n.
template <int N, class F>
__device__ __forceinline__ void plan_above(F &&entry, int n, int top, const int (&x)[N], int (&found)[N]) {
#pragma unroll
  for (int k = 0; k < N; ++k) found[k] = 0;
  for (int w = top; w > 0; w >>= 1) {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if (found[k] + w <= n && entry(found[k] + w - 1) <= x[k]) found[k] += w;
  }
}

__global__ void __launch_bounds__(PLAN_THREADS, 1) paged_plan_kernel(const __grid_constant__ PagedPlanParams P) {
  extern __shared__ int plan_smem[];
  constexpr int EACH = PLAN_MAX_REQUESTS / PLAN_THREADS;
  int *const totals = plan_smem, *const shared_avail = plan_smem + 32;
  int *const len = plan_smem + PLAN_WORDS;                     // [n_requests] keys held
  int *const row_end = len + P.n_requests;                     // rows up to and with request b's, cut off at n_rows
  int *const page_end = row_end + P.n_requests;                // wanted pages up to and with request b's; refused: -1 - that
  paged_enter();
  const int B = P.n_requests, rank = blockIdx.x, n_ranks = gridDim.x, lg = P.lg_page, page = 1 << lg;
  const int room = (int)min((long long)P.table_stride << lg, 0x7fffffffll);
  const int threads = blockDim.x, tid = threadIdx.x, per = (B + threads - 1) / threads, b0 = tid * per;          // per <= EACH
  const int top = B ? 1 << (31 - __clz(B)) : 0;
  int avail = min(max(*P.n_free, 0), P.n_pages);
  auto pages_of = [&](int keys) { return (int)(((unsigned)keys + page - 1) >> lg); };

  // ---- this thread's requests
  int L[EACH], n[EACH], gone_here = 0;                         // n: -1: ended
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    L[i] = n[i] = 0;
    if (i >= per) break;
    if (b0 + i < B) {
      L[i] = min(max(P.lens[b0 + i], 0), room);
      n[i] = min(max(P.n_new[b0 + i], -1), PLAN_MOST);
    }
  }
  int rows_here = 0;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    if (i >= per) break;
    if (n[i] < 0) gone_here = plan_add(gone_here, pages_of(L[i]));
    rows_here = plan_add(rows_here, max(n[i], 0));
    if (b0 + i < B) len[b0 + i] = L[i];
  }
  int gone = 0;
  if (__syncthreads_or(gone_here)) {
    // the first block puts the ended requests' pages on the stack, in the order of requests and pages, ids that are none left out
    int at = plan_scan(gone_here, totals, gone);
    if (rank == 0) {
#pragma unroll
      for (int i = 0; i < EACH; ++i) {
        if (i >= per) break;
        if (n[i] < 0) at = plan_add(at, pages_of(L[i]));
        if (b0 + i < B) page_end[b0 + i] = at;      // for now: pages of ended requests up to and with this one's
      }
      __syncthreads();
      for (int i0 = 0; i0 < gone; i0 += threads * PLAN_RUN) {
        int x[PLAN_RUN], b[PLAN_RUN], ids[PLAN_RUN], good = 0;
#pragma unroll
        for (int k = 0; k < PLAN_RUN; ++k) x[k] = i0 + tid * PLAN_RUN + k;
        if (x[0] < gone) plan_above([&](int i) { return page_end[i]; }, B, top, x, b);
#pragma unroll
        for (int k = 0; k < PLAN_RUN; ++k)
          ids[k] = x[k] < gone ? P.table[(size_t)b[k] * P.table_stride + x[k] - (b[k] ? page_end[b[k] - 1] : 0)] : -1;
#pragma unroll
        for (int k = 0; k < PLAN_RUN; ++k) good += ids[k] >= 0 && ids[k] < P.n_pages;
        int total;
        int to = avail + plan_scan(good, totals, total);
#pragma unroll
        for (int k = 0; k < PLAN_RUN; ++k)
          if (ids[k] >= 0 && ids[k] < P.n_pages) {
            if (to < P.n_pages) P.free_pages[to] = ids[k];
            ++to;
          }
        avail = min(avail + total, P.n_pages);
      }
      if (tid == 0) *shared_avail = avail;
    }
    __syncthreads();                                           // page_end is written anew below
  }

  // ---- rows and pages of every request
  int rows, pages;
  int end = plan_scan(rows_here, totals, rows);
  int want[EACH], want_here = 0;                               // -1: refused or ended
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    want[i] = -1;
    if (i >= per) break;
    end = plan_add(end, max(n[i], 0));
    if (b0 + i < B) {
      if (n[i] >= 0 && n[i] <= room - L[i] && end <= P.n_rows) {
        want[i] = pages_of(L[i] + n[i]) - pages_of(L[i]);
        want_here += want[i];
      }
      row_end[b0 + i] = min(end, P.n_rows);
    }
  }
  int last = plan_scan(want_here, totals, pages);              // (table entries are fewer than PLAN_MOST)
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    if (i >= per) break;
    last += max(want[i], 0);
    // whether the stack holds enough is known once the ended requests' pages are on it
    if (b0 + i < B) page_end[b0 + i] = want[i] >= 0 ? last : -1 - last;
  }

  // ---- everything that the call may overwrite has been read, and the stack is complete
  if (n_ranks > 1) {
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    if (gone > 0) asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(avail) : "r"(cluster_address(smem_u32(shared_avail), 0)) : "memory");
  } else {
    __syncthreads();
  }
  auto upto = [&](int b) { return b < 0 ? 0 : page_end[b] < 0 ? -1 - page_end[b] : page_end[b]; };
  // granted: it fits, and needs no page or finds all of its own on the stack
  auto served = [&](int b) { return page_end[b] >= 0 && (page_end[b] == upto(b - 1) || page_end[b] <= avail); };
  const int first = rank * threads + tid, step = n_ranks * threads;
  const int n_given = min(pages, avail);
  for (int i = first; i < n_given; i += step) {
    const int x[1] = {i};
    int b[1];
    plan_above(upto, B, top, x, b);                            // the first request whose wanted pages go beyond i
    if (b[0] < B && served(b[0])) P.table[(size_t)b[0] * P.table_stride + pages_of(len[b[0]]) + i - upto(b[0] - 1)] = P.free_pages[avail - 1 - i];
  }
  for (int t = first; t < P.n_rows && P.fill_rows; t += step) {
    const int x[1] = {t};
    int found[1], position = 0, slot = -1;
    plan_above([&](int i) { return row_end[i]; }, B, top, x, found);
    const int b = found[0];
    if (b < B && served(b)) {
      const int pos = len[b] + t - (b ? row_end[b - 1] : 0), held = pages_of(len[b]), at = pos >> lg;
      const int id = *(at < held ? P.table + (size_t)b * P.table_stride + at : P.free_pages + (avail - 1 - (upto(b - 1) + at - held)));
      if (id >= 0 && id < P.n_pages) {
        position = pos;
        slot = (id << lg) + (pos & (page - 1));
      }
    }
    P.position[t] = position;
    P.slot[t] = slot;
  }
  for (int b = first; b < B; b += step) {
    const int start = b ? row_end[b - 1] : 0;
    const bool ok = served(b);
    const int n = ok ? row_end[b] - start : 0;
    P.row_start[b] = start;
    P.granted[b] = n;
    P.lens_out[b] = P.n_new[b] < 0 ? 0 : len[b] + n;
  }
  if (rank == 0 && tid == 0) {
    P.row_start[B] = B ? row_end[B - 1] : 0;
    // wanted pages rise along the requests, so the served ones' are the first on the stack: those in front of the first
    // request that goes beyond it
    const int x[1] = {avail};
    int b[1];
    plan_above(upto, B, top, x, b);
    *P.n_free_out = avail - upto(b[0] - 1);
  }
  // no block leaves while another reads its shared memory
  if (n_ranks > 1 && gone > 0) {
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  }
}

// Position and slot of every row out of what paged_plan_kernel has written.  Blocks of PLAN_FILL rows each.
constexpr int PLAN_FILL = 512;
__global__ void __launch_bounds__(PLAN_FILL) paged_rows_of_plan_kernel(const __grid_constant__ PagedPlanParams P) {
  extern __shared__ int plan_smem[];                           // row_start [n_requests + 1]
  paged_enter();
  const int B = P.n_requests, lg = P.lg_page, t = blockIdx.x * PLAN_FILL + threadIdx.x;
  for (int b = threadIdx.x; b <= B; b += PLAN_FILL) plan_smem[b] = P.row_start[b];
  __syncthreads();
  if (t >= P.n_rows) return;
  const int x[1] = {t};
  int found[1], position = 0, slot = -1;
  plan_above([&](int i) { return plan_smem[i + 1]; }, B, B ? 1 << (31 - __clz(B)) : 0, x, found);
  const int b = found[0];
  if (b < B) {
    const int n = P.granted[b], pos = P.lens_out[b] - n + t - plan_smem[b];
    if (n > 0) {
      const int id = P.table[(size_t)b * P.table_stride + (pos >> lg)];
      if (id >= 0 && id < P.n_pages) {
        position = pos;
        slot = (id << lg) + (pos & ((1 << lg) - 1));
      }
    }
  }
  P.position[t] = position;
  P.slot[t] = slot;
}

}  // namespace dmtd
