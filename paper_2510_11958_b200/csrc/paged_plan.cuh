// Pages and slots for a step's new tokens, on the GPU: dmtd_paged_plan.
//
// Request b holds ceil(len / page) pages and wants ceil((len + n) / page) after the step; page i of all the grants in turn is
// the i-th from the top of the stack of free pages.  Two prefix sums (rows, wanted pages) give every request its first row and its
// place in the stack; after that every row and every new page is independent: a binary search of the prefix sums finds its request.
//
// Bound: latency; a step of 8 requests moves 300 bytes, one of 4096 half a megabyte.  One launch of one block, or of one cluster
// of 8 where there is enough to write: every block works the prefix sums out for itself (a thousand lengths are one load a
// thread and two scans), so that the only barrier of the cluster is the one between reading what the call may overwrite
// (lengths and the count of free pages may be updated in place) and writing it.
#pragma once

#include "paged_common.cuh"

namespace dmtd {

constexpr int PLAN_THREADS = 1024;
constexpr int PLAN_CLUSTER = 8;
constexpr int PLAN_MAX_REQUESTS = 8192;
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
};

__device__ __forceinline__ int plan_add(int a, int b) { return min(a + b, PLAN_MOST); }   // of values in [0, PLAN_MOST]

// Inclusive prefix sum over the block's threads; `total`: of all of them.  Whole block.
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
  int t = totals[lane];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int w = __shfl_up_sync(0xffffffffu, t, o);
    if (lane >= o) t = plan_add(t, w);
  }
  const int before = __shfl_sync(0xffffffffu, t, max(warp - 1, 0));
  total = __shfl_sync(0xffffffffu, t, 31);
  return warp ? plan_add(v, before) : v;
}

// The first of n entries of a rising array that is above x (n if none is).
__device__ __forceinline__ int plan_above(const int *a, int n, int x) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (a[mid] > x) hi = mid; else lo = mid + 1;
  }
  return lo;
}

__global__ void __launch_bounds__(PLAN_THREADS, 1) paged_plan_kernel(const __grid_constant__ PagedPlanParams P) {
  extern __shared__ int plan_smem[];
  int *const totals = plan_smem, *const shared_avail = plan_smem + 32;
  int *const len = plan_smem + PLAN_WORDS;                     // [n_requests] keys held
  int *const row_end = len + P.n_requests;                     // rows up to and with request b's, cut off at n_rows
  int *const page_end = row_end + P.n_requests;                // wanted pages up to and with request b's; refused: -1 - that
  paged_enter();
  const int B = P.n_requests, rank = blockIdx.x, n_ranks = gridDim.x, page = 1 << P.lg_page;
  const long long room = (long long)P.table_stride << P.lg_page;
  const int tid = threadIdx.x;
  int avail = min(max(*P.n_free, 0), P.n_pages);

  // ---- lengths and ended requests; page_end holds the pages of ended requests up to and with b's for now
  int gone = 0;
  bool any_ended = false;
  for (int b0 = 0; b0 < B; b0 += PLAN_THREADS) {
    const int b = b0 + tid;
    int held = 0;
    bool ended = false;
    if (b < B) {
      const int L = (int)min((long long)max(P.lens[b], 0), room);
      len[b] = L;
      ended = P.n_new[b] < 0;
      held = ended ? (L + page - 1) >> P.lg_page : 0;
    }
    if (__syncthreads_or(ended)) {
      any_ended = true;
    }
    if (any_ended) {
      int total;
      const int s = plan_scan(held, totals, total);
      if (b < B) page_end[b] = plan_add(gone, s);
      gone = plan_add(gone, total);
    } else if (b < B) {
      page_end[b] = 0;
    }
  }
  if (gone > 0) {
    // the first block puts their pages on the stack, in the order of requests and pages, those that are none left out
    __syncthreads();
    if (rank == 0) {
      for (int i0 = 0; i0 < gone; i0 += PLAN_THREADS) {
        const int i = i0 + tid;
        int id = -1;
        if (i < gone) {
          const int b = plan_above(page_end, B, i);
          id = P.table[(size_t)b * P.table_stride + i - (b ? page_end[b - 1] : 0)];
        }
        const int good = id >= 0 && id < P.n_pages;
        int total;
        const int s = plan_scan(good, totals, total);
        if (good && avail + s <= P.n_pages) P.free_pages[avail + s - 1] = id;
        avail = min(avail + total, P.n_pages);
      }
      if (tid == 0) *shared_avail = avail;
    }
    __syncthreads();                                           // page_end is written anew below
  }

  // ---- rows and pages of every request
  int rows = 0, pages = 0;
  for (int b0 = 0; b0 < B; b0 += PLAN_THREADS) {
    const int b = b0 + tid;
    int n = 0, L = 0;
    bool live = false;
    if (b < B) {
      L = len[b];
      n = P.n_new[b];
      live = n >= 0;
      n = min(max(n, 0), PLAN_MOST);
    }
    int total;
    const int end = plan_add(rows, plan_scan(n, totals, total));
    rows = plan_add(rows, total);
    const bool fits = live && (long long)L + n <= room && end <= P.n_rows;
    const int want = fits ? ((L + n + page - 1) >> P.lg_page) - ((L + page - 1) >> P.lg_page) : 0;
    const int last = plan_add(pages, plan_scan(want, totals, total));
    pages = plan_add(pages, total);
    if (b < B) {
      row_end[b] = min(end, P.n_rows);
      // whether the stack holds enough is known once the ended requests' pages are on it
      page_end[b] = fits ? last : -1 - last;
    }
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
  const int first = rank * PLAN_THREADS + tid, step = n_ranks * PLAN_THREADS;
  for (int b = first; b < B; b += step) {
    const int start = b ? row_end[b - 1] : 0, n = row_end[b] - start;
    const bool ok = served(b);
    P.row_start[b] = start;
    P.granted[b] = ok ? n : 0;
    P.lens_out[b] = P.n_new[b] < 0 ? 0 : len[b] + (ok ? n : 0);
  }
  if (rank == 0 && tid == 0) {
    P.row_start[B] = B ? row_end[B - 1] : 0;
    // wanted pages rise along the requests, so the served ones' are the first on the stack: those in front of the first
    // request that goes beyond it
    int lo = 0, hi = B;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (upto(mid) > avail) hi = mid; else lo = mid + 1;
    }
    *P.n_free_out = avail - upto(lo - 1);
  }
  const int n_given = min(pages, avail);
  for (int i = first; i < n_given; i += step) {
    // the first request whose wanted pages go beyond i
    int lo = 0, hi = B;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (upto(mid) > i) hi = mid; else lo = mid + 1;
    }
    if (lo < B && served(lo)) {
      const int held = (len[lo] + page - 1) >> P.lg_page;
      P.table[(size_t)lo * P.table_stride + held + i - upto(lo - 1)] = P.free_pages[avail - 1 - i];
    }
  }
  for (int t = first; t < P.n_rows; t += step) {
    const int b = plan_above(row_end, B, t);
    int position = 0, slot = -1;
    if (b < B && served(b)) {
      const int pos = len[b] + t - (b ? row_end[b - 1] : 0);
      const int held = (len[b] + page - 1) >> P.lg_page, at = pos >> P.lg_page;
      const int id = at < held ? P.table[(size_t)b * P.table_stride + at] : P.free_pages[avail - 1 - (upto(b - 1) + at - held)];
      if (id >= 0 && id < P.n_pages) {
        position = pos;
        slot = (id << P.lg_page) + (pos & (page - 1));
      }
    }
    P.position[t] = position;
    P.slot[t] = slot;
  }
  // no block leaves while another reads its shared memory
  if (n_ranks > 1 && gone > 0) {
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
  }
}

}  // namespace dmtd
