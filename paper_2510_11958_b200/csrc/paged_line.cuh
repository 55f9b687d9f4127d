// The work of a paged attention launch as one line of units, cut into equal shares for its blocks, and the merge of what is cut.
//
// An item is a row tile (up to `tile` consecutive new positions of a request, all query heads of one kv head) and the
// keys that its last position sees, in units of 1 << lg_unit keys; one unit in front of them stands for what an item costs
// whatever its length is (queries, joining the warps, storing).  Items of unequal length follow each other on the
// line: requests in order, row tiles in order, kv heads.  A block takes an equal share of the line whatever the lengths
// are, so that there is one wave and no tail.  An item that lies across a border between shares leaves a partial
// result (unnormalised sums with their level) per block in scratch memory, and paged_merge_kernel joins them; a block has at
// most two of those, one in front and one behind, so scratch has two places to a block.
#pragma once

#include <type_traits>

#include "paged_attention.cuh"

namespace dmtd {

// Sum of floor((a i + b) / m) over i = 0 .. n - 1, for a, b < m and a n + b < 2^32.  It counts the points (i, j) with j >= 1 and
// j m <= a i + b; column by column instead of row by row these are n - ceil((j m - b) / a) for every j up to the last row's quotient, so
// that n q minus a sum of the same kind with a and m exchanged remains (the reciprocity of such sums: Graham, Knuth, Patashnik, Concrete
// Mathematics, section 3.5), a step of Euclid's algorithm at a time.
// (For groups of 3, 5, 6 ... heads.  Inlined, the chunk kernel takes 263 us instead of 259 for 2000 rows over 8000 keys with groups of 4.)
__host__ __device__ __noinline__ inline long long quotients_sum(unsigned n, unsigned a, unsigned b, unsigned m) {
  long long sum = 0, sign = 1;
  while (n > 0 && a > 0) {
    const unsigned q = (a * (n - 1) + b) / m;
    sum += sign * (long long)n * q;
    // ceil((j m - b) / a), j = 1 .. q, is floor((m j' + m - b + a - 1) / a), j' = 0 .. q - 1; whole parts go to the sum at once
    const unsigned rest = m - b + a - 1, slope = m % a;
    sum -= sign * ((long long)(m / a) * q * (q - 1ll) / 2 + (long long)(rest / a) * q);
    sign = -sign;
    m = a;
    a = slope;
    b = rest % m;
    n = q;
  }
  return sum;
}

// x / y without the 64-bit division where 32 bits do
__host__ __device__ __forceinline__ long long quotient(long long x, long long y) {
  return ((x | y) >> 32) ? x / y : (long long)((unsigned)x / (unsigned)y);
}

// Which requests are on a launch's line, and how they are cut.
struct PagedCut {
  int tile;                          // positions of a row tile
  int lg_tile;                       // -1: no power of two
  int lg_unit;
  int min_new, max_new;              // requests of that many new rows
  int least;                         // units of a share, at least
};

struct PagedRequest {
  int b, row0, n, c;                 // first row of q, new rows, position of the first of them (may be negative)
  int tiles;
  // units of row tile i, and of the first m row tiles, for one kv head
  __host__ __device__ __forceinline__ int units(const PagedCut &K, int i) const {
    const int keys = c + min(n, (i + 1) * K.tile);
    return 1 + (keys <= 0 ? 0 : (int)(((unsigned)keys + (1u << K.lg_unit) - 1) >> K.lg_unit));
  }
  __host__ __device__ __forceinline__ long long units_before(const PagedCut &K, int m) const {
    if (m == 0) return 0;
    if (m == 1) return units(K, 0);
    const int full = min(m, n / K.tile);
    const int none = c < 0 ? min(full, (int)(-(long long)c / K.tile)) : 0;       // tiles in front of position 0
    long long s = full;
    const unsigned n_sum = full - none, lg = K.lg_unit, unit = 1u << lg;
    // Tiles from `none` on see a key at least, so that `base`, their first one's keys + unit - 1, is above 0 whatever c is:
    // ceil(x / unit) = floor((x + unit - 1) / unit)
    const unsigned long long base = (unsigned long long)((long long)c + (none + 1ll) * K.tile) + unit - 1;
    if (n_sum == 0) {
    } else if (K.lg_tile < 0) {
      s += (long long)(base >> lg) * n_sum + quotients_sum(n_sum, K.tile, (unsigned)(base & (unit - 1)), unit);         // (tile < unit: 3 heads or more)
    } else if (K.lg_tile >= (int)lg) {
      s += (long long)(base >> lg) * n_sum + ((long long)n_sum * (n_sum - 1) / 2 << (K.lg_tile - lg));
    } else {
      // base = q unit + rest: q, and floor(j / r) for the n_sum values of j from rest / tile on, r = unit / tile
      const unsigned lr = lg - K.lg_tile, j0 = (unsigned)(base & (unit - 1)) >> K.lg_tile;
      auto sum_below = [&](unsigned j) {                       // floor(0 / r) + ... + floor((j - 1) / r)
        const long long a = j >> lr;
        return (a * (a - 1) / 2 << lr) + a * (j & ((1u << lr) - 1));
      };
      s += (long long)(base >> lg) * n_sum + sum_below(j0 + n_sum) - sum_below(j0);
    }
    return m > full ? s + units(K, full) : s;
  }
};

__host__ __device__ __forceinline__ PagedRequest paged_request(const PagedBatch &batch, int lg_page, const PagedCut &K, int b) {
  PagedRequest r;
  r.b = b;
  r.row0 = batch.row(b);
  r.n = max(0, batch.row(b + 1) - r.row0);
  r.c = batch.keys(b, lg_page) - r.n;
  if (r.n < K.min_new || r.n > K.max_new) r.n = 0;
  r.tiles = (r.n + K.tile - 1) / K.tile;
  return r;
}

// A block's place on the line: an item and the part of its units in the block's share.
struct PagedPiece {
  PagedRequest r;
  int i, kvh;                        // row tile, kv head
  int t0, t1, per_item;              // units [t0, t1) of per_item, the one in front among them
  __host__ __device__ __forceinline__ bool whole() const { return t0 == 0 && t1 == per_item; }
  __host__ __device__ __forceinline__ int first(const PagedCut &K) const { return i * K.tile; }
  __host__ __device__ __forceinline__ int rows(const PagedCut &K) const { return min(K.tile, r.n - i * K.tile); }
  // the piece's units of keys
  __host__ __device__ __forceinline__ int key_begin() const { return max(t0 - 1, 0); }
  __host__ __device__ __forceinline__ int key_end() const { return t1 - 1; }
  // keys that the tile's last row sees, and position of its first row
  __host__ __device__ __forceinline__ int keys(const PagedCut &K) const { return max(0, r.c + min(r.n, (i + 1) * K.tile)); }
  __host__ __device__ __forceinline__ int position(const PagedCut &K) const { return r.c + i * K.tile; }
};

// The first THREADS threads of a block work out the line's length and their block's share.  KEPT: as many requests at most are
// kept in shared memory; of larger batches they are read anew where they are needed.
template <int THREADS, int KEPT>
struct PagedShare {
  long long total, begin, end;
  long long each, rest;              // a share's units: `each`, and `rest` of the shares have one more
  int n_blocks;
  struct Shared {
    long long warp_units[THREADS / 32];
    PagedPiece first;                // the share's first piece, by plan()
    int kept[KEPT][3];               // row0, n, c
  };
  __host__ __device__ __forceinline__ PagedRequest request(const PagedAttentionParams &P, const PagedCut &K, const Shared &sh, int b) const {
    if (P.batch.n_requests > KEPT) return paged_request(P.batch, P.pool.lg_page, K, b);
    PagedRequest r;
    r.b = b;
    r.row0 = sh.kept[b][0];
    r.n = sh.kept[b][1];
    r.c = sh.kept[b][2];
    r.tiles = (r.n + K.tile - 1) / K.tile;
    return r;
  }

  // Whole block; `sh` in shared memory.  The threads' requests follow each other on the line; the thread among whose requests the
  // share begins works out its first piece.
  __device__ __forceinline__ void plan(const PagedAttentionParams &P, const PagedCut &K, Shared &sh, int block, int grid) {
    const int B = P.batch.n_requests, per = (B + THREADS - 1) / THREADS, b0 = threadIdx.x * per, warp = threadIdx.x >> 5;
    long long mine = 0, upto = 0;
    PagedRequest r{};
    if (threadIdx.x < THREADS) {
      for (int b = b0; b < min(B, b0 + per); ++b) {
        r = paged_request(P.batch, P.pool.lg_page, K, b);
        mine += r.units_before(K, r.tiles) * P.nkv;
        if (B <= KEPT) {
          sh.kept[b][0] = r.row0;
          sh.kept[b][1] = r.n;
          sh.kept[b][2] = r.c;
        }
      }
      upto = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long w = __shfl_up_sync(0xffffffffu, upto, o);
        if ((threadIdx.x & 31) >= o) upto += w;
      }
      if ((threadIdx.x & 31) == 31) sh.warp_units[warp] = upto;
    }
    __syncthreads();
    total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 32; ++w) {
      if (w < warp) upto += sh.warp_units[w];
      total += sh.warp_units[w];
    }
    // no empty shares: the pieces of an item are consecutive blocks
    n_blocks = (int)min((long long)grid, quotient(total + K.least - 1, K.least));
    each = n_blocks ? quotient(total, n_blocks) : 0;
    rest = total - each * n_blocks;
    begin = block < n_blocks ? start(block) : total;
    end = block < n_blocks ? start(block + 1) : total;
    if (threadIdx.x < THREADS && begin < end && upto - mine <= begin && begin < upto) {
      long long v = begin - (upto - mine);
      if (per > 1) {
        for (int b = b0;; ++b) {
          r = request(P, K, sh, b);
          const long long all = r.units_before(K, r.tiles) * P.nkv;
          if (v < all || b + 1 >= B) break;
          v -= all;
        }
      }
      sh.first = piece_of(P, K, r, v);
    }
    __syncthreads();
  }
  __host__ __device__ __forceinline__ long long start(int block) const { return each * block + min((long long)block, rest); }
  // the block that holds unit u
  __host__ __device__ __forceinline__ int holder(long long u) const {
    const long long longer = rest * (each + 1);          // units of the longer shares, which come first
    return (int)(u < longer ? quotient(u, each + 1) : rest + quotient(u - longer, each));
  }

  // The piece that begins with the share, at unit v of request r.
  __host__ __device__ __forceinline__ PagedPiece piece_of(const PagedAttentionParams &P, const PagedCut &K, const PagedRequest &r, long long v) const {
    PagedPiece p;
    p.r = r;
    // the row tile: the last whose units begin at or before v
    int t = 0;
    for (int top = r.tiles; top - t > 1;) {
      const int mid = (t + top) >> 1;
      if (r.units_before(K, mid) * P.nkv <= v) t = mid; else top = mid;
    }
    if (t) v -= r.units_before(K, t) * P.nkv;
    p.i = t;
    p.per_item = r.units(K, t);
    p.kvh = (int)quotient(v, p.per_item);
    p.t0 = (int)(v - (long long)p.kvh * p.per_item);
    p.t1 = (int)min((long long)p.per_item, p.t0 + (end - begin));
    return p;
  }
  // The piece behind p, which ends at unit u of the line; false: the share or the batch ends there.
  __host__ __device__ __forceinline__ bool next(const PagedAttentionParams &P, const PagedCut &K, const Shared &sh, PagedPiece &p, long long u) const {
    if (u >= end) return false;
    if (++p.kvh == P.nkv) {
      p.kvh = 0;
      if (++p.i == p.r.tiles) {
        p.i = 0;
        int b = p.r.b;
        do {
          if (++b >= P.batch.n_requests) return false;
          p.r = request(P, K, sh, b);
        } while (p.r.n == 0);
      }
      p.per_item = p.r.units(K, p.i);
    }
    p.t0 = 0;
    p.t1 = (int)min((long long)p.per_item, end - u);
    return true;
  }
};

// What the merge needs to know of an item that begins in a block and goes on behind it.
struct PagedCutItem {
  int pieces;                        // 0: the block's last item ends in the block
  int b, row0, rows, first_seen, kvh;     // request, first row of q, rows, keys that the first row sees
  int pad[2];
};

inline PagedCut paged_cut(int tile, int lg_unit, int min_new, int max_new, int least) {
  return PagedCut{tile, (tile & (tile - 1)) ? -1 : 31 - __builtin_clz((unsigned)tile), lg_unit, min_new, max_new, least};
}

// Scratch: an entry per block, then two partial results per block: [tile rows][D] floats (the chunk kernel: [D / 4][tile
// rows][4]) and (level, sum) per row.
struct PagedScratch {
  PagedCutItem *items;
  float *parts;
  int rows;                          // query rows of a place
  unsigned *entered;                 // PAGED_ENTERED while the chunk kernel has what was written in front of the call in sight
  template <int D> __device__ __forceinline__ float *sums(int place) const { return parts + (size_t)place * rows * (D + 2); }
  template <int D> __device__ __forceinline__ float2 *levels(int place) const {
    return reinterpret_cast<float2 *>(sums<D>(place) + (size_t)rows * D);
  }
};
// The row kernel behind a chunk kernel starts while that one runs.  griddepcontrol.wait alone would make what the launches in front of both have
// written (lengths, tables, queries, the cache's new rows) visible to it, and only at the chunk kernel's end.  So a thread of the
// chunk kernel that has waited releases this word before it lets the row kernel in, the row kernel's blocks acquire it, and
// its first block clears it at its end (in the merge that costs 0.7 us a call).  A block that does not find it waits for the chunk kernel's end.  (Waiting always: 144 us instead of 136 for the rows
// and pieces of `attention_mixed`; the row kernel in front: 141.)
constexpr unsigned PAGED_ENTERED = 0x9d1c6b35u;
__device__ __forceinline__ bool paged_entered(const unsigned *entered) {
  for (int i = 0; i < 64; ++i)
    if (ld_acquire_u32(entered) == PAGED_ENTERED) return true;
  return false;
}

// A block's place for the piece of an item that began in an earlier block / that goes on in a later one.
__device__ __forceinline__ int paged_place(int block, bool began_here) { return 2 * block + (began_here ? 1 : 0); }

// Joins query row qi of the row kernel's item that is cut at the end of `block`'s share, by one warp.  Levels are powers of two.
// The lanes fetch the pieces' levels side by side, and all lanes the pieces' sums, which do not wait for the levels.
template <typename T, typename KVT, int D>
__device__ __forceinline__ void paged_join_row(const PagedAttentionParams &P, const PagedScratch &S, const PagedCutItem &c, int block, int qi) {
  constexpr int E = D / 32, DEEP = 8;
  const int lane = threadIdx.x & 31, G = P.nq / P.nkv;
  float m = -INFINITY, l = 0.f, o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  for (int s0 = 0; s0 < c.pieces; s0 += 32) {
    const int n = min(32, c.pieces - s0);
    auto place = [&](int s) { return paged_place(block + s0 + s, s0 + s == 0); };
    float v[DEEP][E];
    auto load = [&](int first) {
#pragma unroll
      for (int s = 0; s < DEEP; ++s)
        if (first + s < n) load_pack(S.sums<D>(place(first + s)) + (size_t)qi * D + lane * E, v[s]);
    };
    const float2 ml = lane < n ? S.levels<D>(place(lane))[qi] : make_float2(-INFINITY, 0.f);
    load(0);
    const float top = fmaxf(m, warp_max(ml.x));
    const float old = m > -INFINITY ? exp2f(m - top) : 0.f;
    const float w = ml.x > -INFINITY ? exp2f(ml.x - top) : 0.f;
    // (a piece whose scores are all NaN has level -inf and sum NaN, which stays)
    l = l * old + warp_sum(ml.y * w);
    m = top;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] *= old;
    for (int first = 0; first < n; first += DEEP) {
      if (first > 0) load(first);
#pragma unroll
      for (int s = 0; s < DEEP; ++s) {
        const float ws = __shfl_sync(0xffffffffu, w, (first + s) & 31);
        if (first + s < n && ws != 0.f) {
#pragma unroll
          for (int e = 0; e < E; ++e) o[e] = fmaf(ws, v[s][e], o[e]);
        }
      }
    }
  }
  bool good = true;
  const float inv = l != 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    o[e] = l != 0.f ? o[e] * inv : 0.f;
    good = good && isfinite(o[e]);
  }
  const int r = qi / G, row = c.row0 + r, head = c.kvh * G + qi - r * G;
  if (!__all_sync(0xffffffffu, good)) paged_attend_row<T, KVT, D>(P, c.b, row, c.first_seen + r, head);
  else store_pack(reinterpret_cast<T *>(P.out) + ((size_t)row * P.nq + head) * D + lane * E, o);
}

// Joins 16 dimensions from d0 on of 32 query rows from q0 on of the chunk kernel's item: a lane to a row.
template <typename T, int D>
__device__ __forceinline__ void paged_join_rows(const PagedAttentionParams &P, const PagedScratch &S, const PagedCutItem &c, int block, int q0, int d0) {
  const int lane = threadIdx.x & 31, qi = q0 + lane, G = P.nq / P.nkv;
  const bool mine = qi < c.rows * G;
  float m = -INFINITY, l = 0.f, o[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) o[e] = 0.f;
  for (int s = 0; s < c.pieces && mine; ++s) {                // two or three as a rule
    const int place = paged_place(block + s, s == 0);
    float v[4][4];
#pragma unroll
    for (int k = 0; k < 4; ++k) load_pack(S.sums<D>(place) + ((size_t)(d0 / 4 + k) * S.rows + qi) * 4, v[k]);
    const float2 ml = S.levels<D>(place)[qi];
    if (ml.x == -INFINITY) {                                   // a piece without keys: sum 0; one whose scores are all NaN: NaN
      l += ml.y;
      continue;
    }
    const float top = fmaxf(m, ml.x), old = m > -INFINITY ? exp2f(m - top) : 0.f, w = exp2f(ml.x - top);
    m = top;
    l = l * old + ml.y * w;
#pragma unroll
    for (int e = 0; e < 16; ++e) o[e] = fmaf(w, v[e / 4][e % 4], o[e] * old);
  }
  bool good = true;
  const float inv = l != 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    o[e] = l != 0.f ? o[e] * inv : 0.f;
    good = good && isfinite(o[e]);
  }
  if (mine) {
    const int r = qi / G;
    T *dst = reinterpret_cast<T *>(P.out) + ((size_t)(c.row0 + r) * P.nq + c.kvh * G + qi - r * G) * D + d0;
#pragma unroll
    for (int k = 0; k < 2; ++k) store_pack(dst + 8 * k, *reinterpret_cast<float(*)[8]>(o + 8 * k));
  }
  uint32_t bad_rows = __ballot_sync(0xffffffffu, mine && !good);
  __syncwarp();
  while (bad_rows) {
    const int i = q0 + __ffs(bad_rows) - 1, r = i / G;
    bad_rows &= bad_rows - 1;
    // (this warp's dimensions alone: those of a row in other warps may be finite, and the order of the warps is open)
    paged_attend_row<T, T, D>(P, c.b, c.row0 + r, c.first_seen + r, c.kvh * G + i - r * G, d0, d0 + 16);
  }
}

// Joins what was cut: a block to each of the row kernel's `blocks` shares, a warp to a row; then, if the chunk kernel ran
// too, per_chunk blocks to each of its shares.  Bound: two trips to memory, 3 to 4.5 us; behind the chunk kernel the partial results (35 MB), 8 us
// where most of them are still in L2 and 14 with cold caches.
constexpr int PAGED_MERGE_WARPS = 16;
template <int D> __host__ __device__ constexpr int paged_merge_per_chunk(int rows) { return rows / 32 * (D / 16) / PAGED_MERGE_WARPS; }
template <typename T, typename KVT, int D>
__global__ void __launch_bounds__(PAGED_MERGE_WARPS * 32) paged_merge_kernel(const __grid_constant__ PagedAttentionParams P, PagedScratch S, int blocks,
                                                                              PagedScratch S_chunk) {
  paged_enter();
  const int warp = threadIdx.x >> 5, G = P.nq / P.nkv;
  if ((int)blockIdx.x < blocks) {
    const PagedCutItem c = S.items[blockIdx.x];
    if (c.pieces && warp < c.rows * G) paged_join_row<T, KVT, D>(P, S, c, blockIdx.x, warp);
  } else if constexpr (std::is_same<T, KVT>::value) {
    const int per = paged_merge_per_chunk<D>(S_chunk.rows), block = (blockIdx.x - blocks) / per;
    const int task = (blockIdx.x - blocks) % per * PAGED_MERGE_WARPS + warp, q0 = task / (D / 16) * 32;
    const PagedCutItem c = S_chunk.items[block];
    if (c.pieces && q0 < c.rows * G) paged_join_rows<T, D>(P, S_chunk, c, block, q0, task % (D / 16) * 16);
  }
}

}  // namespace dmtd
