// Attention of pieces of prompts over a paged cache on the 5th-generation tensor cores: 16-bit queries, cache of the same type.
//
// A block takes 256 query rows of one (request, kv head) - 256 / G positions x the G query heads - as two halves of 128, and
// walks the keys they see in steps of 64.  Per half and step: S = Q K^T (M = 128 rows, N = 64 keys) into one of two places in
// tensor memory, softmax by a warpgroup (a thread owns a row: no shuffles), P back into tensor memory over S as the A operand
// of O += P V.  While a half's softmax runs, its next S is there already and the tensor cores work on the other half.  (Steps
// of 128 keys have room for one S to a half: softmax and tensor cores took turns, 4125 cycles for 128 keys and 256 rows; 2048 is the tensor
// cores' least, 2560 with N = 64, which reads Q twice as often.)  Each half has an issuing warp of its own: an MMA takes a warp some 70
// cycles to issue, and one warp for both halves was the bound of it all (6130 cycles).
//
// Measured: 2000 rows over 8000 keys, 32 query heads on 8, head_dim 128, pages of 16: 258 us with the merge, 890 TFLOP/s, call after call or as a graph,
// at the 1.78 GHz that the power cap leaves; 233 us in the first milliseconds, at the full clock, which is what the figures of other forms here stand beside.  A step takes
// 2250 cycles: a softmax warp 510 for S and its maximum, 1200 for exponentials and P (800 while the other half's warps have none), 300 for its two
// barriers; an issuing warp's turn takes 1900.  (Freeing S when it is in registers, with P beside it: 254 us against 233; two threads to a row: 262 to 274.)
//
// As in the row kernel a row's reference is raised only when a score lies more than 2^6 above it; then O is read
// back and scaled.
//
// K and V tiles (atoms of 8 rows of 64 values with the 128-byte swizzle, as K-major operand of S and as N-major operand of P V) come
// through one ring, in turn, a TMA copy to a page or 32 of its rows; page ids are looked up a tile ahead.  Pages that are not there are
// copied from behind the pool's end, which fills zeros; the page that holds the last key, whose rows behind it may hold anything,
// comes by 16-byte copies that fill zeros (0 times a stale NaN would not be 0), and so does everything in pools whose pages have fewer than 8
// positions (a swizzle atom) or lie no whole number of heads apart.  (All copies 16 bytes wide, by two warps: 885 us for 2000 rows over 8000 keys, where the tensor cores
// and the softmax take 250.)  One block per SM, persistent, with an equal share of the line of work (paged_line.cuh): no tail, whatever
// the lengths are.
//
// Warps 0-3 and 4-7: softmax of the halves, queries, results; warps 8 and 9 issue their MMAs; warp 10 copies K and V; warp 11 lists the
// pieces of the block's share (what the others would need 50 registers for).  Every wait is bounded.  Rows whose result is not finite, and all
// rows of a block whose wait gave up, are worked out from the definition at the block's end, where nothing waits for them with a limit
// (chunk_again).  Tensor memory is taken before the dependent grid is let in.
#pragma once

#include <cuda.h>

#include "paged_rows.cuh"

namespace dmtd {

constexpr int PC_M = 128, PC_ROWS = 2 * PC_M;                  // query rows of a half, of an item
constexpr int PC_TK = 128, PC_LG_TK = 7;                       // keys of a tile of the ring: the unit of work
constexpr int PC_STEP = 64;                                    // keys of a step
constexpr int PC_THREADS = 384;
constexpr int PC_PIECES = 3;
constexpr int PC_BOX = 32;                                     // rows of a copy, at most
constexpr float PC_ABOVE = 6.f;
constexpr int PC_TMEM = 512;                                   // two S (P over them) and O of both halves
constexpr long long PC_WAIT_TICKS = 2000000000ll;              // about a second

using ChunkShare = PagedShare<128, 64>;

// A piece of a block's share as its warps go through it.
struct ChunkPiece {
  int b, row0, rows, kvh;            // request, first row of q, positions of the tile, kv head
  int pos, keys;                     // position of the first row; keys that the last row sees
  int u0, end[2];                    // first key tile; half h takes steps [2 u0, end[h])
  int began, ends, last;             // the item begins / ends in this piece; the share's last piece
  int pieces;                        // of an item that goes on behind the share
  int holes;                         // some page of the piece is outside the pool
  __device__ __forceinline__ int last_step() const { return max(end[0], end[1]); }
  __device__ __forceinline__ int last_tile() const { return (last_step() + 1) >> 1; }
};
__device__ __forceinline__ ChunkPiece chunk_piece(const PagedPiece &p, long long line_end, const PagedCut &K, const ChunkShare &share, int G) {
  ChunkPiece c;
  c.b = p.r.b;
  c.row0 = p.r.row0 + p.first(K);
  c.rows = p.rows(K);
  c.kvh = p.kvh;
  c.pos = p.position(K);
  c.keys = p.keys(K);
  c.u0 = p.key_begin();
  c.began = p.t0 == 0;
  c.ends = p.t1 == p.per_item;
  c.last = line_end >= share.end;
  c.pieces = c.last && c.began && !c.ends ? share.holder(line_end - 1 + (p.per_item - p.t1)) - (int)blockIdx.x + 1 : 0;
  c.holes = 0;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    // keys that the half's last row sees
    const int n = min(c.rows * G, (h + 1) * PC_M), keys = n > h * PC_M ? max(0, c.pos + (n - 1) / G + 1) : 0;
    c.end[h] = max(2 * c.u0, min(2 * p.key_end(), (int)(((unsigned)keys + PC_STEP - 1) / PC_STEP)));
  }
  return c;
}

struct ChunkShared {
  uint64_t q_full[2], s_full[2][2], p_full[2][2], o_done[2], o_full[2], full[8], empty[8], piece_full[PC_PIECES], piece_empty[PC_PIECES];
  uint32_t tmem;
  int gave_up, again;                // again: some row of a whole item is not finite
  ChunkPiece piece[PC_PIECES];
  ChunkShare::Shared line;
};

template <int D>
struct ChunkTypes {
  static constexpr int TILE = PC_TK * D * 2;
  static constexpr int Q = 0;
  static constexpr int RING = 2 * TILE;
  static constexpr int STAGES = D == 128 ? 5 : 8;
  static constexpr int SMEM = RING + STAGES * TILE;
  static_assert(SMEM + (int)sizeof(ChunkShared) <= 227 * 1024 - 16, "shared memory");
};

// A tile: swizzle atoms of 8 rows x 64 dimensions, [row / 8][dimension / 64].  Byte offset of 16-byte part `part` of row `row`
template <int D>
__device__ __forceinline__ uint32_t pc_part(int row, int part) {
  return (uint32_t)((row >> 3) * (D * 16) + (part >> 3) * 1024 + (row & 7) * 128 + (((part & 7) ^ (row & 7)) << 4));
}
template <int D>
__device__ __forceinline__ uint64_t pc_desc(uint32_t addr, uint32_t lbo) { return umma_smem_desc(addr, lbo, D * 16) | (2ull << 61); }

// Bounded wait.
__device__ __forceinline__ bool pc_wait(uint32_t bar, uint32_t parity, int *gave_up) {
  if (mbar_try_wait(bar, parity)) return true;
  const long long t0 = clock64();
#pragma unroll 1
  for (int i = 1;; ++i) {
    if (mbar_try_wait(bar, parity)) return true;
    if (i % 64 == 0 && (*reinterpret_cast<volatile int *>(gave_up) || clock64() - t0 > PC_WAIT_TICKS)) {
      *reinterpret_cast<volatile int *>(gave_up) = 1;
      return false;
    }
  }
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// The pool's K and V as arrays [cell][groups of 8 rows][D / 64][8 rows][64], cell = page * apart + kv head < cells; on: they can be
// described so, and pages hold a swizzle atom.
struct ChunkMaps {
  CUtensorMap map[2];
  int on, apart, cells;
};

// rows of a page from the group-th eighth on
__device__ __forceinline__ void tma_page(uint32_t dst, const CUtensorMap *map, int group, int cell, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %2, %2, %3, %4}], [%5];" ::"r"(dst),
               "l"(map), "r"(0), "r"(group), "r"(cell), "r"(bar)
               : "memory");
}

// The block's share once more, behind its end: rows of whole items that are not finite, a warp to a row, from the definition; where a wait
// gave up all rows, those of cut items by way of the merge, for which a sum of NaN stands for the block's part.
template <typename T, int D>
__device__ __noinline__ void chunk_again(const PagedAttentionParams &P, const PagedCut &K, const PagedScratch &S, ChunkShared &sh) {
  constexpr int E = D / 32;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, G = P.nq / P.nkv;
  const bool all = sh.gave_up;
  ChunkShare share;
  share.plan(P, K, sh.line, blockIdx.x, gridDim.x);
  PagedPiece p = sh.line.first;
  for (long long end = share.begin;;) {
    end += p.t1 - p.t0;
    const ChunkPiece c = chunk_piece(p, end, K, share, G);
    if (c.began && c.ends) {
      for (int i = warp; i < c.rows * G; i += PC_THREADS / 32) {
        const int r = i / G, head = c.kvh * G + i - r * G;
        float o[E];
        load_pack(reinterpret_cast<const T *>(P.out) + ((size_t)(c.row0 + r) * P.nq + head) * D + lane * E, o);
        bool bad = all;
#pragma unroll
        for (int e = 0; e < E; ++e) bad = bad || !isfinite(o[e]);
        if (__any_sync(0xffffffffu, bad)) paged_attend_row<T, T, D>(P, c.b, c.row0 + r, c.pos + r + 1, head);
      }
    } else if (all) {
      for (int i = threadIdx.x; i < c.rows * G; i += PC_THREADS) S.levels<D>(paged_place(blockIdx.x, c.began))[i] = make_float2(-INFINITY, NAN);
    }
    if (all && c.last && threadIdx.x == 0) S.items[blockIdx.x] = PagedCutItem{c.pieces, c.b, c.row0, c.rows, c.pos + 1, c.kvh, {0, 0}};
    if (!share.next(P, K, sh.line, p, end)) break;
  }
}

template <typename T, int D>
__global__ void __launch_bounds__(PC_THREADS, 1) paged_chunk_kernel(const __grid_constant__ PagedAttentionParams P,
                                                                    const __grid_constant__ ChunkMaps M, PagedCut K, PagedScratch S) {
  using C = ChunkTypes<D>;
  using Op = typename std::conditional<std::is_same<T, __half>::value, OpF16, OpBf16>::type;
  constexpr float LIFT = std::is_same<T, __half>::value ? 8.f : 0.f;             // see the row kernel
  extern __shared__ __align__(1024) unsigned char chunk_smem[];
  __shared__ ChunkShared sh;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int G = P.nq / P.nkv, lg = P.pool.lg_page;
  const uint32_t smem = smem_u32(chunk_smem);

  if (threadIdx.x == 0) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      mbar_init(smem_u32(&sh.q_full[h]), PC_M);
      mbar_init(smem_u32(&sh.o_done[h]), 1);                   // P V of a step
      mbar_init(smem_u32(&sh.o_full[h]), 1);                   // ... of a piece's last step (two steps may be under way then: a phase of its own)
      for (int i = 0; i < 2; ++i) {
        mbar_init(smem_u32(&sh.s_full[h][i]), 1);
        mbar_init(smem_u32(&sh.p_full[h][i]), PC_M);
      }
    }
    for (int i = 0; i < C::STAGES; ++i) {
      mbar_init(smem_u32(&sh.full[i]), 2);                      // the bytes' announcement; the copies that are not TMA's
      mbar_init(smem_u32(&sh.empty[i]), 2);                     // both halves
    }
    for (int i = 0; i < PC_PIECES; ++i) {
      mbar_init(smem_u32(&sh.piece_full[i]), 1);
      mbar_init(smem_u32(&sh.piece_empty[i]), 11);             // a lane of every warp but the one that lists them
    }
    sh.gave_up = sh.again = 0;
    fence_mbar_init();
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem)), "r"(PC_TMEM) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  // in this order: the row kernel behind does not wait for what is in front of this one, but finds it through `entered` (and no grid
  // may hold tensor memory's columns off this block while it waits)
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (blockIdx.x == 0 && threadIdx.x == 0) st_release_u32(S.entered, PAGED_ENTERED);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const uint32_t tmem = sh.tmem;
  ChunkShare share;
  share.plan(P, K, sh.line, blockIdx.x, gridDim.x);
  const bool work = share.begin < share.end;
  if (threadIdx.x == 0) S.items[blockIdx.x].pieces = 0;       // (written anew with the last piece)

  if (work) {
    // the next piece of the list; every warp but the last goes through all of them
    int n_piece = 0;
    auto take_piece = [&](ChunkPiece &c) {
      const int i = n_piece % PC_PIECES;
      const bool there = __all_sync(0xffffffffu, pc_wait(smem_u32(&sh.piece_full[i]), n_piece / PC_PIECES & 1, &sh.gave_up));
      if (there) c = sh.piece[i];
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&sh.piece_empty[i]));
      ++n_piece;
      return there;
    };
    if (warp == 11) {
      // ---- the list of pieces
      PagedPiece p = sh.line.first;
      long long end = share.begin + (p.t1 - p.t0);
      for (int n = 0;; ++n) {
        const int i = n % PC_PIECES;
        ChunkPiece c = chunk_piece(p, end, K, share, G);
        // pages outside the pool are looked for once per piece
        const int *table = P.batch.table + (size_t)c.b * P.batch.table_stride;
        const int last = min(c.keys, c.last_tile() * PC_TK) - 1;
        bool bad = false;
#pragma unroll 8
        for (int pg = (c.u0 * PC_TK >> lg) + lane; pg <= last >> lg; pg += 32) {
          const int id = table[pg];
          bad = bad || id < 0 || id >= P.pool.n_pages;
        }
        c.holes = __any_sync(0xffffffffu, bad);
        if (!__all_sync(0xffffffffu, pc_wait(smem_u32(&sh.piece_empty[i]), (n / PC_PIECES & 1) ^ 1, &sh.gave_up))) break;
        if (lane == 0) {
          sh.piece[i] = c;
          mbar_arrive(smem_u32(&sh.piece_full[i]));
        }
        __syncwarp();
        if (!share.next(P, K, sh.line, p, end)) break;
        end += p.t1 - p.t0;
      }
    } else if (warp == 10) {
      // ---- copies: K and V tiles in turn through the ring
      fence_proxy_async_global();                              // the cache's new rows were written by ordinary stores
      constexpr int PARTS = D / 8;
      const int rows_here = min(1 << lg, PC_BOX);              // of a tile, in one copy
      const int n_copies = PC_TK / rows_here;
      int n = 0;                                               // tiles so far
      bool ok = true;
      ChunkPiece c;
      while (ok && take_piece(c)) {
        const int n_keys = c.keys, end = c.last_tile();
        const int *table = P.batch.table + (size_t)c.b * P.batch.table_stride;
        // lane i: the page of keys 4 i .. 4 i + 3 of the next tile (pages of less than four positions are looked up row by row)
        auto look_up = [&](int tile) {
          const int key = tile * PC_TK + lane * 4;
          return key < n_keys ? table[key >> lg] : -1;
        };
        int ids = look_up(c.u0);
        for (int i = c.u0; ok && i < end; ++i) {
          const int ids_next = i + 1 < end ? look_up(i + 1) : -1;
          const int left = n_keys - i * PC_TK;
          // rows [0, whole) by TMA, the page that the last key shares with rows behind it and nothing else by the lanes
          const int whole = !M.on ? 0 : left >= PC_TK ? PC_TK : left / rows_here * rows_here;
          const int rest = !M.on ? PC_TK : whole < left ? min(PC_TK, whole + rows_here) : whole;          // rows [whole, rest) by the lanes
          const int row_tma = lane * rows_here, id_tma = __shfl_sync(0xffffffffu, ids, row_tma >> 2 & 31);
          const bool real = row_tma < whole && id_tma >= 0 && id_tma < P.pool.n_pages;
          const int cell = real ? id_tma * M.apart + c.kvh : M.cells;                  // behind the end: zeros
          const bool tma = M.on && lane < n_copies && (row_tma < whole || row_tma >= rest);
#pragma unroll 1
          for (int kv = 0; kv < 2; ++kv, ++n) {
            const int st = n % C::STAGES;
            ok = __all_sync(0xffffffffu, pc_wait(smem_u32(&sh.empty[st]), (n / C::STAGES & 1) ^ 1, &sh.gave_up));
            if (!ok) break;
            const uint32_t dst = smem + C::RING + st * C::TILE, bar = smem_u32(&sh.full[st]);
            if (lane == 0) mbar_expect_tx(bar, (PC_TK - (rest - whole)) * D * (int)sizeof(T));
            __syncwarp();
            if (tma) tma_page(dst + row_tma * (D * 2), &M.map[kv], ((i * PC_TK + row_tma) & ((1 << lg) - 1)) >> 3, cell, bar);
            if (rest > whole) {
              const T *src = reinterpret_cast<const T *>(kv ? P.pool.v : P.pool.k) + c.kvh * P.pool.head_stride;
#pragma unroll 4
              for (int j = lane; j < (rest - whole) * PARTS; j += 32) {
                const int row = whole + j / PARTS, part = j % PARTS, key = i * PC_TK + row;
                const int id = key < n_keys ? table[key >> lg] : -1;
                const bool real = id >= 0 && id < P.pool.n_pages;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + pc_part<D>(row, part)),
                             "l"(real ? src + id * P.pool.page_stride + (key & ((1 << lg) - 1)) * P.pool.row_stride + part * 8 : src), "r"(real ? 16 : 0)
                             : "memory");
              }
              asm volatile("cp.async.wait_all;" ::: "memory");
              fence_proxy_async();
              __syncwarp();
            }
            if (lane == 0) mbar_arrive(bar);
          }
          ids = ids_next;
        }
        if (c.last) break;
      }
      // leave no copy in flight: the last tiles of a block that gave up get a bounded wait
      if (!ok && lane == 0) {
        for (int k = max(0, n - C::STAGES); k < n; ++k) {
          const long long t0 = clock64();
          while (!mbar_try_wait(smem_u32(&sh.full[k % C::STAGES]), k / C::STAGES & 1))
            if (clock64() - t0 > PC_WAIT_TICKS) break;
        }
      }
      __syncwarp();
    } else if (warp >= 8) {
      // ---- MMAs of a half
      const int h = warp - 8;
      constexpr uint32_t fmt = std::is_same<T, __half>::value ? 0u : 1u;
      const uint32_t idesc_s = (1u << 4) | (fmt << 7) | (fmt << 10) | ((PC_STEP >> 3) << 17) | ((PC_M >> 4) << 24);
      const uint32_t idesc_o = (1u << 4) | (fmt << 7) | (fmt << 10) | (1u << 16) | ((D >> 3) << 17) | ((PC_M >> 4) << 24);
      const uint32_t t_s = tmem + h * 128, t_o = tmem + 256 + h * 128;
      const uint64_t q_desc = pc_desc<D>(smem + C::Q + h * C::TILE, 16);
      int st = 0, ph = 0, q_ph = 0, o_ph = 0, p_ph = 0, n_pv = 0;          // p_ph: a bit per place; n_pv: P V so far
      bool ok = true, used = false;                            // used: the half had steps in the piece before
      auto all = [&](bool x) { return __all_sync(0xffffffffu, x); };
      auto commit = [&](uint64_t &bar) {
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(&bar)) : "memory");
      };
      auto scores = [&](int slot, int j) {                     // step j: a half of the tile in `slot`
        const uint64_t k_desc = pc_desc<D>(smem + C::RING + slot * C::TILE + (j & 1) * PC_STEP * D * 2, 16);
        const uint32_t d = t_s + (j & 1) * PC_STEP;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) {
          const uint64_t off = ((kk >> 2) * 1024 + (kk & 3) * 32) >> 4;
          asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
                       "l"(q_desc + off), "l"(k_desc + off), "r"(idesc_s), "r"(kk > 0 ? 1u : 0u)
                       : "memory");
        }
        commit(sh.s_full[h][j & 1]);
      };
      auto values = [&](int slot, int j, bool first, bool last) {
        const uint64_t v_desc = pc_desc<D>(smem + C::RING + slot * C::TILE + (j & 1) * PC_STEP * D * 2, 1024);
        const uint32_t p = t_s + (j & 1) * PC_STEP;
#pragma unroll
        for (int kk = 0; kk < PC_STEP / 16; ++kk)
          asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(t_o),
                       "r"(p + kk * 8), "l"(v_desc + kk * (D * 32 >> 4)), "r"(idesc_o), "r"(first && kk == 0 ? 0u : 1u)
                       : "memory");
        commit(sh.o_done[h]);
        if (last) commit(sh.o_full[h]);
      };
      ChunkPiece c;
      while (ok && take_piece(c)) {
        const int j0 = 2 * c.u0, end = h ? c.end[1] : c.end[0], n_tiles = c.last_tile() - c.u0;
        // The ring holds the piece's tiles as K, V, K, V ...; this half needs the first `mine` of each, and lets the others go.
        const int mine = ((end + 1) >> 1) - c.u0;
        const int st0 = st, ph0 = ph;
        auto place_of = [&](int i, int &slot, int &phase) {    // tile i of the piece
          const int k = st0 + i;
          slot = k % C::STAGES;
          phase = ph0 ^ (k / C::STAGES & 1);
        };
        auto take_tile = [&](int i) {
          int slot, phase;
          place_of(i, slot, phase);
          ok = ok && all(pc_wait(smem_u32(&sh.full[slot]), phase, &sh.gave_up));
          return slot;
        };
        // the piece before has left both places of S
        if (used) {
          ok = ok && all(pc_wait(smem_u32(&sh.o_full[h]), o_ph, &sh.gave_up));
          o_ph ^= 1;
        }
        used = end > j0;
        if (used) {
          ok = ok && all(pc_wait(smem_u32(&sh.q_full[h]), q_ph, &sh.gave_up));
          q_ph ^= 1;
          int k_slot = take_tile(0), v_slot = 0;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          if (ok && elect_one()) {
            scores(k_slot, j0);
            if (j0 + 1 < end) scores(k_slot, j0 + 1);
            commit(sh.empty[k_slot]);
          }
          __syncwarp();
          for (int j = j0; ok && j < end; ++j) {
            if ((j & 1) == 0) v_slot = take_tile(j - j0 + 1);
            ok = ok && all(pc_wait(smem_u32(&sh.p_full[h][j & 1]), p_ph >> (j & 1) & 1, &sh.gave_up));
            p_ph ^= 1 << (j & 1);
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            if (ok && elect_one()) {
              values(v_slot, j, j == j0, j + 1 == end);
              if ((j & 1) || j + 1 == end) commit(sh.empty[v_slot]);
            }
            __syncwarp();
            ++n_pv;
            if (j + 2 < end) {
              // S of a step goes where P of the second step before lies: behind the end of that P V
              if ((j & 1) == 0) k_slot = take_tile(j - j0 + 2);
              ok = ok && all(pc_wait(smem_u32(&sh.o_done[h]), (n_pv - 1) & 1, &sh.gave_up));
              asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
              if (ok && elect_one()) {
                scores(k_slot, j + 2);
                if ((j & 1) || j + 3 == end) commit(sh.empty[k_slot]);
              }
              __syncwarp();
            }
          }
        }
        for (int i = 2 * mine; ok && i < 2 * n_tiles; ++i) {
          int slot, phase;
          place_of(i, slot, phase);
          ok = all(pc_wait(smem_u32(&sh.full[slot]), phase, &sh.gave_up));
          if (ok && lane == 0) mbar_arrive(smem_u32(&sh.empty[slot]));
          __syncwarp();
        }
        place_of(2 * n_tiles, st, ph);
        if (c.last) break;
      }
    } else {
      // ---- softmax: thread = query row = lane of tensor memory
      const int h = warp >> 2, row = threadIdx.x & 127, qi = h * PC_M + row;
      const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
      const uint32_t t_s = tmem + h * 128 + lane_off, t_o = tmem + 256 + h * 128 + lane_off;
      const float scale = 1.4426950408889634f * rsqrtf((float)D);
      const int my_p = qi / G, my_g = qi - my_p * G;           // position in the tile, head of the group
      auto has_steps = [&](const ChunkPiece &c) { return (h ? c.end[1] : c.end[0]) > 2 * c.u0; };
      // this half's rows of a piece into shared memory (beyond the tile's rows zero), if it has steps there
      auto fetch_queries = [&](const ChunkPiece &c) {
        if (!has_steps(c)) return;
        constexpr int PARTS = D / 8, AT_ONCE = 128 / PARTS;
        const int part = row % PARTS, nQ = c.rows * G;
        const T *q = reinterpret_cast<const T *>(P.q);
#pragma unroll 4
        for (int r0 = 0; r0 < PC_M; r0 += AT_ONCE) {
          const int r = r0 + row / PARTS, i = h * PC_M + r, p = i / G;
          const bool real = i < nQ;
          asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem + C::Q + h * C::TILE + pc_part<D>(r, part)),
                       "l"(real ? q + (c.row0 + p) * P.q_stride + (c.kvh * G + i - p * G) * D + part * 8 : q), "r"(real ? 16 : 0)
                       : "memory");
        }
      };
      auto publish_queries = [&](const ChunkPiece &c) {
        if (!has_steps(c)) return;
        asm volatile("cp.async.wait_all;" ::: "memory");
        fence_proxy_async();
        mbar_arrive(smem_u32(&sh.q_full[h]));
      };
      int s_ph = 0, o_ph = 0, n_done = 0;                      // s_ph: a bit per place; n_done: P V so far
      ChunkPiece c, next;
      bool ok = take_piece(c);
      if (ok) {
        fetch_queries(c);
        publish_queries(c);
      }
      while (ok) {
        const int j0 = 2 * c.u0, end = h ? c.end[1] : c.end[0], nQ = c.rows * G;
        const int seen = qi < nQ ? c.pos + my_p + 1 : 0;
        float m = -INFINITY, l = 0.f;
        if (j0 == end && !c.last) {
          ok = take_piece(next);
          if (!ok) break;
          fetch_queries(next);
        }
        for (int j = j0; j < end; ++j) {
          ok = __all_sync(0xffffffffu, pc_wait(smem_u32(&sh.s_full[h][j & 1]), s_ph >> (j & 1) & 1, &sh.gave_up));
          s_ph ^= 1 << (j & 1);
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t t_here = t_s + (j & 1) * PC_STEP;
          uint32_t s[PC_STEP];
          tmem_ld32(t_here, *reinterpret_cast<uint32_t(*)[32]>(s));
          tmem_ld32(t_here + 32, *reinterpret_cast<uint32_t(*)[32]>(s + 32));
          asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
          if (j + 1 == end && !c.last) {                       // the half's last S is computed: its queries may go
            ok = take_piece(next);
            if (!ok) break;
            fetch_queries(next);
          }
          const int lim = seen - j * PC_STEP;                  // keys of the step that this row sees
          if (__any_sync(0xffffffffu, lim < PC_STEP)) {
#pragma unroll
            for (int k = 0; k < PC_STEP; ++k) s[k] = k < lim ? s[k] : 0xff800000u;
          }
          if (c.holes) {
            const int *table = P.batch.table + (size_t)c.b * P.batch.table_stride;
#pragma unroll
            for (int k0 = 0; k0 < PC_STEP; k0 += 32) {
              const int key = j * PC_STEP + k0 + lane, id = key < c.keys ? table[key >> lg] : -1;
              const uint32_t good = __ballot_sync(0xffffffffu, id >= 0 && id < P.pool.n_pages);
#pragma unroll
              for (int k = 0; k < 32; ++k) s[k0 + k] = (good >> k) & 1 ? s[k0 + k] : 0xff800000u;
            }
          }
          float mx[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) mx[k] = fmaxf(__uint_as_float(s[k]), __uint_as_float(s[k + 4]));
#pragma unroll
          for (int k = 8; k < PC_STEP; k += 8) {
#pragma unroll
            for (int i = 0; i < 4; ++i) mx[i] = max3(mx[i], __uint_as_float(s[k + i]), __uint_as_float(s[k + 4 + i]));
          }
          const float top = fmaxf(max3(mx[0], mx[1], mx[2]), mx[3]) * scale;
          const bool grow = top > m + (PC_ABOVE + LIFT);
          if (__any_sync(0xffffffffu, grow)) {
            float alpha = 1.f;
            if (grow) {
              alpha = exp2_approx(m - (top - LIFT));
              m = top - LIFT;
              l *= alpha;
            }
            if (j > j0) {
              // P V of the step before may be under way (the one before that is complete: S of this step was issued behind it)
              ok = __all_sync(0xffffffffu, pc_wait(smem_u32(&sh.o_done[h]), (n_done - 1) & 1, &sh.gave_up));
              if (!ok) break;
              asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll 1
              for (int c0 = 0; c0 < D; c0 += 16) {
                uint32_t o[16];
                tmem_ld16(t_o + c0, o);
                asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
                for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * alpha);
                tmem_st16(t_o + c0, o);
              }
            }
          }
          const float ref = m > -INFINITY ? m : 0.f;
          const uint64_t scale2 = f2_pack(scale, scale), ref2 = f2_pack(-ref, -ref);
          uint64_t sum[2] = {0ull, 0ull};
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            uint32_t p[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              float a, b;
              f2_unpack(f2_fma(f2_pack(__uint_as_float(s[32 * q + 2 * k]), __uint_as_float(s[32 * q + 2 * k + 1])), scale2, ref2), a, b);
              a = exp2_approx(a);
              b = exp2_approx(b);
              sum[k & 1] = f2_add(sum[k & 1], f2_pack(a, b));
              p[k] = Op::pack2(a, b);
            }
            tmem_st16(t_here + 16 * q, p);
          }
          asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          mbar_arrive(smem_u32(&sh.p_full[h][j & 1]));
          ++n_done;
          float l0, l1;
          f2_unpack(f2_add(sum[0], sum[1]), l0, l1);
          l += l0 + l1;
        }
        if (ok && !c.last) publish_queries(next);                  // (S of the next piece under the results of this one)

        // ---- results
        const bool any = end > j0, whole = c.began && c.ends;
        if (any && ok) {
          ok = __all_sync(0xffffffffu, pc_wait(smem_u32(&sh.o_full[h]), o_ph, &sh.gave_up));
          o_ph ^= 1;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        }
        const int head = c.kvh * G + my_g, place = paged_place(blockIdx.x, c.began);
        const float inv = !ok ? NAN : l != 0.f ? 1.f / l : 0.f;
        bool good = true;
        if (!whole && qi < nQ) S.levels<D>(place)[qi] = make_float2(ok ? m : 0.f, ok ? l : NAN);
#pragma unroll 1
        for (int c0 = 0; c0 < D; c0 += 32) {
          uint32_t o[32];
          if (any) {
            tmem_ld32(t_o + c0, o);
            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
          }
          if (qi < nQ) {
            float f[32];
#pragma unroll
            for (int k = 0; k < 32; ++k) f[k] = any && l != 0.f ? __uint_as_float(o[k]) : 0.f;
            if (whole) {
#pragma unroll
              for (int k = 0; k < 32; ++k) {
                f[k] *= inv;
                good = good && isfinite(f[k]);
              }
              T *dst = reinterpret_cast<T *>(P.out) + ((size_t)(c.row0 + my_p) * P.nq + head) * D + c0;
#pragma unroll
              for (int k = 0; k < 4; ++k) store_pack(dst + 8 * k, *reinterpret_cast<float(*)[8]>(f + 8 * k));
            } else {
              // four dimensions of all rows after the other: the lanes' values lie side by side
              float *dst = S.sums<D>(place) + ((size_t)(c0 / 4) * PC_ROWS + qi) * 4;
#pragma unroll
              for (int k = 0; k < 8; ++k) store_pack(dst + (size_t)k * PC_ROWS * 4, *reinterpret_cast<float(*)[4]>(f + 4 * k));
            }
          }
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        // rows that are not finite (see the row kernel) wait for the share's end.  (A thread storing for itself, without the vote: 267 us
        // instead of 260 for 2000 rows over 8000 keys, by the rest of the loop's code)
        if (ok) {
          const uint32_t bad_rows = __ballot_sync(0xffffffffu, !good);
          __syncwarp();
          if (bad_rows) sh.again = 1;
        }
        if (c.last || !ok) {
          if (c.last && threadIdx.x == 0) S.items[blockIdx.x] = PagedCutItem{c.pieces, c.b, c.row0, c.rows, c.pos + 1, c.kvh, {0, 0}};
          break;
        }
        c = next;
      }
    }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  if (warp == 8) {
    // Tensor memory is not given back under an MMA.  At a share's end none is left; those that a block had issued when a wait gave up
    // take some microseconds, whatever the wait was for: they get 100.  (A commit and a wait for it: 263 us instead of 260.)
    for (int i = 0; i < 100 * sh.gave_up; ++i) __nanosleep(1000);
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(PC_TMEM) : "memory");
  }
  if (work && (sh.again || sh.gave_up)) chunk_again<T, D>(P, K, S, sh);
}

}  // namespace dmtd
