// Attention of a few new rows per request over a paged cache, for every type: split-KV on mma.sync.
//
// The G query heads of a kv head for up to 16 / G new positions are the 16 rows of an MMA; every warp streams key tiles of
// its own (4 KiB of K, 4 KiB of V) through a private ring filled by its own asynchronous copies, no barrier of the
// block inside the key loop.  The ring runs on across items: the copies' place on the line of work (paged_line.cuh) is
// two tiles ahead of the arithmetic's, so that HBM is busy under an item's end and the next one's queries.  Page ids are read
// 32 at a time, long before they are needed.  Pages of fewer positions than a tile has: a lane looks up each
// key's page a tile ahead, and the lanes that copy a row ask that lane for it.
//
// Softmax.  A row's probabilities are relative to a reference that is raised only when a score lies more than 2^6 above it (as
// the first one does): in between, a tile needs no maximum over the lanes and no scaling of the sums, and the exponentials do not wait for one.
//
// Types.  16-bit queries: one product for Q K^T, two for P V, probabilities in two parts (with one, rounded as the result is, the
// error of the result is 1.4 times that of its own rounding).  fp32 queries: queries and probabilities as two fp16 or three bf16
// parts, exact to 2^-22 and 2^-24, a product per part; the cache's values are exact as they are.  fp32 cache: everything in two tf32 parts (2^-22), three products.
//
// Bound: KV bytes.  An SM's share of HBM is a tile in 360 cycles; its arithmetic takes 260 (32 MMAs) with 16-bit queries.  Measured with
// the merge, inputs cold: 8 requests of one row over up to 16 500 keys (bf16, 272 MB) 48.9 us, 5.6 TB/s; 32 x 3 rows (fp32 queries, fp16 cache,
// 157 MB) 40.6 us, 3.9 TB/s, of which 8 are the start and the merge.
#pragma once

#include <type_traits>

#include "paged_line.cuh"

namespace dmtd {

constexpr int PR_WARPS = 4;
constexpr int PR_THREADS = PR_WARPS * 32;
constexpr int PR_STAGES = 2;
constexpr int PR_HALF = 4096;                                  // bytes of a tile's K, and of its V
constexpr int PR_SLOT = 2 * PR_HALF;
constexpr int PR_ROWS = 16;                                    // query rows of an item
constexpr int PR_LEAST = 2;                                    // units of a block's share, at least: one would be an item's fixed cost alone
constexpr float PR_ABOVE = 6.f;                                // a score may lie this far (in powers of two) above its row's reference

// A piece of a block's share as the warps go through it.
struct RowsPiece {
  int b, row0, rows, kvh;            // request, first row of q, rows, kv head
  int pos, keys;                     // position of the first row; keys that the last row sees (0: the piece has no units of keys)
  int u0, u1;                        // units of keys, one at least
  int began, ends;                   // the item begins / ends in this piece
  int pieces;                        // of an item that goes on behind the share
  int last;                          // the share's last piece
};
constexpr int PR_PIECES = 5;         // in a piece, its copies get as far as the third behind it, page ids to the fourth

using RowsShare = PagedShare<PR_THREADS, 256>;
struct RowsShared {
  RowsShare::Shared line;
  PagedPiece made;                   // the last piece made, by thread 0
  long long made_end;                // ... its end on the line
  RowsPiece piece[PR_PIECES];
  float size[16];                              // powers of two of the query rows (RowsTypes::SIZED)
  uint32_t there[PR_WARPS][PR_STAGES];         // a bit per key of a ring slot
};

// Types of a launch: T queries, KVT cache.
template <typename T, typename KVT, int D>
struct RowsTypes {
  static constexpr bool TF32 = std::is_same<KVT, float>::value;
  static constexpr int PARTS = TF32 ? 2 : !std::is_same<T, float>::value ? 1 : std::is_same<KVT, __half>::value ? 2 : 3;
  static constexpr int P_PARTS = PARTS == 1 ? 2 : PARTS;       // of the probabilities
  static constexpr int ROW = D * (int)sizeof(KVT);             // bytes of a key
  static constexpr int KEYS = PR_HALF / ROW;                   // keys of a tile: 16 (8 to 32)
  static constexpr int NT = KEYS / 8;
  static constexpr int COPIES = ROW / 16;                      // 16-byte parts of a row
  static constexpr int UNIT = PR_WARPS * KEYS;                 // keys of a unit of work
  static constexpr int LG_UNIT = UNIT == 32 ? 5 : UNIT == 64 ? 6 : 7;
  // fp16 keeps its full precision down to 2^-14 and ends at 2^16: probabilities are 2^8 times their size there
  static constexpr float LIFT = std::is_same<KVT, __half>::value ? 8.f : 0.f;
  static constexpr int RAW_ROW = D * (int)sizeof(T) + 16;      // bytes of a query row as it comes; free of bank conflicts
  static constexpr int QROW = ROW + 16;                        // ... of its parts
  static constexpr int Q_PARTS = TF32 ? 1 : PARTS > 1 ? PARTS : 0;      // one part: taken from the rows as they come; tf32: the first is in registers
  static constexpr int OROW = D + 8;
  static constexpr int RAW = PR_WARPS * PR_STAGES * PR_SLOT;
  static constexpr int OS = RAW + PR_ROWS * RAW_ROW;           // the warps' outputs, over the queries' parts
  static constexpr int Q = OS;
  static constexpr int RED = OS + PR_WARPS * PR_ROWS * OROW * 4;
  static constexpr int SMEM = RED + 2 * PR_WARPS * PR_ROWS * 4;
  // fp32 queries in fp16 parts: a row is brought to the size of 1 by a power of two, which its scores are multiplied with
  static constexpr bool SIZED = PARTS == 2 && !TF32;
  static_assert(Q_PARTS * PR_ROWS * QROW <= RED - OS, "parts of the queries");
  static_assert(2 * (SMEM + 1024 + (int)sizeof(RowsShared)) <= 228 * 1024, "two blocks per SM");
};

// byte offset of 16-byte part `part` of row `row` in a tile: conflict-free for the copies, for the 16-byte operand loads of K
// (rows g, parts 4 kb + t) and for ldmatrix on V
template <int ROW>
__device__ __forceinline__ uint32_t pr_part(int row, int part) {
  return (uint32_t)(row * ROW + ((part & ~7) | ((part & 7) ^ (((row & 1) << 2) | ((row >> 1) & 3)))) * 16);
}
// ... of an fp32 V tile: lane (g, t) reads part g of rows 2 t and 2 t + 1
template <int ROW>
__device__ __forceinline__ uint32_t pr_part_v32(int row, int part) {
  return (uint32_t)(row * ROW + ((part & ~7) | ((part & 7) ^ (((row >> 1) & 3) << 1))) * 16);
}

__device__ __forceinline__ uint32_t tf32_of(float x) {
  uint32_t r;
  asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ void tf32_split(float x, uint32_t &hi, uint32_t &lo) {
  hi = tf32_of(x);
  lo = tf32_of(x - __uint_as_float(hi));
}
__device__ __forceinline__ void mma_tf32_1688(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// N 16-bit parts of a pair of values, the larger first: x = part 0 + part 1 + ...
template <class Op, int N>
__device__ __forceinline__ void split_pair(float x, float y, uint32_t (&p)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    p[i] = Op::pack2(x, y);
    const typename Op::T *h = reinterpret_cast<const typename Op::T *>(&p[i]);
    x -= Op::to_float(h[0]);
    y -= Op::to_float(h[1]);
  }
}

// Running sums of 16 query rows: lane (g, t) holds rows g and g + 8.  16-bit: n-tile j holds dimensions 8 j + 2 t, + 1;
// tf32: n-tile 4 blk + j holds dimensions 32 blk + 8 t + j, + 4.
template <int D>
struct RowsAcc {
  float m[2], l[2];                  // per row: level of the sums (powers of two), this lane's share of the sum
  float o[D / 8][4];
  __device__ __forceinline__ void clear() {
    m[0] = m[1] = -INFINITY;
    l[0] = l[1] = 0.f;
#pragma unroll
    for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  }
};

// A warp's tile of keys against the 16 query rows.  q_t: the queries in shared memory; qh: what of them is in registers.
// lim[h]: keys that row g + 8 h sees, counted from the tile's first; good: a bit per key that is there at all.
template <class C, typename KVT, int D, class QRegs>
__device__ __forceinline__ void rows_tile(RowsAcc<D> &A, uint32_t k_t, uint32_t v_t, uint32_t q_t, const QRegs &qh, const float (&scale)[2],
                                          const int (&lim)[2], uint32_t good, bool mask) {
  using Op = typename std::conditional<std::is_same<KVT, __half>::value, OpF16, OpBf16>::type;
  constexpr int NT = C::NT;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  float c[NT][4];
  if constexpr (C::TF32) {
    float lo[NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      c[j][0] = c[j][1] = c[j][2] = c[j][3] = 0.f;
      lo[j][0] = lo[j][1] = lo[j][2] = lo[j][3] = 0.f;
    }
#pragma unroll
    for (int kb = 0; kb < D / 16; ++kb) {
      const uint4 l0 = lds128(q_t + g * C::QROW + kb * 64 + t * 16), l1 = lds128(q_t + (g + 8) * C::QROW + kb * 64 + t * 16);
      const uint4 h0 = qh.v[kb][0], h1 = qh.v[kb][1];
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const uint4 k = lds128(k_t + pr_part<C::ROW>(j * 8 + g, kb * 4 + t));
        uint32_t kh[4], kl[4];
        tf32_split(__uint_as_float(k.x), kh[0], kl[0]);
        tf32_split(__uint_as_float(k.y), kh[1], kl[1]);
        tf32_split(__uint_as_float(k.z), kh[2], kl[2]);
        tf32_split(__uint_as_float(k.w), kh[3], kl[3]);
        mma_tf32_1688(c[j], h0.x, h1.x, h0.y, h1.y, kh[0], kh[1]);
        mma_tf32_1688(lo[j], h0.x, h1.x, h0.y, h1.y, kl[0], kl[1]);
        mma_tf32_1688(lo[j], l0.x, l1.x, l0.y, l1.y, kh[0], kh[1]);
        mma_tf32_1688(c[j], h0.z, h1.z, h0.w, h1.w, kh[2], kh[3]);
        mma_tf32_1688(lo[j], h0.z, h1.z, h0.w, h1.w, kl[2], kl[3]);
        mma_tf32_1688(lo[j], l0.z, l1.z, l0.w, l1.w, kh[2], kh[3]);
      }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
#pragma unroll
      for (int e = 0; e < 4; ++e) c[j][e] = (c[j][e] + lo[j][e]) * scale[e >> 1];
    }
  } else {
    float c2[NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      c[j][0] = c[j][1] = c[j][2] = c[j][3] = 0.f;
      c2[j][0] = c2[j][1] = c2[j][2] = c2[j][3] = 0.f;
    }
#pragma unroll
    for (int kb = 0; kb < D / 32; ++kb) {
      uint4 k[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j) k[j] = lds128(k_t + pr_part<C::ROW>(j * 8 + g, kb * 4 + t));
#pragma unroll
      for (int part = 0; part < C::PARTS; ++part) {
        uint4 h0, h1;
        if constexpr (C::PARTS == 1) {
          h0 = qh.v[kb][0];
          h1 = qh.v[kb][1];
        } else {
          const uint32_t at = q_t + part * PR_ROWS * C::QROW + g * C::QROW + kb * 64 + t * 16;
          h0 = lds128(at);
          h1 = lds128(at + 8 * C::QROW);
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          // the larger parts' products in sums of their own
          Op::mma(part ? c2[j] : c[j], h0.x, h1.x, h0.y, h1.y, k[j].x, k[j].y);
          Op::mma(part || C::PARTS == 1 ? c2[j] : c[j], h0.z, h1.z, h0.w, h1.w, k[j].z, k[j].w);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
#pragma unroll
      for (int e = 0; e < 4; ++e) c[j][e] = (c[j][e] + c2[j][e]) * scale[e >> 1];
    }
  }
  if (mask) {
#pragma unroll
    for (int j = 0; j < NT; ++j) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int key = j * 8 + 2 * t + (e & 1);
        if (key >= lim[e >> 1] || !((good >> key) & 1)) c[j][e] = -INFINITY;
      }
    }
  }
  float mx[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    mx[h] = fmaxf(c[0][2 * h], c[0][2 * h + 1]);
#pragma unroll
    for (int j = 1; j < NT; ++j) mx[h] = fmaxf(mx[h], fmaxf(c[j][2 * h], c[j][2 * h + 1]));
  }
  if (__any_sync(0xffffffffu, mx[0] > A.m[0] + (PR_ABOVE + C::LIFT) || mx[1] > A.m[1] + (PR_ABOVE + C::LIFT))) {
    float f[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 1));
      mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 2));
      const float level = fmaxf(mx[h] - C::LIFT, A.m[h]);
      f[h] = level > -INFINITY ? exp2_approx(A.m[h] - level) : 1.f;
      A.m[h] = level;
      A.l[h] *= f[h];
    }
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      A.o[i][0] *= f[0]; A.o[i][1] *= f[0]; A.o[i][2] *= f[1]; A.o[i][3] *= f[1];
    }
  }
#pragma unroll
  for (int j = 0; j < NT; ++j) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      // (a row without any key so far has no reference; NaN stays)
      c[j][e] = c[j][e] == -INFINITY ? 0.f : exp2_approx(c[j][e] - A.m[e >> 1]);
      A.l[e >> 1] += c[j][e];
    }
  }
  if constexpr (C::TF32) {
    // column k = t of the A operand is key 2 t, column t + 4 key 2 t + 1
    uint32_t ph[NT][4], pl[NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      tf32_split(c[j][0], ph[j][0], pl[j][0]);
      tf32_split(c[j][2], ph[j][1], pl[j][1]);
      tf32_split(c[j][1], ph[j][2], pl[j][2]);
      tf32_split(c[j][3], ph[j][3], pl[j][3]);
    }
#pragma unroll
    for (int blk = 0; blk < D / 32; ++blk) {
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const uint4 v0 = lds128(v_t + pr_part_v32<C::ROW>(j * 8 + 2 * t, blk * 8 + g));
        const uint4 v1 = lds128(v_t + pr_part_v32<C::ROW>(j * 8 + 2 * t + 1, blk * 8 + g));
        const uint32_t a[4] = {v0.x, v0.y, v0.z, v0.w}, b[4] = {v1.x, v1.y, v1.z, v1.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t ah, al, bh, bl;
          tf32_split(__uint_as_float(a[i]), ah, al);
          tf32_split(__uint_as_float(b[i]), bh, bl);
          float(&o)[4] = A.o[blk * 4 + i];
          mma_tf32_1688(o, ph[j][0], ph[j][1], ph[j][2], ph[j][3], al, bl);
          mma_tf32_1688(o, pl[j][0], pl[j][1], pl[j][2], pl[j][3], ah, bh);
          mma_tf32_1688(o, ph[j][0], ph[j][1], ph[j][2], ph[j][3], ah, bh);
        }
      }
    }
  } else {
    constexpr int KS = NT / 2;
    uint32_t p[KS][4][C::P_PARTS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
      for (int i = 0; i < 4; ++i) split_pair<Op, C::P_PARTS>(c[2 * ks + (i >> 1)][(i & 1) * 2], c[2 * ks + (i >> 1)][(i & 1) * 2 + 1], p[ks][i]);
    }
    const int mi = lane >> 3, rr = (mi & 1) * 8 + (lane & 7);
#pragma unroll
    for (int d2 = 0; d2 < D / 16; ++d2) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        uint32_t b0, b1, b2, b3;
        ldmatrix_x4_trans(v_t + pr_part<C::ROW>(ks * 16 + rr, d2 * 2 + (mi >> 1)), b0, b1, b2, b3);
#pragma unroll
        for (int part = C::P_PARTS - 1; part >= 0; --part) {
          Op::mma(A.o[2 * d2], p[ks][0][part], p[ks][1][part], p[ks][2][part], p[ks][3][part], b0, b1);
          Op::mma(A.o[2 * d2 + 1], p[ks][0][part], p[ks][1][part], p[ks][2][part], p[ks][3][part], b2, b3);
        }
      }
    }
  }
}

template <typename C, int D>
struct RowsQueries {                 // what of the queries is in registers: all (one part), or the first of two tf32 parts
  uint4 v[C::TF32 ? D / 16 : D / 32][2];
};

// Thread 0: `p`, which ends at unit `end` of the line, as the warps need it.
__device__ __forceinline__ void rows_describe(RowsPiece &d, const PagedPiece &p, long long end, const PagedCut &K, const RowsShare &share) {
  const bool any = p.key_end() > p.key_begin();
  d.b = p.r.b;
  d.row0 = p.r.row0 + p.first(K);
  d.rows = p.rows(K);
  d.kvh = p.kvh;
  d.pos = p.position(K);
  d.keys = any ? p.keys(K) : 0;
  d.u0 = any ? p.key_begin() : 0;
  d.u1 = any ? p.key_end() : 1;
  d.began = p.t0 == 0;
  d.ends = p.t1 == p.per_item;
  d.last = end >= share.end;
  d.pieces = d.last && d.began && !d.ends ? share.holder(end - 1 + (p.per_item - p.t1)) - (int)blockIdx.x + 1 : 0;
}

template <typename T, typename KVT, int D>
__global__ void __launch_bounds__(PR_THREADS, 2) paged_rows_kernel(const __grid_constant__ PagedAttentionParams P, PagedCut K, PagedScratch S,
                                                                    int behind_chunk) {
  using C = RowsTypes<T, KVT, D>;
  using Op = typename std::conditional<std::is_same<KVT, __half>::value, OpF16, OpBf16>::type;
  extern __shared__ __align__(128) unsigned char sc[];
  __shared__ RowsShared sh;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int G = P.nq / P.nkv, lg = P.pool.lg_page;
  const uint32_t g_inv = (65536 + G - 1) / G;                  // i / G == i * g_inv >> 16 for i < 16
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  // Behind the chunk kernel this one reads nothing that that kernel writes: it acquires what lies in front of both (paged_line.cuh) and
  // waits at its end, for the grids behind it.
  auto wait = [] { asm volatile("griddepcontrol.wait;" ::: "memory"); };
  auto leave = [&] {
    if (!behind_chunk) return;
    wait();
    // (a block that comes later waits for the chunk kernel, which has ended)
    if (blockIdx.x == 0 && threadIdx.x == 0) *S.entered = 0;
  };
  if (!behind_chunk || !__syncthreads_or(threadIdx.x == 0 && paged_entered(S.entered))) wait();
  RowsShare share;
  share.plan(P, K, sh.line, blockIdx.x, gridDim.x);
  if (share.begin >= share.end) {
    if (threadIdx.x == 0) S.items[blockIdx.x].pieces = 0;
    leave();
    return;
  }
  // thread 0 keeps the list of pieces five ahead, so that what a piece looks at was made before a barrier
  auto make_piece = [&](int index) {
    PagedPiece p = sh.made;
    long long end = sh.made_end;
    if (!share.next(P, K, sh.line, p, end)) return;
    end += p.t1 - p.t0;
    rows_describe(sh.piece[index % PR_PIECES], p, end, K, share);
    sh.made = p;
    sh.made_end = end;
  };
  if (threadIdx.x == 0) {
    const PagedPiece p = sh.line.first;
    sh.made = p;
    sh.made_end = share.begin + (p.t1 - p.t0);
    rows_describe(sh.piece[0], p, sh.made_end, K, share);
    for (int i = 1; i < PR_PIECES && sh.made_end < share.end; ++i) make_piece(i);
  }
  __syncthreads();
  const uint32_t ring = smem_u32(sc) + warp * PR_STAGES * PR_SLOT, raw_t = smem_u32(sc) + C::RAW, q_t = smem_u32(sc) + C::Q;
  float *const o_s = reinterpret_cast<float *>(sc + C::OS), *const red_m = reinterpret_cast<float *>(sc + C::RED);
  float *const red_l = red_m + PR_WARPS * PR_ROWS;
  const float scale = 1.4426950408889634f * rsqrtf((float)D);
  const KVT *const kb = reinterpret_cast<const KVT *>(P.pool.k), *const vb = reinterpret_cast<const KVT *>(P.pool.v);

  // ---- the copies' place: the piece, its next unit of keys, the page ids at hand
  const int copy_part = lane % C::COPIES, copy_row = lane / C::COPIES;
  constexpr int COPY_ROWS = 32 / C::COPIES;                    // rows of one instruction
  constexpr int LG_KEYS = C::KEYS == 8 ? 3 : C::KEYS == 16 ? 4 : 5;
  const bool one_page = lg >= LG_KEYS;                         // a tile lies in one page
  int ahead = 0, ahead_unit, ahead_end, ahead_keys, ahead_kvh, ahead_last;
  const int *ahead_table;
  // one_page: lane i has the id of page page0 + i, and once they are asked for of page page0 + 32 + i; else lane i has that
  // of the page of the next tile's key i.  first_ids: the same for the first tile of the piece behind
  int ids = -1, ids_next = -1, page0 = 0, first_ids = -1;
  bool asked = false;
  auto page_of = [&](const int *table, int keys, int page) { return ((long long)page << lg) < keys ? table[page] : -1; };
  auto table_of = [&](int b) { return P.batch.table + (size_t)b * P.batch.table_stride; };
  auto first_page = [&](int unit) {                            // this lane's page at the first tile of a piece
    const int key = unit * C::UNIT + warp * C::KEYS;
    return one_page ? (key >> lg) + lane : (key + (lane & (C::KEYS - 1))) >> lg;
  };
  auto ask_first = [&](int index) {
    const RowsPiece &d = sh.piece[index % PR_PIECES];
    first_ids = page_of(table_of(d.b), d.keys, first_page(d.u0));
  };
  auto enter_piece = [&](int index) {                          // its first ids are in first_ids
    const RowsPiece &d = sh.piece[index % PR_PIECES];
    ahead_unit = d.u0;
    ahead_end = d.u1;
    ahead_keys = d.keys;
    ahead_kvh = d.kvh;
    ahead_last = d.last;
    ahead_table = table_of(d.b);
    page0 = (ahead_unit * C::UNIT + warp * C::KEYS) >> lg;
    ids = first_ids;
    asked = false;
    if (!ahead_last) ask_first(index + 1);
  };
  bool ahead_on = true;
  auto fetch = [&](int slot) {
    if (ahead_on) {
      const int key0 = ahead_unit * C::UNIT + warp * C::KEYS, left = ahead_keys - key0;      // left: keys from the tile's first on
      const uint32_t dst = ring + slot * PR_SLOT;
      auto copy = [&](int row, long long src, bool real) {
        const int bytes = real ? 16 : 0;                       // what is not there is filled with zeros: 0 times stale bits must stay 0
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + pr_part<C::ROW>(row, copy_part)), "l"(kb + src), "r"(bytes) : "memory");
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                         dst + PR_HALF + (C::TF32 ? pr_part_v32<C::ROW>(row, copy_part) : pr_part<C::ROW>(row, copy_part))),
                     "l"(vb + src), "r"(bytes) : "memory");
      };
      constexpr int PER_PART = 16 / (int)sizeof(KVT);
      uint32_t mask;
      if (one_page) {
        const int id = __shfl_sync(0xffffffffu, ids, (key0 >> lg) - page0);
        const bool ok = id >= 0 && id < P.pool.n_pages;
        mask = !ok || left <= 0 ? 0 : left >= C::KEYS ? (C::KEYS == 32 ? 0xffffffffu : (1u << C::KEYS) - 1) : (1u << left) - 1;
        const long long at = ok ? P.pool.at(id, ahead_kvh, (key0 & ((1 << lg) - 1)) + copy_row) + copy_part * PER_PART : 0;
#pragma unroll
        for (int j = 0; j < C::KEYS / COPY_ROWS; ++j) {
          const int row = j * COPY_ROWS + copy_row;
          const bool real = (mask >> row) & 1;
          copy(row, real ? at + j * COPY_ROWS * P.pool.row_stride : 0, real);
        }
      } else {
        mask = __ballot_sync(0xffffffffu, lane < C::KEYS && lane < left && ids >= 0 && ids < P.pool.n_pages);
#pragma unroll
        for (int j = 0; j < C::KEYS / COPY_ROWS; ++j) {
          const int row = j * COPY_ROWS + copy_row, id = __shfl_sync(0xffffffffu, ids, row);
          const bool real = (mask >> row) & 1;
          copy(row, real ? P.pool.at(id, ahead_kvh, (key0 + row) & ((1 << lg) - 1)) + copy_part * PER_PART : 0, real);
        }
      }
      if (lane == 0) sh.there[warp][slot] = mask;
      // the next tile, and its page ids
      if (++ahead_unit == ahead_end) {
        if (ahead_last) ahead_on = false;
        else enter_piece(++ahead);
      } else if (!one_page) {
        ids = page_of(ahead_table, ahead_keys, first_page(ahead_unit));
      } else {
        const int page = (ahead_unit * C::UNIT + warp * C::KEYS) >> lg;          // (a unit spans four pages at most)
        if (page - page0 >= 32) {
          page0 += 32;
          ids = ids_next;
          asked = false;
        } else if (page - page0 >= 16 && !asked) {
          ids_next = page_of(ahead_table, ahead_keys, page0 + 32 + lane);
          asked = true;
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");       // an empty group past the share keeps the counts uniform
  };
  // a piece's query rows as they are: row qi = (row row0 + qi / G, head kvh * G + qi % G); beyond the tile's rows zero
  auto fetch_queries = [&](int index) {
    const RowsPiece &d = sh.piece[index % PR_PIECES];
    constexpr int PER_ROW = D * (int)sizeof(T) / 16;
    const T *q = reinterpret_cast<const T *>(P.q);
#pragma unroll
    for (int k = 0; k < PR_ROWS * PER_ROW / PR_THREADS; ++k) {
      const int idx = threadIdx.x + k * PR_THREADS, qi = idx / PER_ROW, part = idx % PER_ROW, r = qi * g_inv >> 16;
      const bool real = r < d.rows;
      const T *src = real ? q + (d.row0 + r) * P.q_stride + (d.kvh * G + qi - r * G) * D + part * (16 / (int)sizeof(T)) : q;
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(raw_t + qi * C::RAW_ROW + part * 16), "l"(src), "r"(real ? 16 : 0) : "memory");
    }
  };
  fetch_queries(0);                                            // (part of the first tile's group)
  ask_first(0);
  enter_piece(0);
#pragma unroll 1
  for (int s = 0; s < PR_STAGES; ++s) fetch(s);

  int slot = 0;
  bool q_behind = false;                                       // this piece's queries may be in the newest group of copies
  for (int index = 0;; ++index) {
    const RowsPiece d = sh.piece[index % PR_PIECES];
    const int nQ = d.rows * G;
    // ---- queries
    if (q_behind) asm volatile("cp.async.wait_group 0;" ::: "memory");
    else asm volatile("cp.async.wait_group %0;" ::"n"(PR_STAGES - 1) : "memory");
    __syncthreads();                                           // ... of every thread; the outputs before them have been read
    RowsQueries<C, D> qh;
    if constexpr (C::TF32) {
      // the first parts in registers, the second ones to shared memory by one warp
#pragma unroll
      for (int k = 0; k < D / 16; ++k) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint4 x = lds128(raw_t + (g + 8 * h) * C::RAW_ROW + k * 64 + t * 16);
          uint4 &y = qh.v[k][h];
          uint4 z;
          tf32_split(__uint_as_float(x.x), y.x, z.x);
          tf32_split(__uint_as_float(x.y), y.y, z.y);
          tf32_split(__uint_as_float(x.z), y.z, z.z);
          tf32_split(__uint_as_float(x.w), y.w, z.w);
          if (warp == (k & 3)) sts128(q_t + (g + 8 * h) * C::QROW + k * 64 + t * 16, z);
        }
      }
    } else if constexpr (C::PARTS == 1) {
#pragma unroll
      for (int k = 0; k < D / 32; ++k) {
        qh.v[k][0] = lds128(raw_t + g * C::RAW_ROW + k * 64 + t * 16);
        qh.v[k][1] = lds128(raw_t + (g + 8) * C::RAW_ROW + k * 64 + t * 16);
      }
    } else {
#pragma unroll
      for (int k = 0; k < PR_ROWS * D / 8 / PR_THREADS; ++k) {
        const int idx = threadIdx.x + k * PR_THREADS, qi = idx / (D / 8), at = idx % (D / 8);
        const uint4 x = lds128(raw_t + qi * C::RAW_ROW + at * 32), y = lds128(raw_t + qi * C::RAW_ROW + at * 32 + 16);
        float f[8] = {__uint_as_float(x.x), __uint_as_float(x.y), __uint_as_float(x.z), __uint_as_float(x.w),
                      __uint_as_float(y.x), __uint_as_float(y.y), __uint_as_float(y.z), __uint_as_float(y.w)};
        if constexpr (C::SIZED) {
          float most = 0.f;
#pragma unroll
          for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(f[j]));
#pragma unroll
          for (int o = 1; o < D / 8; o <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
          // the exponent of the largest, kept where 2^+-exponent is a normal number (0, infinities: any)
          const int exponent = min(max((int)(__float_as_uint(most) >> 23) - 127, -100), 100);
          const float down = __uint_as_float((uint32_t)(127 - exponent) << 23);
#pragma unroll
          for (int j = 0; j < 8; ++j) f[j] *= down;
          if (at == 0) sh.size[qi] = __uint_as_float((uint32_t)(127 + exponent) << 23);
        }
        uint32_t w[4][C::PARTS];
#pragma unroll
        for (int j = 0; j < 4; ++j) split_pair<Op, C::PARTS>(f[2 * j], f[2 * j + 1], w[j]);
#pragma unroll
        for (int part = 0; part < C::PARTS; ++part)
          sts128(q_t + (part * PR_ROWS + qi) * C::QROW + at * 16, make_uint4(w[0][part], w[1][part], w[2][part], w[3][part]));
      }
    }
    __syncthreads();                                           // parts written, rows as they came and this piece's place read
    if (!d.last) fetch_queries(index + 1);                     // (part of the next tile's group)
    q_behind = d.u1 - d.u0 < 2;
    if (threadIdx.x == 0) make_piece(index + PR_PIECES);

    // ---- keys
    RowsAcc<D> A;
    A.clear();
    const float row_scale[2] = {C::SIZED ? scale * sh.size[g] : scale, C::SIZED ? scale * sh.size[g + 8] : scale};
    const int lim0[2] = {min(d.keys, d.pos + (int)(g * g_inv >> 16) + 1), min(d.keys, d.pos + (int)((g + 8) * g_inv >> 16) + 1)};
#pragma unroll 1
    for (int i = d.u0; i < d.u1; ++i) {
      asm volatile("cp.async.wait_group %0;" ::"n"(PR_STAGES - 1) : "memory");
      __syncwarp();
      const int key0 = i * C::UNIT + warp * C::KEYS;
      const uint32_t k_t = ring + slot * PR_SLOT;
      if (key0 < d.keys) {
        const uint32_t good = sh.there[warp][slot];
        const int lim[2] = {lim0[0] - key0, lim0[1] - key0};
        rows_tile<C, KVT, D>(A, k_t, k_t + PR_HALF, q_t, qh, row_scale, lim, good,
                             key0 + C::KEYS > d.pos + 1 || good != (C::KEYS == 32 ? 0xffffffffu : (1u << C::KEYS) - 1));
      }
      __syncwarp();                                            // the slot is free
      fetch(slot);
      if (++slot == PR_STAGES) slot = 0;
    }

    // ---- the warps' results to shared memory, joined there
    if (C::Q_PARTS) __syncthreads();                           // they lie over the queries' parts
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float l = A.l[h];
      l += __shfl_xor_sync(0xffffffffu, l, 1);
      l += __shfl_xor_sync(0xffffffffu, l, 2);
      const int q = g + 8 * h;
      if (t == 0) { red_m[warp * PR_ROWS + q] = A.m[h]; red_l[warp * PR_ROWS + q] = l; }
      if (q < nQ) {
        float *row = o_s + (warp * PR_ROWS + q) * C::OROW;
#pragma unroll
        for (int j = 0; j < D / 8; ++j) {
          if constexpr (C::TF32) {
            row[(j >> 2) * 32 + 8 * t + (j & 3)] = A.o[j][2 * h];
            row[(j >> 2) * 32 + 8 * t + (j & 3) + 4] = A.o[j][2 * h + 1];
          } else {
            *reinterpret_cast<float2 *>(row + j * 8 + 2 * t) = make_float2(A.o[j][2 * h], A.o[j][2 * h + 1]);
          }
        }
      }
    }
    __syncthreads();
    const bool whole = d.began && d.ends;
    const int place = paged_place(blockIdx.x, d.began);
    bool good = true;
    for (int idx = threadIdx.x; idx < nQ * (D / 4); idx += PR_THREADS) {
      const int qi = idx / (D / 4), at = idx % (D / 4) * 4, r = qi * g_inv >> 16;
      float m = -INFINITY, l = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < PR_WARPS; ++w) m = fmaxf(m, red_m[w * PR_ROWS + qi]);
#pragma unroll
      for (int w = 0; w < PR_WARPS; ++w) {
        const float mw = red_m[w * PR_ROWS + qi];
        // a warp without keys has sum 0, one whose scores are all NaN sum NaN, which stays (a branch around the first: 43.5 us instead of
        // 41.2 for 32 requests of three rows)
        const float f = mw > -INFINITY ? exp2_approx(mw - m) : 0.f;
        const float4 v = *reinterpret_cast<const float4 *>(o_s + (w * PR_ROWS + qi) * C::OROW + at);
        l = fmaf(red_l[w * PR_ROWS + qi], f, l);
        acc[0] = fmaf(v.x, f, acc[0]); acc[1] = fmaf(v.y, f, acc[1]); acc[2] = fmaf(v.z, f, acc[2]); acc[3] = fmaf(v.w, f, acc[3]);
      }
      if (whole) {
        const float inv = l != 0.f ? 1.f / l : 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          acc[j] = l != 0.f ? acc[j] * inv : 0.f;
          good = good && isfinite(acc[j]);
        }
        store_pack(reinterpret_cast<T *>(P.out) + ((size_t)(d.row0 + r) * P.nq + d.kvh * G + qi - r * G) * D + at, acc);
      } else {
        store_pack(S.sums<D>(place) + (size_t)qi * D + at, acc);
        if (at == 0) S.levels<D>(place)[qi] = make_float2(m, l);
      }
    }
    // A row that is not finite: a probability of zero may have met an infinity or a NaN in a row of V that it does not see
    // (a later one of the same tile), or the second part of a value an infinity.  Such tiles are worked out again row by row.
    if (__syncthreads_or(!good)) {
      for (int qi = warp; qi < nQ; qi += PR_WARPS) {
        const int r = qi * g_inv >> 16;
        paged_attend_row<T, KVT, D>(P, d.b, d.row0 + r, d.pos + r + 1, d.kvh * G + qi - r * G);
      }
    }
    if (d.last) {
      if (threadIdx.x == 0) S.items[blockIdx.x] = PagedCutItem{d.pieces, d.b, d.row0, d.rows, d.pos + 1, d.kvh, {0, 0}};
      break;
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  leave();
}

}  // namespace dmtd
