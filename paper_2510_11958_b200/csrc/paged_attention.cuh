// Attention of new tokens over a paged cache: what its kernels are given, and a row worked out from the definition.
#pragma once

#include "paged_common.cuh"

namespace dmtd {

struct PagedAttentionParams {
  const void *q;
  long long q_stride;                        // between rows, in values
  void *out;                                 // [n_rows][nq][D]
  PagedBatch batch;
  PagedPool pool;
  int nq, nkv;
};

// One query row and head by one warp, from the definition: the keys it sees one by one, softmax with a running maximum.  Slow
// (a key takes some 100 cycles of latency); for rows that the tiled kernels cannot answer, see there.  Dimensions [d0, d1) are written
// (multiples of D / 32).
template <typename T, typename KVT, int D>
__device__ __noinline__ void paged_attend_row(const PagedAttentionParams &P, int b, int row, int seen, int head, int d0 = 0,
                                             int d1 = D) {
  constexpr int E = D / 32;
  const int lane = threadIdx.x & 31, kvh = head / (P.nq / P.nkv), lg = P.pool.lg_page;
  const KVT *kb = reinterpret_cast<const KVT *>(P.pool.k), *vb = reinterpret_cast<const KVT *>(P.pool.v);
  const int *table = P.batch.table + (size_t)b * P.batch.table_stride;
  float q[E], o[E], m = -INFINITY, l = 0.f;
  load_pack(reinterpret_cast<const T *>(P.q) + row * P.q_stride + head * D + lane * E, q);
#pragma unroll
  for (int e = 0; e < E; ++e) {
    q[e] *= rsqrtf((float)D);
    o[e] = 0.f;
  }
  for (int j = 0; j < seen; ++j) {
    const int page = table[j >> lg];
    if (page < 0 || page >= P.pool.n_pages) continue;
    const long long at = P.pool.at(page, kvh, j & ((1 << lg) - 1)) + lane * E;
    float k[E], v[E], s = 0.f;
    load_pack(kb + at, k);
    load_pack(vb + at, v);
#pragma unroll
    for (int e = 0; e < E; ++e) s = fmaf(q[e], k[e], s);
    s = warp_sum(s);
    if (s == -INFINITY) continue;
    if (s > m) {
      const float f = __expf(m - s);
      m = s;
      l *= f;
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] *= f;
    }
    const float p = __expf(s - m);
    l += p;
    if (isnan(l)) break;                               // the row is NaN, whatever follows
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = fmaf(p, v[e], o[e]);
  }
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = l != 0.f ? o[e] / l : 0.f;
  if (lane * E >= d0 && lane * E < d1) store_pack(reinterpret_cast<T *>(P.out) + ((size_t)row * P.nq + head) * D + lane * E, o);
}

}  // namespace dmtd
