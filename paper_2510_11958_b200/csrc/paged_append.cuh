// Step a3 for a paged cache: dmtd_paged_append.  QK-norm and rotary embedding of the new rows' queries and keys, keys and
// values rounded once to the cache's type and written into their slots, queries to an array of their own.
//
//   x <- x * rsqrt(mean x^2 + eps) * w                     (where a norm is given)
//   (x[i], x[i + D/2]) <- turned by position * theta^(-2i/D)
//
// A group of D/2 / V threads takes one vector (V = 16 bytes of the activations), each thread the same V places of both
// halves, so that a pair to be turned is in one thread and all loads are 16 bytes wide.  A block takes ROWS rows and a range of their
// vectors (queries, keys and values of all heads are one line of vectors); cosines and sines of a row are worked out once per block.
// The angle is taken in turns of the circle, in 64 bits up to the fraction (at position 10^6 fp32 would be off by 0.06
// radians), and the fraction's cosine and sine in 32.
//
// Bound: bytes (each value is read and written once) from some thousand rows on, below that one trip to memory.
#pragma once

#include "paged_common.cuh"

namespace dmtd {

constexpr int APPEND_THREADS = 256;
constexpr int APPEND_ROWS = 4;               // rows of a block, many-row form

struct PagedAppendParams {
  const void *q, *k, *v;
  long long q_stride, k_stride, v_stride;    // between rows, in values
  int n_rows, nq, nkv;
  const float *q_norm, *k_norm;
  float eps;
  int rotate;
  const int *position, *slot;
  PagedPool pool;
  void *q_out;                               // [n_rows][nq][D]
  int per_block;                             // vectors of a row to a block
  double turns[64];                          // theta^(-2i/D) / (2 pi)
};

template <typename T, typename KVT, int D, int ROWS>
__global__ void __launch_bounds__(APPEND_THREADS) paged_append_kernel(const __grid_constant__ PagedAppendParams P) {
  constexpr int V = 16 / sizeof(T), HALF = D / 2, GROUP = HALF / V;
  __shared__ float2 angle[ROWS][HALF];       // (cos, sin)
  __shared__ int slots[ROWS];
  paged_enter();
  const int r0 = blockIdx.x * ROWS;
  for (int i = threadIdx.x; i < ROWS * HALF; i += APPEND_THREADS) {
    const int r = r0 + i / HALF;
    float2 cs = make_float2(1.f, 0.f);
    if (P.rotate && r < P.n_rows) {
      const double t = (double)P.position[r] * P.turns[i % HALF];
      float s, c;
      sincospif(2.f * (float)(t - rint(t)), &s, &c);
      cs = make_float2(c, s);
    }
    angle[i / HALF][i % HALF] = cs;
  }
  if (threadIdx.x < ROWS) {
    const int r = r0 + threadIdx.x;
    const int s = r < P.n_rows ? P.slot[r] : -1;
    slots[threadIdx.x] = (s >> P.pool.lg_page) < P.pool.n_pages ? s : -1;      // (negative stays negative)
  }
  __syncthreads();
  const int n_vec = P.nq + 2 * P.nkv, v0 = blockIdx.y * P.per_block, n_here = min(P.per_block, n_vec - v0);
  const int lane = threadIdx.x % GROUP, at = lane * V;
  // (whole groups leave the loop together; the norm's shuffles run inside a group)
  const unsigned mask = (GROUP == 32 ? 0xffffffffu : ((1u << GROUP) - 1)) << (threadIdx.x % 32 / GROUP * GROUP);
  for (int i = threadIdx.x / GROUP; i < ROWS * n_here; i += APPEND_THREADS / GROUP) {
    const int lr = i / n_here, vec = v0 + i % n_here, slot = slots[lr];
    if (slot < 0) continue;
    const size_t row = r0 + lr;
    const bool is_q = vec < P.nq, is_k = !is_q && vec < P.nq + P.nkv;
    const T *src = is_q ? reinterpret_cast<const T *>(P.q) + row * P.q_stride + vec * D
                 : is_k ? reinterpret_cast<const T *>(P.k) + row * P.k_stride + (vec - P.nq) * D
                        : reinterpret_cast<const T *>(P.v) + row * P.v_stride + (vec - P.nq - P.nkv) * D;
    float a[V], b[V];
    load_pack(src + at, a);
    load_pack(src + HALF + at, b);
    if (is_q || is_k) {
      const float *w = is_q ? P.q_norm : P.k_norm;
      if (w) {
        float ss = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) ss += a[j] * a[j] + b[j] * b[j];
#pragma unroll
        for (int o = 1; o < GROUP; o <<= 1) ss += __shfl_xor_sync(mask, ss, o);
        const float inv = rsqrtf(ss / (float)D + P.eps);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          a[j] = a[j] * inv * w[at + j];
          b[j] = b[j] * inv * w[HALF + at + j];
        }
      }
#pragma unroll
      for (int j = 0; j < V; ++j) {
        const float2 cs = angle[lr][at + j];
        const float x = a[j], y = b[j];
        a[j] = x * cs.x - y * cs.y;
        b[j] = y * cs.x + x * cs.y;
      }
    }
    if (is_q) {
      T *dst = reinterpret_cast<T *>(P.q_out) + (row * P.nq + vec) * D;
      store_pack(dst + at, a);
      store_pack(dst + HALF + at, b);
    } else {
      const int h = is_k ? vec - P.nq : vec - P.nq - P.nkv;
      KVT *dst = reinterpret_cast<KVT *>(const_cast<void *>(is_k ? P.pool.k : P.pool.v)) +
                 P.pool.at(slot >> P.pool.lg_page, h, slot & ((1 << P.pool.lg_page) - 1));
      store_pack(dst + at, a);
      store_pack(dst + HALF + at, b);
    }
  }
}

}  // namespace dmtd
