// Step a3 for a paged cache: dmtd_paged_append.  QK-norm and rotary embedding of the new rows' queries and keys, keys and
// values rounded once to the cache's type and written into their slots, queries to an array of their own.
//
//   x <- x * rsqrt(mean x^2 + eps) * w                     (where a norm is given)
//   (x[i], x[i + D/2]) <- turned by position * theta^(-2i/D)
//
// A warp takes a row, or where there are few rows a part of its vectors (queries, keys and values of all heads are one line of
// vectors), and a group of D/2 / V of its threads a vector at a time (V = 16 bytes of the activations), each thread the same V places of
// both halves: a pair to be turned is in one thread, all loads are 16 bytes wide, and a thread's cosines, sines and query norm
// stay in registers for the whole row.  The next vectors are on their way to places of the thread's own in shared memory: no barrier anywhere.
// (A block to four rows with angles and norms in L1: 49 us for 8191 rows of 32 + 2 x 8 vectors, bound by L1.)
// The angle is taken in turns of the circle, in 64 bits up to the fraction (at position 10^6 fp32 would be off by 0.06
// radians), and the fraction's cosine and sine in 32.
//
// Bound: bytes (each value is read and written once) from some thousand rows on, below that one trip to memory.  Measured: 8191 rows of
// 32 + 2 x 8 vectors of 128, bf16: 34.3 us, 5.9 TB/s; 32 rows 3.0 us.
#pragma once

#include "paged_common.cuh"

namespace dmtd {

constexpr int APPEND_THREADS = 256, APPEND_WARPS = APPEND_THREADS / 32;
constexpr int APPEND_DEPTH = 4;              // vectors of a thread that are under way
constexpr int APPEND_SMEM = APPEND_DEPTH * APPEND_THREADS * 32;

struct PagedAppendParams {
  const void *q, *k, *v;
  long long q_stride, k_stride, v_stride;    // between rows, in values
  int n_rows, nq, nkv;
  const float *q_norm, *k_norm;
  float eps;
  const int *position, *slot;
  PagedPool pool;
  void *q_out;                               // [n_rows][nq][D]
  int slices, per_slice;                     // parts of a row, and their vectors (a multiple of 32 / GROUP)
  double turns[64];                          // theta^(-2i/D) / (2 pi)
};

// ROTATE: a form of its own, since cosine 1 and sine 0 would let an infinity of one half make the other NaN, and a branch around the
// rotation costs 1.2 of 35.5 us (8191 rows).
template <typename T, typename KVT, int D, bool ROTATE>
__global__ void __launch_bounds__(APPEND_THREADS, 3) paged_append_kernel(const __grid_constant__ PagedAppendParams P) {
  constexpr int V = 16 / sizeof(T), HALF = D / 2, GROUP = HALF / V, SUBS = 32 / GROUP;
  constexpr int SHARE = V / SUBS > 0 ? V / SUBS : 1;         // angles that a thread works out; the groups share them
  extern __shared__ __align__(16) unsigned char append_smem[];               // [DEPTH][2][threads] 16 bytes
  paged_enter();
  const int lane = threadIdx.x & 31, sub = lane / GROUP, at = lane % GROUP * V;
  const int task = blockIdx.x * APPEND_WARPS + (threadIdx.x >> 5);
  const int row = P.slices == 1 ? task : task / P.slices, v0 = P.slices == 1 ? 0 : (task - row * P.slices) * P.per_slice;
  if (row >= P.n_rows) return;
  const int v1 = min(P.nq + 2 * P.nkv, v0 + P.per_slice);
  const uint32_t mine = smem_u32(append_smem) + threadIdx.x * 16;
  auto place = [&](int k, int half) { return mine + (k * 2 + half) * APPEND_THREADS * 16; };
  auto fetch = [&](int k, int vec) {
    if (vec < v1) {
      const T *src = vec < P.nq ? reinterpret_cast<const T *>(P.q) + row * P.q_stride + vec * D
                   : vec < P.nq + P.nkv ? reinterpret_cast<const T *>(P.k) + row * P.k_stride + (vec - P.nq) * D
                                        : reinterpret_cast<const T *>(P.v) + row * P.v_stride + (vec - P.nq - P.nkv) * D;
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(place(k, 0)), "l"(src + at) : "memory");
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(place(k, 1)), "l"(src + HALF + at) : "memory");
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  float wq[2][V];
  auto load_norm = [&](const float *norm, float (&w)[2][V]) {
#pragma unroll
    for (int j = 0; j < V; j += 4) {
      load_pack(norm + at + j, *reinterpret_cast<float(*)[4]>(w[0] + j));
      load_pack(norm + HALF + at + j, *reinterpret_cast<float(*)[4]>(w[1] + j));
    }
  };
  const int slot = P.slot[row], position = P.position[row];
  if (P.q_norm) load_norm(P.q_norm, wq);
#pragma unroll
  for (int k = 0; k < APPEND_DEPTH; ++k) fetch(k, v0 + k * SUBS + sub);
  if (slot < 0 || (slot >> P.pool.lg_page) >= P.pool.n_pages) {
    asm volatile("cp.async.wait_all;" ::: "memory");
    return;
  }
  float c[V], s[V];
  if constexpr (ROTATE) {
    float ca[SHARE], sa[SHARE];
#pragma unroll
    for (int j = 0; j < SHARE; ++j) {
      const double t = (double)position * P.turns[at + (sub * SHARE + j) % V];
      sincospif(2.f * (float)(t - rint(t)), &sa[j], &ca[j]);
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int from = j / SHARE * GROUP + lane % GROUP;
      c[j] = __shfl_sync(0xffffffffu, ca[j % SHARE], from);
      s[j] = __shfl_sync(0xffffffffu, sa[j % SHARE], from);
    }
  }
  const size_t cell = P.pool.at(slot >> P.pool.lg_page, 0, slot & ((1 << P.pool.lg_page) - 1)) + at;
  // (the norm's shuffles run inside a group; its threads take the same way)
  const unsigned mask = (GROUP == 32 ? 0xffffffffu : ((1u << GROUP) - 1)) << (sub * GROUP);
  for (int j0 = v0 + sub; j0 < v1; j0 += APPEND_DEPTH * SUBS) {
#pragma unroll
    for (int k = 0; k < APPEND_DEPTH; ++k) {
      const int vec = j0 + k * SUBS;
      if (vec >= v1) break;
      asm volatile("cp.async.wait_group %0;" ::"n"(APPEND_DEPTH - 1) : "memory");
      const uint4 lo = lds128(place(k, 0)), hi = lds128(place(k, 1));
      const Pack<T, V> &x = reinterpret_cast<const Pack<T, V> &>(lo), &y = reinterpret_cast<const Pack<T, V> &>(hi);
      float a[V], b[V];
#pragma unroll
      for (int j = 0; j < V; ++j) {
        a[j] = to_f32(x.v[j]);
        b[j] = to_f32(y.v[j]);
      }
      fetch(k, vec + APPEND_DEPTH * SUBS);
      const bool is_q = vec < P.nq, is_k = !is_q && vec < P.nq + P.nkv;
      if (is_q || is_k) {
        if (is_q ? P.q_norm : P.k_norm) {
          float ss = 0.f;
#pragma unroll
          for (int j = 0; j < V; ++j) ss = fmaf(a[j], a[j], fmaf(b[j], b[j], ss));
#pragma unroll
          for (int o = 1; o < GROUP; o <<= 1) ss += __shfl_xor_sync(mask, ss, o);
          const float inv = rsqrtf(ss * (1.f / D) + P.eps);
          if (is_q) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
              a[j] *= inv * wq[0][j];
              b[j] *= inv * wq[1][j];
            }
          } else {
            float wk[2][V];
            load_norm(P.k_norm, wk);
#pragma unroll
            for (int j = 0; j < V; ++j) {
              a[j] *= inv * wk[0][j];
              b[j] *= inv * wk[1][j];
            }
          }
        }
        if constexpr (ROTATE) {
#pragma unroll
          for (int j = 0; j < V; ++j) {
            const float p = a[j], q = b[j];
            a[j] = p * c[j] - q * s[j];
            b[j] = q * c[j] + p * s[j];
          }
        }
      }
      if (is_q) {
        T *dst = reinterpret_cast<T *>(P.q_out) + ((size_t)row * P.nq + vec) * D + at;
        store_pack(dst, a);
        store_pack(dst + HALF, b);
      } else {
        const int h = is_k ? vec - P.nq : vec - P.nq - P.nkv;
        KVT *dst = reinterpret_cast<KVT *>(const_cast<void *>(is_k ? P.pool.k : P.pool.v)) + cell + h * P.pool.head_stride;
        store_pack(dst, a);
        store_pack(dst + HALF, b);
      }
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

}  // namespace dmtd
