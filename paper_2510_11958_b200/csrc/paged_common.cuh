// The paged KV cache: what the kernels of paged.cu share.
//
// Requests of unequal length keep their keys and values in pages of a pool, [page][kv head][row][head_dim] or in any other
// order of those axes that strides describe; the table of a request names its pages in the order of positions.  Lengths,
// tables and row offsets live in device memory and are read by the kernels, so that a captured graph stays valid as requests
// grow; every one of them is cut to what the buffers hold before it is used.
#pragma once

#include "ptx.cuh"

namespace dmtd {

// One layer's pool.  Strides in values.
struct PagedPool {
  const void *k, *v;
  int n_pages, lg_page;                       // pages of 1 << lg_page positions
  long long page_stride, head_stride, row_stride;
  __device__ __forceinline__ long long at(int page, int kvh, int row) const {
    return page * page_stride + kvh * head_stride + row * row_stride;
  }
};

// The requests of a step: new rows [row_start[b], row_start[b + 1]) of q belong to request b, whose keys, the new ones
// among them, fill positions [0, lens[b]).
struct PagedBatch {
  const int *row_start, *lens, *table;
  int n_requests, table_stride, n_rows;
  __host__ __device__ __forceinline__ int row(int b) const { return min(max(row_start[b], 0), n_rows); }
  // keys of request b, as far as its table goes
  __host__ __device__ __forceinline__ int keys(int b, int lg_page) const {
    return (int)min((long long)max(lens[b], 0), (long long)table_stride << lg_page);
  }
};

template <typename T> __device__ __forceinline__ float to_f32(T v) { return (float)v; }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// N consecutive values from / to memory aligned to their size or to 16 bytes, whichever is less.
template <typename T, int N>
struct alignas(sizeof(T) * N < 16 ? sizeof(T) * N : 16) Pack { T v[N]; };
template <typename T, int N>
__device__ __forceinline__ void load_pack(const T *p, float (&f)[N]) {
  const Pack<T, N> x = *reinterpret_cast<const Pack<T, N> *>(p);
#pragma unroll
  for (int i = 0; i < N; ++i) f[i] = to_f32(x.v[i]);
}
template <typename T, int N>
__device__ __forceinline__ void store_pack(T *p, const float (&f)[N]) {
  Pack<T, N> x;
#pragma unroll
  for (int i = 0; i < N; ++i) x.v[i] = from_f32<T>(f[i]);
  *reinterpret_cast<Pack<T, N> *>(p) = x;
}

// Start of a kernel in a chain of dependent launches: the kernel behind this one may become resident, and nothing is read or
// written before the kernels in front of this one are complete.
__device__ __forceinline__ void paged_enter() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
}

}  // namespace dmtd
