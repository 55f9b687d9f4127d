// Host side of the paged KV cache's calls (include/dmtd.h): checks of arguments, launches.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include "host.h"
#include "paged_append.cuh"
#include "paged_plan.cuh"
#include "paged_chunk.cuh"

using namespace dmtd;

namespace {

dmtd_status launched(cudaError_t e, const char *what) {
  if (e == cudaSuccess) e = cudaGetLastError();
  return e == cudaSuccess ? DMTD_OK : call_failed(DMTD_ERR_CUDA, "%s: launch failed: %s", what, cudaGetErrorString(e));
}

constexpr int APPEND_LEAST_WARPS = 2000;

size_t dtype_bytes(int t) { return t == DMTD_F32 ? 4 : 2; }
bool known_dtype(int t) { return t == DMTD_F32 || t == DMTD_BF16 || t == DMTD_F16; }
bool aligned16(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

// Positions to a page as a power of two; -1: it is none.
int page_log2(int32_t page_size) {
  return page_size >= 1 && (page_size & (page_size - 1)) == 0 ? 31 - __builtin_clz((unsigned)page_size) : -1;
}

dmtd_status pool_check(const char *what, const dmtd_paged_cache *c, PagedPool *out) {
  if (!c || !c->k || !c->v || c->n_pages < 1) return call_failed(DMTD_ERR_INVALID_ARG, "%s: null cache or no pages", what);
  if (!known_dtype(c->dtype)) return call_failed(DMTD_ERR_SHAPE, "%s: cache dtype", what);
  if (c->head_dim != 64 && c->head_dim != 128) return call_failed(DMTD_ERR_SHAPE, "%s: head_dim must be 64 or 128", what);
  if (c->n_kv_heads < 1) return call_failed(DMTD_ERR_SHAPE, "%s: n_kv_heads", what);
  const int lg = page_log2(c->page_size);
  if (lg < 0) return call_failed(DMTD_ERR_SHAPE, "%s: page_size must be a power of two", what);
  if ((int64_t)c->n_pages << lg > INT32_MAX) return call_failed(DMTD_ERR_CAPACITY, "%s: more than 2^31 - 1 slots", what);
  *out = PagedPool{c->k, c->v, c->n_pages, lg, c->page_stride, c->head_stride, c->row_stride};
  if (c->n_pages == 1) out->page_stride = 0;             // (the stride of an axis of one means nothing)
  if (c->n_kv_heads == 1) out->head_stride = 0;
  if (c->page_size == 1) out->row_stride = 0;
  const int64_t unit = 16 / dtype_bytes(c->dtype);
  const int64_t least = c->head_dim;
  if ((c->n_pages > 1 && c->page_stride < least) || (c->n_kv_heads > 1 && c->head_stride < least) || (c->page_size > 1 && c->row_stride < least))
    return call_failed(DMTD_ERR_INVALID_ARG, "%s: a stride of the cache is shorter than a row", what);
  if (!aligned16(c->k) || !aligned16(c->v) || out->page_stride % unit || out->head_stride % unit || out->row_stride % unit)
    return call_failed(DMTD_ERR_INVALID_ARG, "%s: the cache's rows must begin on 16-byte boundaries", what);
  return DMTD_OK;
}

template <int D, bool ROTATE>
cudaError_t append_launch(const PagedAppendParams &P, int act, int kv, int blocks, cudaStream_t stream) {
  auto go = [&](auto kernel) { return launch_pdl(kernel, dim3(blocks), dim3(APPEND_THREADS), APPEND_SMEM, stream, P); };
  auto by_kv = [&](auto t) {
    using T = decltype(t);
    return kv == DMTD_F32 ? go(paged_append_kernel<T, float, D, ROTATE>)
         : kv == DMTD_BF16 ? go(paged_append_kernel<T, __nv_bfloat16, D, ROTATE>) : go(paged_append_kernel<T, __half, D, ROTATE>);
  };
  return act == DMTD_F32 ? by_kv(float{}) : act == DMTD_BF16 ? by_kv(__nv_bfloat16{}) : by_kv(__half{});
}

int sm_count() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
  return n;
}

// Scratch: the places of the row kernel's blocks, then those of the chunk kernel's, then a word (paged_line.cuh).
constexpr int ROWS_BLOCKS = 304, CHUNK_BLOCKS = 152;
constexpr size_t scratch_part(int blocks, int rows) { return (blocks * (sizeof(PagedCutItem) + 2ull * rows * 130 * 4) + 255) / 256 * 256; }
constexpr size_t SCRATCH_ENTERED = scratch_part(ROWS_BLOCKS, PR_ROWS) + scratch_part(CHUNK_BLOCKS, PC_ROWS);
static_assert(SCRATCH_ENTERED + 256 <= DMTD_PAGED_ATTENTION_SCRATCH_BYTES, "scratch");
PagedScratch scratch_at(void *scratch, size_t offset, int blocks, int rows) {
  unsigned char *const at = static_cast<unsigned char *>(scratch);
  PagedCutItem *items = reinterpret_cast<PagedCutItem *>(at + offset);
  return PagedScratch{items, reinterpret_cast<float *>(items + blocks), rows, reinterpret_cast<unsigned *>(at + SCRATCH_ENTERED)};
}

// The pool as TMA sees it: [page and kv head][groups of 8 rows][64 dimensions][8 rows][64 values of them], up to 32 rows of a page with
// all their dimensions to a copy (a small copy takes its SM some 100 cycles whatever its size: two of 64 dimensions each cost 330 us for
// 2000 rows over 8000 keys in pages of 8, now 236; whole pages of 128 rows come later than four parts of them, 244 against 232).
using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                 const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled() {
  static const EncodeTiled f = [] {
    void *p = nullptr;
    cudaDriverEntryPointQueryResult found;
    return cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found) == cudaSuccess && found == cudaDriverEntryPointSuccess
               ? reinterpret_cast<EncodeTiled>(p) : nullptr;
  }();
  return f;
}
ChunkMaps chunk_maps(const PagedPool &pool, int nkv, int D, bool f16) {
  ChunkMaps m{};
  // page and head are one axis: pages are a whole number of heads apart
  if (pool.lg_page < 3 || !encode_tiled()) return m;
  const long long head = nkv > 1 ? pool.head_stride : pool.n_pages > 1 ? pool.page_stride : D;
  const long long apart = pool.n_pages > 1 ? pool.page_stride / head : 1, cells = (pool.n_pages - 1) * apart + nkv;
  if ((pool.n_pages > 1 && pool.page_stride % head) || cells > INT32_MAX) return m;
  const cuuint64_t row = pool.row_stride * 2;
  const cuuint64_t dims[5] = {64, 8, (cuuint64_t)D / 64, 1ull << (pool.lg_page - 3), (cuuint64_t)cells};
  const cuuint64_t strides[4] = {row, 128, 8 * row, (cuuint64_t)head * 2};
  const cuuint32_t box[5] = {64, 8, (cuuint32_t)D / 64, (cuuint32_t)std::min(1 << pool.lg_page, PC_BOX) / 8, 1}, step[5] = {1, 1, 1, 1, 1};
  const void *base[2] = {pool.k, pool.v};
  m.on = 1;
  m.apart = (int)apart;
  m.cells = (int)cells;
  for (int i = 0; i < 2; ++i)
    if (encode_tiled()(&m.map[i], f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void *>(base[i]), dims, strides, box,
                       step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                       CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      m.on = 0;                                          // (strides that TMA cannot hold: 16-byte copies)
  return m;
}

// Requests with at least this many query rows to a kv head go to the chunk kernel, which takes the same time for 16 and for
// 128 of them; the row kernel reads the keys anew for every 16.  us, chunk / row kernel, bf16, head_dim 128, 8 kv heads: 8 requests x
// 4000 keys 48 / 42 with 32 rows, 49 / 57 with 48; 32 x 1000 keys 52 / 48 and 53 / 63; one request x 1000 keys 19 / 13 and 20 / 14 (the
// lengths are not known here).  head_dim 64: 8 x 4000 keys 41 / 40 with 48 rows, 41 / 50 with 64.
constexpr int chunk_least_rows(int D) { return D == 128 ? 33 : 49; }

template <typename T, int D>
cudaError_t chunk_launch(const PagedAttentionParams &P, int min_new, const PagedScratch &S, int blocks, cudaStream_t stream) {
  using C = ChunkTypes<D>;
  const auto kernel = paged_chunk_kernel<T, D>;
  const PagedCut K = paged_cut(PC_ROWS / (P.nq / P.nkv), PC_LG_TK, min_new, INT32_MAX, 2);
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
  if (e == cudaSuccess) e = launch_pdl(kernel, dim3(blocks), dim3(PC_THREADS), C::SMEM, stream, P,
                                        chunk_maps(P.pool, P.nkv, D, std::is_same<T, __half>::value), K, S);
  return e;
}

template <typename T, typename KVT, int D>
cudaError_t attention_launch_t(const PagedAttentionParams &P, int max_new, void *scratch, int n_sms, cudaStream_t stream) {
  using C = RowsTypes<T, KVT, D>;
  const int G = P.nq / P.nkv, blocks = std::min(2 * n_sms, ROWS_BLOCKS);
  PagedCut K = paged_cut(PR_ROWS / G, C::LG_UNIT, 1, INT32_MAX, PR_LEAST);
  const PagedScratch S = scratch_at(scratch, 0, ROWS_BLOCKS, PR_ROWS);
  const PagedScratch S_chunk = scratch_at(scratch, scratch_part(ROWS_BLOCKS, PR_ROWS), CHUNK_BLOCKS, PC_ROWS);
  int chunk_blocks = 0;
  cudaError_t e = cudaSuccess;
  if constexpr (std::is_same<T, KVT>::value && !std::is_same<T, float>::value) {
    const int min_new = (chunk_least_rows(D) + G - 1) / G;
    if (max_new >= min_new) {
      chunk_blocks = std::min(n_sms, CHUNK_BLOCKS);
      e = chunk_launch<T, D>(P, min_new, S_chunk, chunk_blocks, stream);
      K.max_new = min_new - 1;
    }
  }
  if (e == cudaSuccess) e = cudaFuncSetAttribute(paged_rows_kernel<T, KVT, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::SMEM);
  if (e == cudaSuccess)
    e = launch_pdl(paged_rows_kernel<T, KVT, D>, dim3(blocks), dim3(PR_THREADS), C::SMEM, stream, P, K, S, chunk_blocks > 0);
  if (e == cudaSuccess)
    e = launch_pdl(paged_merge_kernel<T, KVT, D>, dim3(blocks + chunk_blocks * paged_merge_per_chunk<D>(PC_ROWS)), dim3(PAGED_MERGE_WARPS * 32), 0, stream, P, S,
                   blocks, S_chunk);
  return e;
}

template <int D>
cudaError_t attention_launch(const PagedAttentionParams &P, int qt, int kv, int max_new, void *scratch, int n_sms, cudaStream_t stream) {
  if (qt == DMTD_BF16) return attention_launch_t<__nv_bfloat16, __nv_bfloat16, D>(P, max_new, scratch, n_sms, stream);
  if (qt == DMTD_F16) return attention_launch_t<__half, __half, D>(P, max_new, scratch, n_sms, stream);
  if (kv == DMTD_F32) return attention_launch_t<float, float, D>(P, max_new, scratch, n_sms, stream);
  return kv == DMTD_BF16 ? attention_launch_t<float, __nv_bfloat16, D>(P, max_new, scratch, n_sms, stream)
                         : attention_launch_t<float, __half, D>(P, max_new, scratch, n_sms, stream);
}

}  // namespace

extern "C" {

dmtd_status dmtd_paged_plan(const int32_t *lens, const int32_t *n_new, int32_t n_requests, int32_t page_size, int32_t *table,
                            int32_t table_stride, int32_t *free_pages, int32_t n_pages, const int32_t *n_free, int32_t n_rows,
                            int32_t *row_start, int32_t *position, int32_t *slot, int32_t *granted, int32_t *lens_out,
                            int32_t *n_free_out, void *cuda_stream) {
  if (n_requests < 0 || n_rows < 0 || n_pages < 1 || table_stride < 1)
    return call_failed(DMTD_ERR_INVALID_ARG, "paged_plan: negative or zero size");
  if (!free_pages || !n_free || !row_start || !n_free_out || (n_requests && (!lens || !n_new || !table || !granted || !lens_out)) ||
      (n_rows && (!position || !slot)))
    return call_failed(DMTD_ERR_INVALID_ARG, "paged_plan: null pointer");
  const int lg = page_log2(page_size);
  if (lg < 0) return call_failed(DMTD_ERR_SHAPE, "paged_plan: page_size must be a power of two");
  if (n_requests > PLAN_MAX_REQUESTS) return call_failed(DMTD_ERR_CAPACITY, "paged_plan: more than %d requests", PLAN_MAX_REQUESTS);
  if (((int64_t)n_pages << lg) > INT32_MAX || n_pages >= PLAN_MOST || n_rows >= PLAN_MOST || (int64_t)n_requests * table_stride >= PLAN_MOST)
    return call_failed(DMTD_ERR_CAPACITY, "paged_plan: more than 2^31 - 1 slots, or 2^30 rows or table entries");
  const bool fill = n_rows <= 16384;
  const PagedPlanParams P{lens, n_new, n_requests, lg, table, table_stride, free_pages, n_pages, n_free, n_rows,
                          row_start, position, slot, granted, lens_out, n_free_out, fill};
  const int smem = plan_smem_bytes(n_requests);
  cudaError_t e = cudaSuccess;
  if (smem > 48 * 1024) e = cudaFuncSetAttribute(paged_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return call_failed(DMTD_ERR_CUDA, "paged_plan: %s", cudaGetErrorString(e));
  // few requests: few warps, whose scans are the shorter ones
  const int ranks = n_rows > PLAN_THREADS || n_requests > PLAN_THREADS ? PLAN_CLUSTER : 1;
  const int threads = n_requests > 512 || n_rows > 8 * 512 * PLAN_CLUSTER ? PLAN_THREADS : n_requests > 128 || n_rows > 512 ? 512 : 128;
  e = launch_cluster(paged_plan_kernel, dim3(ranks), dim3(threads), smem, static_cast<cudaStream_t>(cuda_stream), ranks, P);
  if (e == cudaSuccess && !fill)
    e = launch_pdl(paged_rows_of_plan_kernel, dim3((n_rows + PLAN_FILL - 1) / PLAN_FILL), dim3(PLAN_FILL), (n_requests + 1) * 4,
                   static_cast<cudaStream_t>(cuda_stream), P);
  return launched(e, "paged_plan");
}

dmtd_status dmtd_paged_append(const void *q, const void *k, const void *v, int32_t dtype, int64_t q_stride, int64_t k_stride,
                              int64_t v_stride, int32_t n_rows, int32_t n_q_heads, const float *q_norm, const float *k_norm,
                              float rms_eps, float rope_theta, const int32_t *position, const int32_t *slot,
                              const dmtd_paged_cache *cache, void *q_out, void *cuda_stream) {
  PagedAppendParams P{};
  const dmtd_status st = pool_check("paged_append", cache, &P.pool);
  if (st != DMTD_OK) return st;
  if (n_rows < 0 || n_q_heads < 0) return call_failed(DMTD_ERR_INVALID_ARG, "paged_append: negative size");
  if (!known_dtype(dtype)) return call_failed(DMTD_ERR_SHAPE, "paged_append: dtype");
  if (!(rope_theta >= 0.f) || !(rms_eps >= 0.f) || std::isinf(rope_theta)) return call_failed(DMTD_ERR_INVALID_ARG, "paged_append: rope_theta / rms_eps");
  if (n_rows == 0) return DMTD_OK;
  if (!k || !v || !position || !slot || (n_q_heads && (!q || !q_out))) return call_failed(DMTD_ERR_INVALID_ARG, "paged_append: null pointer");
  const int D = cache->head_dim, nkv = cache->n_kv_heads;
  if (n_q_heads > 65536 || nkv > 65536) return call_failed(DMTD_ERR_CAPACITY, "paged_append: more than 2^16 heads");
  const int64_t unit = 16 / dtype_bytes(dtype);
  if (n_rows == 1) q_stride = k_stride = v_stride = 0;
  else if ((n_q_heads && q_stride < (int64_t)n_q_heads * D) || k_stride < (int64_t)nkv * D || v_stride < (int64_t)nkv * D)
    return call_failed(DMTD_ERR_INVALID_ARG, "paged_append: a row stride is shorter than a row");
  if (!aligned16(k) || !aligned16(v) || k_stride % unit || v_stride % unit || (n_q_heads && (!aligned16(q) || !aligned16(q_out) || q_stride % unit)))
    return call_failed(DMTD_ERR_INVALID_ARG, "paged_append: rows must begin on 16-byte boundaries");
  if (q_out == q && n_q_heads && n_rows > 1 && q_stride != (int64_t)n_q_heads * D)
    return call_failed(DMTD_ERR_INVALID_ARG, "paged_append: q_out may be q only where q is dense");
  if (!aligned16(q_norm) || !aligned16(k_norm)) return call_failed(DMTD_ERR_INVALID_ARG, "paged_append: norms must begin on 16-byte boundaries");
  P.q = q; P.k = k; P.v = v;
  P.q_stride = q_stride; P.k_stride = k_stride; P.v_stride = v_stride;
  P.n_rows = n_rows; P.nq = n_q_heads; P.nkv = nkv;
  P.q_norm = q_norm; P.k_norm = k_norm; P.eps = rms_eps;
  P.position = position; P.slot = slot; P.q_out = q_out;
  if (rope_theta > 0.f) {                                // (else there is no rotation)
    const double ratio = std::pow((double)rope_theta, -2.0 / D);
    double f = 0.15915494309189533577;                   // 1 / (2 pi)
    for (int i = 0; i < D / 2; ++i, f *= ratio) P.turns[i] = f;
  }
  // a row to a warp; fewer rows than make some 2000 warps are cut, as far as to a vector for every group of threads
  const int n_vec = n_q_heads + 2 * nkv, at_once = 32 / (D / 2 / (int)unit), most = (n_vec + at_once - 1) / at_once;
  P.slices = std::min(most, std::max(1, APPEND_LEAST_WARPS / n_rows));
  P.per_slice = (most + P.slices - 1) / P.slices * at_once;
  P.slices = (n_vec + P.per_slice - 1) / P.per_slice;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const int64_t warps = (int64_t)n_rows * P.slices, blocks = (warps + APPEND_WARPS - 1) / APPEND_WARPS;
  if (warps > INT32_MAX - APPEND_WARPS) return call_failed(DMTD_ERR_CAPACITY, "paged_append: too many rows");
  const auto launch = D == 128 ? rope_theta > 0.f ? append_launch<128, true> : append_launch<128, false>
                               : rope_theta > 0.f ? append_launch<64, true> : append_launch<64, false>;
  const cudaError_t e = launch(P, dtype, cache->dtype, (int)blocks, stream);
  return launched(e, "paged_append");
}

dmtd_status dmtd_paged_attention(const void *q, int32_t q_dtype, int64_t q_stride, int32_t n_rows, int32_t n_q_heads,
                                 const int32_t *row_start, const int32_t *lens, int32_t n_requests, const int32_t *table,
                                 int32_t table_stride, int32_t max_new, const dmtd_paged_cache *cache, void *scratch,
                                 size_t scratch_bytes, void *out, void *cuda_stream) {
  PagedAttentionParams P{};
  const dmtd_status st = pool_check("paged_attention", cache, &P.pool);
  if (st != DMTD_OK) return st;
  const int D = cache->head_dim, nkv = cache->n_kv_heads;
  if (n_rows < 0 || n_requests < 0 || max_new < 0 || table_stride < 1) return call_failed(DMTD_ERR_INVALID_ARG, "paged_attention: negative or zero size");
  if (!known_dtype(q_dtype)) return call_failed(DMTD_ERR_SHAPE, "paged_attention: q_dtype");
  if (q_dtype != DMTD_F32 && q_dtype != cache->dtype)
    return call_failed(DMTD_ERR_UNSUPPORTED, "paged_attention: 16-bit queries need a cache of their own type");
  if (n_q_heads < 1 || n_q_heads % nkv || n_q_heads / nkv > 16)
    return call_failed(DMTD_ERR_SHAPE, "paged_attention: n_q_heads must be a multiple of n_kv_heads, at most 16 per kv head");
  if ((int64_t)n_rows * n_q_heads > INT32_MAX / 128) return call_failed(DMTD_ERR_CAPACITY, "paged_attention: more than 2^24 query rows and heads");
  if (n_requests > DMTD_PAGED_MAX_REQUESTS) return call_failed(DMTD_ERR_CAPACITY, "paged_attention: more than %d requests", DMTD_PAGED_MAX_REQUESTS);
  if (((int64_t)table_stride << P.pool.lg_page) > 1 << 30)
    return call_failed(DMTD_ERR_CAPACITY, "paged_attention: a table row names more than 2^30 positions");
  if (n_rows == 0 || n_requests == 0) return DMTD_OK;
  if (!q || !out || !row_start || !lens || !table || !scratch) return call_failed(DMTD_ERR_INVALID_ARG, "paged_attention: null pointer");
  if (scratch_bytes < DMTD_PAGED_ATTENTION_SCRATCH_BYTES)
    return call_failed(DMTD_ERR_CAPACITY, "paged_attention: scratch of %zu bytes is smaller than the %zu needed", scratch_bytes,
                       (size_t)DMTD_PAGED_ATTENTION_SCRATCH_BYTES);
  if (n_rows == 1) q_stride = 0;
  else if (q_stride < (int64_t)n_q_heads * D) return call_failed(DMTD_ERR_INVALID_ARG, "paged_attention: the row stride is shorter than a row");
  if (!aligned16(q) || !aligned16(out) || !aligned16(scratch) || q_stride % (16 / (int64_t)dtype_bytes(q_dtype)))
    return call_failed(DMTD_ERR_INVALID_ARG, "paged_attention: rows and scratch must begin on 16-byte boundaries");
  if (out == q) return call_failed(DMTD_ERR_INVALID_ARG, "paged_attention: out must not be q");
  P.q = q; P.q_stride = q_stride; P.out = out;
  P.batch = PagedBatch{row_start, lens, table, n_requests, table_stride, n_rows};
  P.nq = n_q_heads; P.nkv = nkv;
  cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
  const int n_sms = sm_count();
  if (n_sms < 1) return call_failed(DMTD_ERR_CUDA, "paged_attention: device query failed");
  return launched(D == 128 ? attention_launch<128>(P, q_dtype, cache->dtype, max_new ? max_new : n_rows, scratch, n_sms, stream)
                           : attention_launch<64>(P, q_dtype, cache->dtype, max_new ? max_new : n_rows, scratch, n_sms, stream), "paged_attention");
}

}  // extern "C"
