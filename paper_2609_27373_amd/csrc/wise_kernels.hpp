// wise_kernels.hpp — host-side launchers of the libwise kernels.  Shapes are
// validated by the C ABI layer before any of these is called.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace wise {

// Validated geometry: bh = batch * heads, nb = n / block; gq = heads /
// kv_heads query heads share one key-value head.
struct Dims {
  int bh, n, d, block, nb, heads, gq;
  float scale;
};

// Validated paged cache and the queries that read it (wise_cache, wise_queries).
struct Cache {
  int pages, page, kv_heads, head_dim, planes, seqs, max_pages;
};
struct Queries {
  int batch, heads, q_len;
  float scale;
};

constexpr int kMaxEntries = 1024;       // sequences named by one call on a cache
constexpr int kMaxQueryRows = 128;      // query rows of a sequence per key-value head
constexpr int kMaxPages = 1 << 27;      // of a pool: 256 GB of the smallest pages

constexpr int kMaxSelectBlocks = 1024;  // selection keeps a row's candidates in LDS

hipError_t launch_dense(const Dims& s, const void* q, const void* k, const void* v, void* o,
                        float* lse, float* acc, void* ws, hipStream_t st);
size_t mass_workspace_bytes(const Dims& s);
int dense_query_tile(const Dims& s);   // queries per dense work-group of a full grid: 64, 128 or 256
hipError_t launch_sparse(const Dims& s, const void* q, const void* k, const void* v,
                         const int32_t* row_ptr, const int32_t* col_idx, const int32_t* order,
                         void* o, float* lse, hipStream_t st);
// Blocks of 64 keys (groups of 4 rows at head_dim 128, else 2) and of 128
// keys at head_dim 128 (groups of 2 rows): work-groups of consecutive rows
// over the union of their supports (sparse_group_rows(s) rows per group; 0:
// not available, and launch_sparse_grouped runs launch_sparse instead).
int sparse_group_rows(const Dims& s);
hipError_t launch_sparse_grouped(const Dims& s, const void* q, const void* k, const void* v,
                                 const int32_t* row_ptr, const int32_t* col_idx, void* o,
                                 float* lse, hipStream_t st);
hipError_t launch_select(const Dims& s, const float* acc, float tau, uint32_t flags,
                         int32_t* row_ptr, int32_t* col_idx, int32_t* row_order, void* ws,
                         hipStream_t st);
size_t select_workspace_bytes(const Dims& s);
hipError_t launch_select_noalloc(const Dims& s, const float* acc, float tau, uint32_t flags,
                                 int32_t* row_ptr, int32_t* col_idx, int32_t* row_order,
                                 hipStream_t st);
int mask_words(const Dims& s);
hipError_t launch_select_step(const Dims& s, const float* r, float tau, uint64_t* mask,
                              hipStream_t st);
hipError_t launch_support_from_masks(const Dims& s, const uint64_t* masks, int n_masks,
                                     uint32_t flags, int32_t* row_ptr, int32_t* col_idx,
                                     int32_t* row_order, void* ws, hipStream_t st);
hipError_t launch_mask_union(const Dims& s, const uint64_t* masks, int n_masks, uint64_t* out,
                             hipStream_t st);
hipError_t launch_mask_overlap(const Dims& s, const uint64_t* a, const uint64_t* b,
                               int64_t* counts, hipStream_t st);
hipError_t launch_support_mass(const Dims& s, const float* r, const int32_t* row_ptr,
                               const int32_t* col_idx, double* row_mass, double* totals,
                               hipStream_t st);

hipError_t launch_cache_fork(const Cache& c, int n, const int32_t* src, const int32_t* dst, int32_t* tables, int32_t* lens,
                             int32_t* refs, int32_t* done, hipStream_t st);
hipError_t launch_cache_trim(const Cache& c, int n, const int32_t* ids, const int32_t* new_lens, int32_t* tables, int32_t* lens,
                             int32_t* refs, hipStream_t st);
hipError_t launch_cache_reserve(const Cache& c, int n, const int32_t* ids, const int32_t* counts, int32_t* tables, int32_t* lens,
                                int32_t* refs, int32_t* granted, void* pool, void* ws, hipStream_t st);
hipError_t launch_cache_append(const Cache& c, int n, int tokens, const int32_t* ids, const int32_t* counts, const void* k,
                               const void* v, const int32_t* tables, const int32_t* lens, void* kp, void* vp, hipStream_t st);
hipError_t launch_cache_compact(const Cache& c, int32_t* tables, int32_t* refs, void* pool, int32_t* live, void* ws,
                                hipStream_t st);
hipError_t launch_cache_shared(const Cache& c, int batch, int min_pages, const int32_t* ids, const int32_t* tables,
                               const int32_t* lens, int32_t* shared, hipStream_t st);
size_t cache_workspace_bytes(const Cache& c);
hipError_t launch_prefix(const Cache& c, const Queries& a, const void* q, const void* kp, const void* vp, const int32_t* tables,
                         const int32_t* lens, const int32_t* ids, const int32_t* shared, void* o, float* lse, void* ws,
                         hipStream_t st);
size_t prefix_workspace_bytes(const Cache& c, const Queries& a);

}  // namespace wise
