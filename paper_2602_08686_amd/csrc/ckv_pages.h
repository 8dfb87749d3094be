// Lists of pages as the kernels see them (private; the definitions are at ckv_pages in ckv.h).
#ifndef CKV_PAGES_H_
#define CKV_PAGES_H_

#include "ckv_internal.h"

namespace ckv {

// For lambdas: one that is called from several places may stay a function, and all it refers to lies in memory then.
#define CKV_INLINE __attribute__((always_inline))

struct PageLists {
  const int32_t *table, *length, *count;  // count may be null: all n new rows
  int64_t table_b, table_h;               // entries between batch elements, between KV heads
  int64_t ks[3], vs[3];                   // BYTES between pages, KV heads, rows
  int shift, n_pages, capacity;           // log2(page_rows); pages of the pools; rows of a list (max_pages * page_rows)
};

// New rows of a list, of at most n.
__device__ __forceinline__ int new_rows(const PageLists &l, int unit, int n) {
  return l.count ? min(max(l.count[unit], 0), n) : n;
}

// Bytes from a pool's start to row `row` of a page, for the page number and byte strides of one of the pools.
__device__ __forceinline__ int64_t in_pool(const int64_t (&s)[3], int page, int g, int row) {
  return page * s[0] + g * s[1] + row * s[2];
}

// Two floats as bf16, to the nearest, ties to even (NaN stays one), the first in the lower half: v_cvt_pk_bf16_f32.
__device__ __forceinline__ uint32_t pack_bf16(float x, float y) {
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
  const bf16x2 both = {(__bf16)x, (__bf16)y};
  return __builtin_bit_cast(uint32_t, both);
}

PageLists page_lists(const Shape &s, const ckv_pages *pages, const int32_t *table, const int32_t *length, const int32_t *count);
hipError_t launch_rows(const ckv_params *p, const Shape &s, const ckv_rotation *rotation, const ckv_pages *pages, const void *q,
                       const void *k, const void *v, const int32_t *positions, const float *inv_freq, const void *q_weight,
                       const void *k_weight, const int32_t *table, const int32_t *length, const int32_t *count, void *q_out, void *k_out,
                       void *v_out, hipStream_t stream);

// Attention over the pages: how a call is shared out, from sizes alone.
struct PagedPlan {
  bool by_rows;      // paged_rows_kernel: few columns, a workgroup's waves share out the rows
  int tile_cols;     // query columns (heads of a group times new tokens) of a workgroup
  int col_tiles;     // such tiles of a (batch element, KV head)
  int stage_rows;    // rows of a list are shared out in multiples of this
  int n_chunks;      // workgroups along the rows of a list
  bool joined;       // chunks are joined in the same launch
  bool halves;       // tiles of eight waves for 128 columns, of which four take one half of the rows each
  int64_t workgroups;
  size_t workspace_bytes;
};
constexpr int64_t kMostPagedWorkgroups = 1 << 22;  // 512 threads of each have to be fewer than 2^32
PagedPlan plan_paged(const Shape &s, int n_rows, bool tree);
hipError_t launch_paged_attention(const ckv_params *p, const Shape &s, const PagedPlan &plan, const ckv_pages *pages, const void *q,
                                  const void *k_pages, const void *v_pages, const int32_t *table, const int32_t *length,
                                  const int32_t *count, int n_rows, const uint64_t *sees, void *out, const int64_t *out_stride, float *lse,
                                  char *ws, hipStream_t stream);

// Trees of drafted tokens.
constexpr int kMostTreeTokens = 65536;  // a token's words times the tokens stay below 2^31
constexpr int kMostDrafts = 4096;       // of ckv_tree_sees: a word and a number of each in LDS
int64_t tree_workgroups(int batch, int n);
hipError_t launch_tree_sees(int batch, int n, const int32_t *parent, const int32_t *start, uint64_t *sees, int32_t *positions, hipStream_t stream);

// Rows and pages that move.
hipError_t launch_compact(const Shape &s, const ckv_pages *pages, const int32_t *table, const int32_t *length, const int32_t *count,
                          const int32_t *idx, const int64_t *idx_stride, int cap, const int32_t *kept, void *k_pages, void *v_pages,
                          int32_t *length_out, hipStream_t stream);
int64_t copy_workgroups(const Shape &s, const ckv_pages *pages, int n);
hipError_t launch_pages_copy(const Shape &s, const ckv_pages *pages, const int32_t *copy, int n, void *k_pages, void *v_pages, hipStream_t stream);

// Which lists have which pages.
int64_t entry_workgroups(const ckv_lists *lists);  // at most, of a launch with a thread for an entry
hipError_t launch_fork(const ckv_lists *lists, const int32_t *table, const int32_t *parent, int32_t *table_out, int32_t *refs, uint32_t *taken,
                       const int32_t *length, int32_t *length_out, hipStream_t stream);
hipError_t launch_reserve(const ckv_lists *lists, int32_t *table, const int32_t *first, const int32_t *end, int32_t *refs, uint32_t *taken,
                          int32_t *copy, int n_copy, int32_t *result, hipStream_t stream);
hipError_t launch_free(const ckv_lists *lists, int32_t *table, const int32_t *keep, int32_t *refs, uint32_t *taken, hipStream_t stream);

}  // namespace ckv
#endif
