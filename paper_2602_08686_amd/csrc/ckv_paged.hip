// Attention of new tokens over lists of pages (ckv_paged_attention, ckv_paged_tree_attention): tiles of many columns (ckv_paged_tile.h), the merge of
// what workgroups along the rows leave, and how a call is shared out.
#include "ckv_paged_tile.h"

#include <algorithm>

namespace ckv {

template <int DT, int DH, int WAVES>
__global__ void __launch_bounds__(WAVES *kWave, tile_occupancy(DT, DH, WAVES)) paged_tile_kernel(PagedArgs a) {
  attend_tile<DT, DH, WAVES, 1>(a);
}

// Chunks of a column, in their order. A column's lanes take four components each, and for the weights a chunk each; loads of eight chunks are in flight
// together (one after the other, sixteen chunks took 12 us, now 5), the first ones beside those for the weights.
constexpr int kMergeThreads = 256;
template <int DT, int DH>
__global__ void __launch_bounds__(kMergeThreads) paged_merge_kernel(PagedArgs a) {
  constexpr int PIECES = DH / 4, COLS = kMergeThreads / PIECES, SHARE = kMostChunks / PIECES;
  const int blocks = (a.G * a.n + COLS - 1) / COLS;
  const int unit = blockIdx.x / blocks, col = blockIdx.x % blocks * COLS + threadIdx.x / PIECES, piece = threadIdx.x % PIECES;
  const bool valid = col < a.G * new_rows(a.lists, unit, a.n);
  const int tile = col / a.tile_cols, local = col % a.tile_cols, b = unit / a.Hkv;
  const TileRange range = tile_range(a, unit, tile);
  const int chunks = valid ? (range.stages + range.per_chunk - 1) / range.per_chunk : 0;
  const size_t first = ((size_t)unit * a.col_tiles + tile) * a.n_chunks * a.tile_cols + local;
  constexpr int BATCH = 8;
  f32x4_p x[BATCH];
  const auto fetch = [&](int i0) CKV_INLINE {
#pragma unroll
    for (int j = 0; j < BATCH; ++j) {
      x[j] = f32x4_p{0.0f, 0.0f, 0.0f, 0.0f};
      if (i0 + j < chunks) x[j] = *reinterpret_cast<const f32x4_p *>(a.part + (first + (size_t)(i0 + j) * a.tile_cols) * DH + 4 * piece);
    }
  };
  float2 st[SHARE];
  float top = -INFINITY;
#pragma unroll
  for (int k = 0; k < SHARE; ++k) {
    const int i = k * PIECES + piece;
    st[k] = make_float2(-INFINITY, 0.0f);
    if (i < chunks) st[k] = a.stats[first + (size_t)i * a.tile_cols];
  }
  fetch(0);
#pragma unroll
  for (int k = 0; k < SHARE; ++k) top = fmaxf(top, st[k].x);
#pragma unroll
  for (int o = 1; o < PIECES; o <<= 1) top = fmaxf(top, __shfl_xor(top, o));
  const float ref = top == -INFINITY ? 0.0f : top;
  float sum = 0.0f, weight[SHARE];
#pragma unroll
  for (int k = 0; k < SHARE; ++k) {
    weight[k] = st[k].y * __builtin_amdgcn_exp2f(st[k].x - ref);
    sum += weight[k];
  }
#pragma unroll
  for (int o = 1; o < PIECES; o <<= 1) sum += __shfl_xor(sum, o);
  const float inv = inverse_sum(sum);
#pragma unroll
  for (int k = 0; k < SHARE; ++k) weight[k] *= inv;
  f32x4_p num = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int k = 0; k < SHARE; ++k) {
    for (int c0 = 0; c0 < PIECES && k * PIECES + c0 < a.n_chunks; c0 += BATCH) {  // the same for all lanes
      if (k > 0 || c0 > 0) fetch(k * PIECES + c0);
#pragma unroll
      for (int j = 0; j < BATCH; ++j) num = add_part(num, x[j], __shfl(weight[k], (threadIdx.x & 63) / PIECES * PIECES + c0 + j));
    }
  }
  if (!valid) return;
  const Column c = column(a, unit, tile, local);
  store_out<DT>(out_row(a, b, c), 4 * piece, num);
  if (piece == 0) store_lse(a, b, c, top, sum);
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------
// Workgroups along the rows: as many as fill the chip (one of eight waves a CU, or two of four), if each of them has enough rows to be worth
// the way through memory that its sums then take, and none beside the first for so few rows that the merge would cost more than it saves.
// Eight waves a tile once that fills the chip: 2048 new tokens, 32k rows, 32/8 heads 1062 us with four, 990 with eight, 4096 tokens over
// themselves 162 / 151, batch 4 of 1024 tokens 59 / 56, but 512 tokens over themselves 23 / 27.
// Of the tiles in f32 with rows of 512 bytes one fits a CU: for long lists chunks for one, 300 tokens, 8/1 heads, batch 3, 2000 rows 99 / 88, 80 tokens,
// 8/2 heads, 20000 rows 116 / 92, 512 tokens, 32/8 heads, 4096 rows 300 / 296; but 101 tokens, 8/1 heads, batch 8, 523 rows 35 / 44.
// Least rows of a chunk, us with half / these / twice: few columns, bf16, one token, 32/8 heads, 2000 rows 10.8 / 11.4 / 12.7, batch 4
// 12.6 / 12.6 / 14.3; f32, 4/4 heads of 64, batch 4, 1000 rows 11.4 / 10.8 / 13.1, 200 tokens, 1024 rows 13.9 / 13.1 / 15.5; tiles, bf16, 512 tokens over
// themselves 24.1 / 19.5 / 19.5; f32, heads of 64, 101 tokens, 523 rows (64 / 128) 24.3 / 29.6. One chunk up to 1024 (bf16) or 256 (f32) rows
// of few columns: 500 rows 10.1, two chunks 11.0; batch 16, 544 rows 10.7, two chunks 11.6, 1000 rows 16.9, two 16.3; but batch 4 over 2000 rows
// 23.7 with one, 12.6 with the rule's.
// For trees, bf16. Tiles of 256 columns, which read a row once where two of 128 read it twice, where hardly any column is there for nothing, about as many
// waves stay busy (a list has 64 chunks at most) and a chunk is so long that its rows outweigh its start and end: 1024 rows of 128, or six times as many
// where tiles of 128 need no chunks, and so no merge. us, 128 / 256 columns: 60 tokens, batch 4, 32768 rows 235 / 217, 8192 (chunks of 1024) 74 / 70, 6144
// 58.6 / 58.6, 4096 43.5 / 46.1; 32/8 heads, one sequence, 32768 rows (1024) 71.8 / 70.1, 16384 43.0 / 46.5; 500 tokens, batch 2, 32771 rows 767 / 722, and, 128
// in one chunk, 12288 (6144) 305 / 295, 8195 199 / 207; heads of 64, batch 4, 16384 rows 78.5 / 76.9, 8192 43.6 / 44.9. Workgroups of eight waves: 8/1 heads, 32
// tokens, 131072 rows 62 in 128 / 91 in 64; 16/2 heads, 65536 rows 47 in 256 / 58 in 128; 24/3 heads, 131072 rows 101.6 in 252 / 101.5 in 192. 328
// columns (384 / 512), batch 8, 9312 rows 58.9 / 63.5. Otherwise tiles of 128 by two groups of four waves, where that leaves about as many waves busy as
// workgroups of four would be: 150 tiles on 256 CUs, batch 3, 9068 rows 178 in 450 workgroups of four waves, 221 in 150 of eight; and not for the few stages of
// short lists, 180 rows 14.8 / 15.8.
constexpr int64_t kFarRow = 1024 * 128;  // components of a row times rows of a chunk
PagedPlan plan_paged(const Shape &s, int n_rows, bool tree) {
  PagedPlan p;
  const bool bf16 = s.esize == 2;
  const int64_t units = (int64_t)s.Bz * s.Hkv, cols = (int64_t)s.G * s.T;
  p.by_rows = cols <= (bf16 ? kMostRowsCols : kMostRowsColsF32);
  const int least = p.by_rows ? (bf16 ? 256 : 128) : bf16 ? 512 : s.d == 64 ? 64 : 128;
  const int64_t most = p.by_rows && n_rows <= (bf16 ? 1024 : 256) ? 1 : (n_rows + least - 1) / least;
  const auto chunks_of = [&](int64_t tiles, int64_t places) { return std::min<int64_t>({places / tiles, most, kMostChunks}); };
  const int64_t narrow = units * ((cols + 127) / 128), wide = units * ((cols + 255) / 256);  // tiles
  bool far = tree && bf16 && !p.by_rows && wide <= kComputeUnits && wide * 2 * 20 <= narrow * 21;
  if (far) {
    const int64_t of_wide = chunks_of(wide, kComputeUnits), of_narrow = chunks_of(narrow, kComputeUnits);
    const int64_t busy = narrow <= kComputeUnits ? narrow * of_narrow : narrow / 2;  // in workgroups of eight waves
    far = 4 * wide * of_wide >= 3 * busy && (int64_t)n_rows * s.d >= of_wide * kFarRow * (of_wide > 1 && of_narrow == 1 ? 6 : 1);
  }
  const int waves = wide >= kComputeUnits || far ? 8 : 4;
  p.tile_cols = p.by_rows ? kRowsCols : waves * 32;
  p.stage_rows = p.by_rows ? 32 : kStageRows;
  p.col_tiles = (int)((cols + p.tile_cols - 1) / p.tile_cols);
  const int64_t tiles = units * p.col_tiles;
  const bool two = !p.by_rows && waves == 4 && (bf16 || s.d == 64 || n_rows < 1024);
  int64_t chunks = (two ? 2 : 1) * kComputeUnits / tiles;
  if (chunks > most) chunks = most;
  if (chunks > kMostChunks) chunks = kMostChunks;
  if (chunks < 1) chunks = 1;
  const int64_t pairs = chunks_of(tiles, kComputeUnits);
  p.halves = tree && bf16 && !p.by_rows && waves == 4 && pairs > 0 && 11 * pairs >= 5 * chunks && n_rows > 4 * kStageRows;
  if (p.halves) chunks = pairs;
  p.n_chunks = (int)chunks;
  p.workgroups = tiles * chunks;
  p.joined = p.by_rows && cols <= kMostJoinedCols && cols * chunks <= kMostJoined;
  p.workspace_bytes = chunks == 1 ? 0 : (size_t)p.workgroups * p.tile_cols * (s.d + 2) * sizeof(float) + (p.joined ? p.workgroups * sizeof(tag_t) : 0);
  return p;
}

template <int DT, int DH, int WAVES>
static void launch_tiles(const PagedArgs &a, hipStream_t stream) {
  hipLaunchKernelGGL((paged_tile_kernel<DT, DH, WAVES>), dim3((unsigned)a.workgroups), dim3(WAVES * kWave), 0, stream, a);
}

template <int DT, int DH>
static void launch_paged_of(const TreeArgs &a, const PagedPlan &plan, int units, hipStream_t stream) {
  if (a.sees) launch_tree(a, plan, DT == CKV_BF16, DH, stream);
  else if (plan.by_rows) launch_paged_rows(a, DT == CKV_BF16, DH, stream);
  else if (plan.tile_cols == 256) launch_tiles<DT, DH, 8>(a, stream);
  else launch_tiles<DT, DH, 4>(a, stream);
  if (plan.n_chunks > 1 && !plan.joined) {
    constexpr int COLS = kMergeThreads / (DH / 4);
    const unsigned blocks = (unsigned)(a.G * a.n + COLS - 1) / COLS;
    hipLaunchKernelGGL((paged_merge_kernel<DT, DH>), dim3(units * blocks), dim3(kMergeThreads), 0, stream, a);
  }
}

PageLists page_lists(const Shape &s, const ckv_pages *pages, const int32_t *table, const int32_t *length, const int32_t *count) {
  PageLists l;
  l.table = table;
  l.length = length;
  l.count = count;
  l.table_b = pages->table_stride[0];
  l.table_h = pages->table_stride[1];
  for (int i = 0; i < 3; ++i) {
    l.ks[i] = pages->k_stride[i] * s.esize;
    l.vs[i] = pages->v_stride[i] * s.esize;
  }
  l.shift = __builtin_ctz((unsigned)pages->page_rows);
  l.n_pages = pages->n_pages;
  l.capacity = pages->max_pages * pages->page_rows;
  return l;
}

hipError_t launch_paged_attention(const ckv_params *p, const Shape &s, const PagedPlan &plan, const ckv_pages *pages, const void *q,
                                  const void *k_pages, const void *v_pages, const int32_t *table, const int32_t *length,
                                  const int32_t *count, int n_rows, const uint64_t *sees, void *out, const int64_t *out_stride, float *lse,
                                  char *ws, hipStream_t stream) {
  const int units = s.Bz * s.Hkv;
  TreeArgs a;
  a.sees = reinterpret_cast<const uint32_t *>(sees);
  a.words = 2 * ((s.T + 63) / 64);
  a.q = static_cast<const char *>(q);
  a.k = static_cast<const char *>(k_pages);
  a.v = static_cast<const char *>(v_pages);
  a.out = static_cast<char *>(out);
  const int64_t dense[3] = {(int64_t)s.Hq * s.T * s.d, (int64_t)s.T * s.d, s.d};
  for (int i = 0; i < 3; ++i) {
    a.qs[i] = p->q_stride[i] * s.esize;
    a.os[i] = (out_stride ? out_stride[i] : dense[i]) * s.esize;
  }
  a.lists = page_lists(s, pages, table, length, count);
  a.lse = lse;
  a.part = reinterpret_cast<float *>(ws);
  a.stats = reinterpret_cast<float2 *>(a.part + (plan.n_chunks > 1 ? (size_t)plan.workgroups * plan.tile_cols * s.d : 0));
  a.marks = plan.n_chunks > 1 && plan.joined ? reinterpret_cast<tag_t *>(a.stats + plan.workgroups * plan.tile_cols) : nullptr;
  a.tag = a.marks ? launch_tag() : 0;
  a.Hq = s.Hq; a.Hkv = s.Hkv; a.G = s.G;
  a.n = s.T;
  a.n_rows = n_rows;
  a.tile_cols = plan.tile_cols;
  a.col_tiles = plan.col_tiles;
  a.stage_rows = plan.stage_rows;
  a.n_chunks = plan.n_chunks;
  a.workgroups = (int)plan.workgroups;
  a.scale2 = s.scale * kLog2e;
  if (p->dtype == CKV_BF16) {
    if (s.d == 128) launch_paged_of<CKV_BF16, 128>(a, plan, units, stream);
    else launch_paged_of<CKV_BF16, 64>(a, plan, units, stream);
  } else {
    if (s.d == 128) launch_paged_of<CKV_F32, 128>(a, plan, units, stream);
    else launch_paged_of<CKV_F32, 64>(a, plan, units, stream);
  }
  return hipGetLastError();
}

}  // namespace ckv
