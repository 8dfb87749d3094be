// Attention of new tokens over lists of pages (ckv_paged_attention).
//
// Columns: the queries of a (batch element, KV head), G * i + head, so that neighbours see nearly the same rows and a row is read once
// for all heads of a group. A workgroup takes a tile of columns, 32 per wave, and sweeps the rows that the last of them sees, in stages
// of 64 (bf16) or 32 (f32) rows that go from memory to LDS without registers between and are read by all of its waves.
// Rows x queries (32 x 32 matrix tiles, 16 or 2 components at a time) leaves a lane with 16 logits of one column, whose running
// maximum and sum stay in the lane but for one exchange with the other half of the wave, and which are the operand of the second product as
// they lie: the contraction over rows may be permuted if both operands agree, so V's operand takes the rows in the order that the
// logits have. V lies in LDS as it does in memory and is transposed on its way into registers.
// LDS images are swizzled in units that one cycle reads (16 bytes of eight rows of K, 32 bytes of four rows of V).
//
// What a token does not see must not touch its result even if it is infinite or NaN, and zero times infinity is NaN: where a sweep leaves
// something that is not finite, the workgroup sweeps again, with V's finite components only, and twice more for where its
// infinite and NaN ones are.
#include "ckv_paged.h"

namespace ckv {

constexpr int kTileWaves = 4;
constexpr int tile_stage_rows(bool bf16) { return bf16 ? 64 : 32; }

template <int DT, int DH, int WAVES>
__global__ void __launch_bounds__(WAVES *kWave, 2) paged_tile_kernel(PagedArgs a) {
  typedef Image<DT, DH> I;
  constexpr int ROWS = tile_stage_rows(DT == CKV_BF16), BLOCKS = ROWS / 32, BYTES = ROWS * I::ROW;
  constexpr int LOADS = BYTES / 1024 / WAVES;  // of K per wave and stage, and of V
  static_assert(LOADS * WAVES * 1024 == BYTES, "whole loads");
  __shared__ __align__(1024) char s_k[2][BYTES];
  __shared__ __align__(1024) char s_v[2][BYTES];
  __shared__ int s_missing, s_undefined;

  int at = work_item(blockIdx.x, a.workgroups);
  const int chunk = at % a.n_chunks;
  at /= a.n_chunks;
  const int tile = a.col_tiles - 1 - at % a.col_tiles, unit = at / a.col_tiles;  // the longest first
  const int b = unit / a.Hkv, g = unit % a.Hkv;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  const TileRange range = tile_range(a, unit, tile);
  if (range.cols <= 0) return;
  const int first = chunk * range.per_chunk, last = min(first + range.per_chunk, range.stages);
  const bool single = a.n_chunks == 1;
  if (first >= last && !single) return;  // the merge reads the chunks that have stages

  const int local = wave * 32 + (lane & 31);
  const bool valid = local < range.cols;
  const Column c = column(a, unit, tile, valid ? local : 0);
  // of the wave: its first column sees the fewest rows, the last that exists the most
  const int sees_least = __builtin_amdgcn_readfirstlane(c.limit);
  const int sees_most = wave * 32 < range.cols ? column(a, unit, tile, min(range.cols, wave * 32 + 32) - 1).limit : 0;
  u32x4_d qf[I::STEPS];
  load_query<DT, DH>(a, b, c, valid, half, qf);

  const int32_t *list = a.lists.table + b * a.lists.table_b + g * a.lists.table_h;
  const char *kb = a.k + g * a.lists.ks[1], *vb = a.v + g * a.lists.vs[1];
  if (threadIdx.x == 0) s_missing = s_undefined = 0;
  __syncthreads();

  // Rows behind the end are the last one again; a page that is not in the pool is page 0 (they weigh nothing).
  auto fetch = [&](int stage, int buf) {
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int block = wave * LOADS + j, row = block * I::ROWS_PER_LOAD + lane / I::PIECES, piece = lane % I::PIECES;
      const int at_row = min(stage * ROWS + row, range.end - 1);
      int page = list[at_row >> a.lists.shift];
      if ((unsigned)page >= (unsigned)a.lists.n_pages) {
        page = 0;
        s_missing = 1;
      }
      const int64_t r = at_row & ((1 << a.lists.shift) - 1);
      dma_16<false>(kb + page * a.lists.ks[0] + r * a.lists.ks[2] + I::k_piece(row, piece) * 16, s_k[buf] + block * 1024);
      dma_16<false>(vb + page * a.lists.vs[0] + r * a.lists.vs[2] + I::v_piece(row, piece) * 16, s_v[buf] + block * 1024);
    }
  };

  Running run;
  f32x16_p acc[I::DTILES];
  auto sweep = [&](auto careful, int mode) {
    constexpr bool CAREFUL = decltype(careful)::value;
    run = Running{-INFINITY, 0.0f};
#pragma unroll
    for (int t = 0; t < I::DTILES; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[t][r] = 0.0f;
    if (first < last) fetch(first, 0);
    for (int stage = first; stage < last; ++stage) {
      const int buf = (stage - first) & 1, base = stage * ROWS;
      wait_vm_at_most<0>();
      __syncthreads();  // the stage is there, and the other buffer has been read
      if (stage + 1 < last) fetch(stage + 1, buf ^ 1);
      if (base >= sees_most) continue;
      const bool missing = s_missing;
      f32x16_p z[BLOCKS];
#pragma unroll
      for (int k = 0; k < BLOCKS; ++k) first_product<DT, DH>(s_k[buf] + 32 * k * I::ROW, lane, qf, z[k]);
      if (missing || base + ROWS > sees_least) {
#pragma unroll
        for (int k = 0; k < BLOCKS; ++k)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int row = base + 32 * k + block_row(r, half);
            bool seen = row < c.limit;
            if (missing && seen) seen = (unsigned)list[row >> a.lists.shift] < (unsigned)a.lists.n_pages;
            if (!seen) z[k][r] = -INFINITY;
          }
      }
      online_softmax<BLOCKS, I::DTILES, CAREFUL>(z, a.scale2, run, acc, mode);
#pragma unroll
      for (int k = 0; k < BLOCKS; ++k) second_product<DT, DH, CAREFUL>(s_v[buf] + 32 * k * I::ROW, lane, z[k], acc, mode);
    }
  };
  sweep(std::false_type{}, kFinite);
  if (valid && not_finite(acc)) s_undefined = 1;
  __syncthreads();
  if (s_undefined) {  // the same for all waves, as there are barriers in the sweeps
    Marks marks;
    for (int mode = kUp; mode <= kFinite; ++mode) {
      __syncthreads();  // the buffers have been read
      sweep(std::true_type{}, mode);
      take_marks(marks, acc, mode);
    }
  }
  run.sum = over_halves(run.sum, [](float x, float y) { return x + y; });
  if (!valid) return;

  const size_t row = (((size_t)unit * a.col_tiles + tile) * a.n_chunks + chunk) * a.tile_cols + local;
  char *to = out_row(a, b, c);
  const float inv = inverse_sum(run.sum);
#pragma unroll
  for (int t = 0; t < I::DTILES; ++t)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const f32x4_p x = {acc[t][4 * r], acc[t][4 * r + 1], acc[t][4 * r + 2], acc[t][4 * r + 3]};
      const int d = 32 * t + block_row(4 * r, half);
      if (single) store_out<DT>(to, d, x * inv);
      else *reinterpret_cast<f32x4_p *>(a.part + row * DH + d) = x;
    }
  if (half == 0) {
    if (single) store_lse(a, b, c, run.top, run.sum);
    else a.stats[row] = make_float2(run.top, run.sum);
  }
}

// Chunks of a column, in their order. A thread takes four components of one column.
constexpr int kMergeThreads = 256;
template <int DT, int DH>
__global__ void __launch_bounds__(kMergeThreads) paged_merge_kernel(PagedArgs a) {
  constexpr int PIECES = DH / 4, COLS = kMergeThreads / PIECES;
  const int blocks = (a.G * a.n + COLS - 1) / COLS;
  const int unit = blockIdx.x / blocks, col = blockIdx.x % blocks * COLS + threadIdx.x / PIECES, d = threadIdx.x % PIECES * 4;
  if (col >= a.G * new_rows(a.lists, unit, a.n)) return;
  const int tile = col / a.tile_cols, local = col % a.tile_cols, b = unit / a.Hkv;
  const TileRange range = tile_range(a, unit, tile);
  const int chunks = (range.stages + range.per_chunk - 1) / range.per_chunk;
  const size_t first = ((size_t)unit * a.col_tiles + tile) * a.n_chunks * a.tile_cols + local;
  float top = -INFINITY, sum = 0.0f;
  for (int i = 0; i < chunks; ++i) top = fmaxf(top, a.stats[first + (size_t)i * a.tile_cols].x);
  const float ref = top == -INFINITY ? 0.0f : top;
  f32x4_p num = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int i = 0; i < chunks; ++i) {
    const size_t row = first + (size_t)i * a.tile_cols;
    const float2 st = a.stats[row];
    const float f = __builtin_amdgcn_exp2f(st.x - ref);
    sum = fmaf(st.y, f, sum);
    num = add_part(num, *reinterpret_cast<const f32x4_p *>(a.part + row * DH + d), f);
  }
  const Column c = column(a, unit, tile, local);
  store_out<DT>(out_row(a, b, c), d, num * inverse_sum(sum));
  if (d == 0) store_lse(a, b, c, top, sum);
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------
PagedPlan plan_paged(const Shape &s, int n_rows) {
  PagedPlan p;
  const bool bf16 = s.esize == 2;
  const int64_t units = (int64_t)s.Bz * s.Hkv, cols = (int64_t)s.G * s.T;
  p.by_rows = cols <= kRowsCols;
  p.tile_cols = p.by_rows ? kRowsCols : kTileWaves * 32;
  p.stage_rows = p.by_rows ? 32 : tile_stage_rows(bf16);
  p.col_tiles = (int)((cols + p.tile_cols - 1) / p.tile_cols);
  const int64_t tiles = units * p.col_tiles;
  int64_t chunks = (p.by_rows ? 1 : 2) * kComputeUnits / tiles, most = (n_rows + (p.by_rows ? 511 : 255)) / (p.by_rows ? 512 : 256);
  if (chunks > most) chunks = most;
  if (chunks > 64) chunks = 64;
  if (chunks < 1) chunks = 1;
  p.n_chunks = (int)chunks;
  p.workgroups = tiles * chunks;
  p.workspace_bytes = chunks == 1 ? 0 : (size_t)p.workgroups * p.tile_cols * (s.d + 2) * sizeof(float);
  return p;
}

template <int DT, int DH>
static void launch_paged_of(const PagedArgs &a, const PagedPlan &plan, int units, hipStream_t stream) {
  if (plan.by_rows) launch_paged_rows(a, DT == CKV_BF16, DH, stream);
  else hipLaunchKernelGGL((paged_tile_kernel<DT, DH, kTileWaves>), dim3((unsigned)plan.workgroups), dim3(kTileWaves * kWave), 0, stream, a);
  if (plan.n_chunks > 1) {
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
                                  const int32_t *count, int n_rows, void *out, const int64_t *out_stride, float *lse, char *ws,
                                  hipStream_t stream) {
  PagedArgs a;
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
  a.Hq = s.Hq; a.Hkv = s.Hkv; a.G = s.G;
  a.n = s.T;
  a.n_rows = n_rows;
  a.tile_cols = plan.tile_cols;
  a.col_tiles = plan.col_tiles;
  a.stage_rows = plan.stage_rows;
  a.n_chunks = plan.n_chunks;
  a.workgroups = (int)plan.workgroups;
  a.scale2 = s.scale * kLog2e;
  const int units = s.Bz * s.Hkv;
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
