// Attention over pages for few columns (decoding steps, drafted tokens): bound by memory, every row once.
//
// All of a tile's columns are one operand of the matrix products (32 of them, however many exist), and the workgroup's waves
// share out the rows, 32 at a time, each with a place in LDS of its own for them: no barrier between the first row and the last. A wave's
// loads go straight to LDS. K's place is free once the first product has read it and V's once the second has, so the next
// 32 rows' K is on its way during the softmax and the second product, their V during the next first product. Page numbers
// come the same way, one block further ahead; a lane per row turns them into offsets.
// Measured: bf16, 32/8 heads of 128, batch 4, 32768 rows, one token 85.9 us, 6.3 TB/s of K and V; 65000 rows, batch 1 48.3 us, 5.5. Short lists are
// a chain of latencies: batch 16, up to 544 rows 11.4 us, in cycles of a mean workgroup 4500 until the page numbers, 2900 more until K, 6400 for
// the first wave's two or three blocks and 7300 for waiting for the other waves and joining them. (Four waves, and two or four times as many chunks, were slower.)
// Waves are joined in LDS in wave order, chunks in chunk order: by paged_merge_kernel, or where their sums are few in this launch. Each workgroup
// then leaves its sums, past its own caches, and behind them a mark, the launch's tag (another value for every launch, which undefined memory
// does not hold), and looks at the marks of its tile. Who finds all of them, which the last one to mark does unless somebody else has before,
// joins the chunks and takes the marks back, as a replay of the launch has the same tag. Nobody waits for anybody; two that find them
// all write the same values.
#include "ckv_paged.h"

namespace ckv {

template <int DT, int DH, int WAVES, bool STREAM>
__global__ void __launch_bounds__(WAVES *kWave, WAVES / 4) paged_rows_kernel(PagedArgs a) {
  typedef Image<DT, DH> I;
  constexpr int LOADS = 32 / I::ROWS_PER_LOAD;  // of K, and of V, per block
  constexpr int BLOCK = 32 * I::ROW;
  constexpr int PIECES = DH / 4;                // of 16 bytes of a column's fp32 sums
  __shared__ __align__(1024) char s_rows[WAVES][2 * BLOCK];  // K's rows, V's rows
  __shared__ __align__(256) int32_t s_ids[WAVES][2][kWave];
  struct Offsets {
    int64_t k, v;
  };
  __shared__ Offsets s_at[WAVES][32];
  __shared__ float2 s_stats[WAVES][32];
  __shared__ int s_last;
  static_assert(kMostJoinedCols * kMostChunks * sizeof(float) <= sizeof(s_rows), "the chunks' weights lie there too");
  static_assert(32 * DH * 4 <= 2 * BLOCK, "a wave's sums take its rows' place");

  // a list's column tiles, which read the same rows, one behind the other
  const int units = a.workgroups / a.col_tiles / a.n_chunks;
  const int unit = blockIdx.x % units, tile = blockIdx.x / units % a.col_tiles, chunk = blockIdx.x / units / a.col_tiles;
  const int b = unit / a.Hkv, g = unit % a.Hkv;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 31, half = lane >> 5;
  const bool single = a.n_chunks == 1;
  const int32_t *list = a.lists.table + b * a.lists.table_b + g * a.lists.table_h;
  const char *kb = a.k + g * a.lists.ks[1], *vb = a.v + g * a.lists.vs[1];
  // A single workgroup knows its first rows before it knows the length: their page numbers come beside it.
  // Page numbers of a block, from the list alone; rows behind the end are the last one again, and a page that is not in the pool is page 0
  // (they weigh nothing).
  auto fetch_ids = [&](int block, int slot) CKV_INLINE { dma_4(list + (min(block * 32 + m, a.n_rows - 1) >> a.lists.shift), s_ids[wave][slot]); };
  if (single) {
    fetch_ids(wave, 0);
    fetch_ids(wave + WAVES, 1);
  }
  const TileRange range = tile_range(a, unit, tile);
  const int first = chunk * range.per_chunk, last = min(first + range.per_chunk, range.stages);  // blocks of 32 rows
  const int used = (range.stages + range.per_chunk - 1) / range.per_chunk;  // chunks that have blocks, which are what the merge reads
  const bool alone = single || (a.marks && used <= 1);
  if (range.cols <= 0 || (first >= last && !(alone && chunk == 0))) {
    wait_vm_at_most<0>();
    return;
  }

  const bool valid = m < range.cols;
  const Column c = column(a, unit, tile, valid ? m : 0);
  const int sees_least = __builtin_amdgcn_readfirstlane(c.limit);
  u32x4_d qf[I::STEPS];
  load_query<DT, DH>(a, b, c, valid, half, qf);
  char *k_rows = s_rows[wave], *v_rows = s_rows[wave] + BLOCK;
  auto find_rows = [&](int block, int slot) CKV_INLINE {  // returns which of the 32 are on no page
    const int at = min(m, range.end - 1 - block * 32);
    const int id = s_ids[wave][slot][at], row = (block * 32 + at) & ((1 << a.lists.shift) - 1);
    const bool ok = (unsigned)id < (unsigned)a.lists.n_pages;
    const int64_t page = ok ? id : 0;
    if (half == 0) s_at[wave][m] = Offsets{page * a.lists.ks[0] + row * a.lists.ks[2], page * a.lists.vs[0] + row * a.lists.vs[2]};
    const uint32_t missing = (uint32_t)__ballot(!ok);
    wait_lds_reads();
    return missing;
  };
  auto fetch_k = [&]() CKV_INLINE {
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int row = j * I::ROWS_PER_LOAD + lane / I::PIECES;
      dma_16<STREAM>(kb + s_at[wave][row].k + I::k_piece(row, lane % I::PIECES) * 16, k_rows + 1024 * j);
    }
  };
  auto fetch_v = [&]() CKV_INLINE {
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int row = j * I::ROWS_PER_LOAD + lane / I::PIECES;
      dma_16<STREAM>(vb + s_at[wave][row].v + I::v_piece(row, lane % I::PIECES) * 16, v_rows + 1024 * j);
    }
  };

  Running run;
  f32x16_p acc[I::DTILES];
  const float room = room_for(range.end);
  auto sweep = [&](auto careful, int mode) CKV_INLINE {
    constexpr bool CAREFUL = decltype(careful)::value;
    run = none_yet();
#pragma unroll
    for (int t = 0; t < I::DTILES; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[t][r] = 0.0f;
    int block = first + wave, slot = 0;
    if (block >= last) {
      wait_vm_at_most<0>();  // page numbers that a single workgroup asks for ahead
      return;
    }
    if (!single || CAREFUL) {
      fetch_ids(block, 0);
      fetch_ids(block + WAVES, 1);
    }
    wait_vm_at_most<0>();
    uint32_t missing = find_rows(block, 0);
    fetch_k();
    fetch_v();
    for (; block < last; block += WAVES, slot ^= 1) {
      const bool more = block + WAVES < last;
      uint32_t next_missing = 0;
      f32x16_p z;
      wait_vm_at_most<LOADS>();  // K, and the next page numbers; V may be on its way
      first_product<DT, DH>(k_rows, lane, qf, z);
      wait_lds_reads();
      if (more) {
        next_missing = find_rows(block + WAVES, slot ^ 1);
        fetch_ids(block + 2 * WAVES, slot);
        fetch_k();
      }
      if (missing || (block + 1) * 32 > sees_least) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int row = block_row(r, half);
          if (block * 32 + row >= c.limit || (missing >> row & 1)) z[r] = -INFINITY;
        }
      }
      to_weights<CAREFUL>(z, a.scale2, run, mode, room);
      if (!CAREFUL || mode == kFinite) rescale(acc, run);  // marks are counted, whatever the rows behind them weigh
      if (more) wait_vm_at_most<LOADS + 1>();  // V; the next page numbers and K may be on their way
      else wait_vm_at_most<0>();
      const Weights<DT> weights = as_operand<DT>(z);
      if constexpr (DT == CKV_BF16) second_product<DT, DH, CAREFUL>(v_rows, lane, weights, acc, mode, rest_of(z, weights));
      else second_product<DT, DH, CAREFUL>(v_rows, lane, weights, acc, mode);
      wait_lds_reads();
      if (more) fetch_v();
      missing = next_missing;
    }
  };
  sweep(std::false_type{}, kFinite);
  if (__any(valid && not_finite(acc))) {
    Marks marks;
    for (int mode = kUp; mode <= kFinite; ++mode) {
      sweep(std::true_type{}, mode);
      take_marks(marks, acc, mode);
    }
  }
  run.sum = over_halves(run.sum, [](float x, float y) { return x + y; });

  // the waves' sums in their rows' places, the pieces of a column permuted by it
  if (valid) {
    char *to = s_rows[wave] + m * DH * 4;
#pragma unroll
    for (int t = 0; t < I::DTILES; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *reinterpret_cast<f32x4_p *>(to + (((8 * t + 2 * r + half) ^ m) % PIECES) * 16) =
            f32x4_p{acc[t][4 * r], acc[t][4 * r + 1], acc[t][4 * r + 2], acc[t][4 * r + 3]};
    if (half == 0) s_stats[wave][m] = make_float2(run.top, run.sum);
  }
  __syncthreads();
  const size_t row0 = (((size_t)unit * a.col_tiles + tile) * a.n_chunks + chunk) * kRowsCols;
  for (int i = threadIdx.x; i < range.cols * PIECES; i += WAVES * kWave) {
    const int local = i / PIECES, piece = i % PIECES;
    float top = s_stats[0][local].x, sum = 0.0f;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) top = fmaxf(top, s_stats[w][local].x);
    const float ref = top == -INFINITY ? 0.0f : top;
    float f[WAVES];
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float2 st = s_stats[w][local];
      f[w] = __builtin_amdgcn_exp2f(st.x - ref);
      sum = fmaf(st.y, f[w], sum);
    }
    const float inv = inverse_sum(sum);
    f32x4_p num = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w)
      num = add_part(num, *reinterpret_cast<const f32x4_p *>(s_rows[w] + local * DH * 4 + ((piece ^ local) % PIECES) * 16), f[w] * inv);
    if (alone) {
      const Column o = column(a, unit, tile, local);
      store_out<DT>(out_row(a, b, o), 4 * piece, num);
      if (piece == 0) store_lse(a, b, o, top, sum);
    } else {
      uint64_t *to = reinterpret_cast<uint64_t *>(a.part + (row0 + local) * DH + 4 * piece);
      store_across(to, __builtin_bit_cast(uint64_t, make_float2(num[0], num[1])));
      store_across(to + 1, __builtin_bit_cast(uint64_t, make_float2(num[2], num[3])));
      if (piece == 0) store_across(reinterpret_cast<uint64_t *>(a.stats + row0 + local), __builtin_bit_cast(uint64_t, make_float2(top, sum)));
    }
  }
  if (alone || !a.marks) return;

  wait_vm_at_most<0>();  // what this lane left has arrived
  __syncthreads();
  tag_t *marks = a.marks + ((size_t)unit * a.col_tiles + tile) * a.n_chunks;
  if (wave == 0) {
    if (lane == 0) store_across(marks + chunk, a.tag);
    wait_vm_at_most<0>();
    const bool missing = lane < used && load_across(marks + lane) != a.tag;
    if (lane == 0) s_last = 1;
    if (__any(missing)) s_last = 0;
  }
  __syncthreads();
  if (!s_last) return;
  const size_t tile0 = row0 - (size_t)chunk * kRowsCols;
  float *weights = reinterpret_cast<float *>(s_rows);  // [column][chunk], a wave for a column, a lane for a chunk
  for (int local = wave; local < range.cols; local += WAVES) {
    float2 st = make_float2(-INFINITY, 0.0f);
    if (lane < used)
      st = __builtin_bit_cast(float2, load_across(reinterpret_cast<const uint64_t *>(a.stats + tile0 + (size_t)lane * kRowsCols + local)));
    const float top = over_wave(st.x, -INFINITY, [](float x, float y) { return fmaxf(x, y); });
    const float weight = st.y * __builtin_amdgcn_exp2f(st.x - (top == -INFINITY ? 0.0f : top));
    const float sum = over_wave(weight, 0.0f, [](float x, float y) { return x + y; });
    if (lane < used) weights[local * kMostChunks + lane] = weight * inverse_sum(sum);
    if (lane == 0) store_lse(a, b, column(a, unit, tile, local), top, sum);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < range.cols * PIECES; i += WAVES * kWave) {
    const int local = i / PIECES, piece = i % PIECES;
    const uint64_t *from = reinterpret_cast<const uint64_t *>(a.part + (tile0 + local) * DH + 4 * piece);
    f32x4_p num = {0.0f, 0.0f, 0.0f, 0.0f};
    constexpr int BATCH = 8;
    for (int c0 = 0; c0 < used; c0 += BATCH) {
      float2 x[BATCH][2];
#pragma unroll
      for (int j = 0; j < BATCH; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) x[j][e] = __builtin_bit_cast(float2, load_across(from + (size_t)min(c0 + j, used - 1) * (kRowsCols * DH / 2) + e));
#pragma unroll
      for (int j = 0; j < BATCH; ++j)
        if (c0 + j < used) num = add_part(num, f32x4_p{x[j][0].x, x[j][0].y, x[j][1].x, x[j][1].y}, weights[local * kMostChunks + c0 + j]);
    }
    store_out<DT>(out_row(a, b, column(a, unit, tile, local)), 4 * piece, num);
  }
  if (wave == 0 && lane < used) store_across(marks + lane, (tag_t)0);  // a replay of this launch has the same tag
}

template <int DT, int DH, int WAVES>
static void launch_rows_attention(const PagedArgs &a, hipStream_t stream) {
  // rows that one workgroup only reads are used once
  if (a.col_tiles == 1) hipLaunchKernelGGL((paged_rows_kernel<DT, DH, WAVES, true>), dim3((unsigned)a.workgroups), dim3(WAVES * kWave), 0, stream, a);
  else hipLaunchKernelGGL((paged_rows_kernel<DT, DH, WAVES, false>), dim3((unsigned)a.workgroups), dim3(WAVES * kWave), 0, stream, a);
}

// As many waves as have a place for 32 rows of K and of V each, eight at most.
void launch_paged_rows(const PagedArgs &a, bool bf16, int d, hipStream_t stream) {
  if (bf16 && d == 128) launch_rows_attention<CKV_BF16, 128, 8>(a, stream);
  else if (bf16) launch_rows_attention<CKV_BF16, 64, 8>(a, stream);
  else if (d == 128) launch_rows_attention<CKV_F32, 128, 4>(a, stream);
  else launch_rows_attention<CKV_F32, 64, 8>(a, stream);
}

}  // namespace ckv
