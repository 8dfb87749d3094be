// Attention of new tokens over lists of pages (ckv_paged_attention).
//
// Columns: the queries of a (batch element, KV head), G * i + head, so that neighbours see nearly the same rows and a row is read once
// for all heads of a group. A workgroup takes a tile of columns, 32 per wave, and sweeps the rows that the last of them sees, in stages
// of 64 rows that go from memory to LDS without registers between and are read by all of its waves.
// Rows x queries (32 x 32 matrix tiles, 16 or 2 components at a time) leaves a lane with 16 logits of one column, whose running
// maximum and sum stay in the lane but for one exchange with the other half of the wave, and which are the operand of the second product as
// they lie: the contraction over rows may be permuted if both operands agree, so V's operand takes the rows in the order that the
// logits have. V lies in LDS as it does in memory and is transposed on its way into registers.
// LDS images are swizzled in units that one cycle reads (16 bytes of eight rows of K, 32 bytes of four rows of V).
// Measured: bf16, 32/8 heads of 128, 2048 new tokens behind 30720 rows: 1.00 to 1.07 ms by card, up to 1064 TFLOP/s of the two products, where a
// plain 8192^3 product reaches 1241; batch 2, 32/32 heads, up to 4096 tokens over themselves: 270 to 290 us, up to 827 TFLOP/s. A stage of 64 rows
// takes a wave 3720 cycles, in 55 % of which the matrix cores work; without operands from LDS it is 6 % less, without the softmax's sums 3 %, so that what is left is
// the issue of what stands beside the products, at the 1.93 GHz that the card holds under this load. (No gain: loads
// spread over a step's slots, operands three slots ahead, priorities of waves.) f32: the f32 products' rate, a sixteenth of bf16's.
//
// What a token does not see must not touch its result even if it is infinite or NaN, and zero times infinity is NaN: where a sweep leaves
// something that is not finite, the workgroup sweeps again, with V's finite components only, and twice more for where its
// infinite and NaN ones are. Sums that are beyond fp32 where their mean is not get a reference there that leaves them room.
#include "ckv_paged.h"

namespace ckv {

constexpr int kStageRows = 64;  // two blocks of 32 rows

// A whole step in bf16, its instructions in the order that they are issued in: slot by slot a matrix product (the two kinds in turn), the operands
// of those two or four slots further on, and a share of the softmax: first the maximum, then a few exponentials each. Left to itself the compiler puts
// all products first, each behind a wait for its operand. `next` gets the logits of K's block, `weights` changes from the block before to z's.
template <int DT, int DH>
__device__ __forceinline__ void whole_step(const char *k_image, const char *v_image, int lane, const u32x4_d (&qf)[Image<DT, DH>::STEPS],
                                           const f32x16_p &z, f32x16_p &next, Weights<DT> &weights, f32x16_p (&acc)[DH / 32], float scale2, Running &run) {
  constexpr int STEPS = DH / 16, DTILES = DH / 32, SLOTS = 2 * STEPS, MAX_SLOTS = SLOTS / 4, EXP_SLOTS = SLOTS - MAX_SLOTS;
  constexpr int AHEAD = 2;
  static_assert(DT == CKV_BF16 && 2 * DTILES == STEPS, "as many products of one kind as of the other");
  const int k_at = k_lane<CKV_BF16, DH>(lane), v_at = v_lane<DH>(lane);
  u32x4_d kf[STEPS], vf[STEPS];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) {
    kf[i] = k_operand(k_image, k_at, i);
    vf[i] = v_operand<DH>(v_image, v_at, i % DTILES, i / DTILES);
  }
  float mx = z[0], part[4], w[16];
  Weights<DT> made;
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int slot = 0; slot < SLOTS; ++slot) {
    const int i = slot / 2;
    if (slot % 2 == 0) {
      if (i + AHEAD < STEPS) kf[i + AHEAD] = k_operand(k_image, k_at, i + AHEAD);
      if (i == 0) {
#pragma unroll
        for (int r = 0; r < 16; ++r) next[r] = 0.0f;
      }
      mma_piece<CKV_BF16>(next, kf[i], qf[i]);
    } else {
      if (i + AHEAD < STEPS) vf[i + AHEAD] = v_operand<DH>(v_image, v_at, (i + AHEAD) % DTILES, (i + AHEAD) / DTILES);
      mma_piece<CKV_BF16>(acc[i % DTILES], vf[i], weights.piece[i / DTILES]);
    }
    if (slot < MAX_SLOTS) {
#pragma unroll
      for (int r = slot * 16 / MAX_SLOTS; r < (slot + 1) * 16 / MAX_SLOTS; ++r) mx = fmaxf(mx, z[r]);
      if (slot == MAX_SLOTS - 1) take_maximum(mx, scale2, run);
    } else {
#pragma unroll
      for (int r = (slot - MAX_SLOTS) * 16 / EXP_SLOTS; r < (slot - MAX_SLOTS + 1) * 16 / EXP_SLOTS; ++r) {
        w[r] = __builtin_amdgcn_exp2f(fmaf(z[r], scale2, -run.ref));
        part[r % 4] = r < 4 ? w[r] : part[r % 4] + w[r];
        if (r % 2) made.piece[r / 8][r / 2 % 4] = pack_bf16(w[r - 1], w[r]);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  run.sum += (part[0] + part[1]) + (part[2] + part[3]);
  weights = made;
}

template <int DT, int DH, int WAVES>
__global__ void __launch_bounds__(WAVES *kWave, WAVES == 4 && DT == CKV_F32 && DH == 128 ? 1 : 2) paged_tile_kernel(PagedArgs a) {
  typedef Image<DT, DH> I;
  constexpr int BYTES = kStageRows * I::ROW;
  constexpr int LOADS = BYTES / 1024 / WAVES;       // of K per wave and stage, and of V
  static_assert(LOADS * WAVES * 1024 == BYTES && kStageRows == kWave, "whole loads, a lane for every row");
  __shared__ __align__(1024) char s_k[2][BYTES];
  __shared__ __align__(1024) char s_v[2][BYTES];
  __shared__ __align__(256) int32_t s_ids[2][kWave];
  struct Offsets {
    int64_t k, v;
  };
  __shared__ Offsets s_at[4][kStageRows];
  __shared__ int s_missing, s_undefined;

  // The longest tiles first, of all lists; the lists side by side, so that with a multiple of eight of them a list's workgroups share an L2.
  const int units = a.workgroups / a.col_tiles / a.n_chunks;
  const int unit = blockIdx.x % units, chunk = blockIdx.x / units % a.n_chunks;
  const int tile = a.col_tiles - 1 - blockIdx.x / units / a.n_chunks;
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
  const int sees_least = __builtin_amdgcn_readfirstlane(c.limit);  // the wave's first column sees the fewest rows
  // The wave is through behind the rows that its own columns see.
  const int sees_most = wave * 32 < range.cols ? column(a, unit, tile, min(range.cols, wave * 32 + 32) - 1).limit : 0;
  const int own_last = max(min(last, (sees_most + kStageRows - 1) / kStageRows), first + 1);
  u32x4_d qf[I::STEPS];
  load_query<DT, DH>(a, b, c, valid, half, qf);

  const int32_t *list = a.lists.table + b * a.lists.table_b + g * a.lists.table_h;
  const char *kb = a.k + g * a.lists.ks[1], *vb = a.v + g * a.lists.vs[1];
  if (threadIdx.x == 0) s_missing = s_undefined = 0;
  __syncthreads();

  // Where the rows of a stage are: one wave, another for every stage, turns its page numbers into offsets, two stages ahead of the first loads that
  // need them. Rows behind the end are the last one again; a page that is not in the pool is page 0 (they weigh nothing).
  auto row_of = [&](int stage) CKV_INLINE { return min(stage * kStageRows + lane, range.end - 1); };
  auto fetch_ids = [&](int stage) CKV_INLINE {
    if (wave == stage % WAVES) dma_4(list + (row_of(stage) >> a.lists.shift), s_ids[stage & 1]);
  };
  auto find_rows = [&](int stage) CKV_INLINE {
    if (wave != stage % WAVES) return;
    const int id = s_ids[stage & 1][lane], row = row_of(stage) & ((1 << a.lists.shift) - 1);
    const bool ok = (unsigned)id < (unsigned)a.lists.n_pages;
    const int64_t page = ok ? id : 0;
    if (!ok) s_missing = 1;
    s_at[stage & 3][lane] = Offsets{page * a.lists.ks[0] + row * a.lists.ks[2], page * a.lists.vs[0] + row * a.lists.vs[2]};
  };
  auto fetch_k = [&](int stage) CKV_INLINE {
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int row = (wave * LOADS + j) * I::ROWS_PER_LOAD + lane / I::PIECES;
      dma_16<false>(kb + s_at[stage & 3][row].k + I::k_piece(row, lane % I::PIECES) * 16, s_k[(stage - first) & 1] + (wave * LOADS + j) * 1024);
    }
  };
  auto fetch_v = [&](int stage) CKV_INLINE {
#pragma unroll
    for (int j = 0; j < LOADS; ++j) {
      const int row = (wave * LOADS + j) * I::ROWS_PER_LOAD + lane / I::PIECES;
      dma_16<false>(vb + s_at[stage & 3][row].v + I::v_piece(row, lane % I::PIECES) * 16, s_v[(stage - first) & 1] + (wave * LOADS + j) * 1024);
    }
  };

  Running run;
  f32x16_p acc[I::DTILES];
  auto begin = [&]() CKV_INLINE {
    run = none_yet();
#pragma unroll
    for (int t = 0; t < I::DTILES; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[t][r] = 0.0f;
  };
  // logits of rows that the column does not see
  auto hide = [&](f32x16_p &z, int z_row) CKV_INLINE {
    if (!s_missing && z_row + 32 <= sees_least) return;
    const int sees = c.limit - z_row - 4 * half;  // rows of the block from the half's first one on
    uint32_t there = ~0u;
    if (s_missing) {
      there = 0;
#pragma unroll 1
      for (int r = 0; r < 16; ++r) {
        const int row = min(z_row + block_row(r, half), range.end - 1);
        there |= ((unsigned)list[row >> a.lists.shift] < (unsigned)a.lists.n_pages ? 1u : 0u) << r;
      }
    }
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (block_row(r, 0) >= sees || !(there >> r & 1)) z[r] = -INFINITY;
  };
  constexpr int HALF = 32 * I::ROW;

  begin();
  if (first < last) {
    for (int i = 0; i < 2; ++i) {  // the first two stages' rows, each by its wave, one behind the other
      fetch_ids(first + i);
      wait_vm_at_most<0>();
      find_rows(first + i);
      __syncthreads();
    }
    fetch_ids(first + 2);
    fetch_k(first);
    f32x16_p z;           // logits of the block in work
    Weights<DT> weights;  // of the one before
    // Steps of the pipeline: the first product of a block, the softmax of the one before, the second product of the one before that, none
    // of which waits for another: the matrix cores have work while the vector units are at the softmax. What is a branch comes in
    // front, so that the rest is one block of instructions to be scheduled.
    auto softmax = [&]() CKV_INLINE {
      to_weights<false>(z, a.scale2, run, kFinite);
      weights = as_operand<DT>(z);
    };
    auto step = [&](const char *k_image, int z_row, const char *v_image) CKV_INLINE {
      rescale(acc, run);
      hide(z, z_row);
      f32x16_p next;
      if constexpr (DT == CKV_BF16) {
        whole_step<DT, DH>(k_image, v_image, lane, qf, z, next, weights, acc, a.scale2, run);
      } else {
        first_product<DT, DH>(k_image, lane, qf, next);
        second_product<DT, DH, false>(v_image, lane, weights, acc, kFinite);
        softmax();
      }
      pin(weights, run.sum);  // or the exponentials move behind the next step's branch, away from these products
      z = next;
    };
    auto advance = [&](int stage) CKV_INLINE {
      wait_vm_at_most<0>();
      __syncthreads();  // K of this stage and V of the one before are there, and the buffers of the next loads have been read
      if (stage + 2 < last) find_rows(stage + 2);
      if (stage < last) fetch_v(stage);
      if (stage + 1 < last) fetch_k(stage + 1);
      if (stage + 3 < last) fetch_ids(stage + 3);
    };
    f32x16_p next;
    advance(first);
    first_product<DT, DH>(s_k[0], lane, qf, z);
    hide(z, first * kStageRows);
    first_product<DT, DH>(s_k[0] + HALF, lane, qf, next);
    softmax();
    z = next;
    // buffers known at compile time: operands at fixed offsets from a few addresses
    auto stage_of = [&](auto parity, int stage) CKV_INLINE {
      constexpr int BUF = decltype(parity)::value;
      advance(stage);
      step(s_k[BUF], stage * kStageRows - 32, s_v[BUF ^ 1]);
      step(s_k[BUF] + HALF, stage * kStageRows, s_v[BUF ^ 1] + HALF);
    };
    int stage = first + 1;
#pragma unroll 1
    for (; stage + 1 < own_last; stage += 2) {
      stage_of(std::integral_constant<int, 1>{}, stage);
      stage_of(std::integral_constant<int, 0>{}, stage + 1);
    }
    if (stage < own_last) stage_of(std::integral_constant<int, 1>{}, stage);
    advance(own_last);
    const char *v = s_v[(own_last - 1 - first) & 1];
    rescale(acc, run);
    second_product<DT, DH, false>(v, lane, weights, acc, kFinite);
    hide(z, own_last * kStageRows - 32);
    softmax();
    rescale(acc, run);
    second_product<DT, DH, false>(v + HALF, lane, weights, acc, kFinite);
    for (stage = own_last + 1; stage <= last; ++stage) advance(stage);  // the other waves' rows, and all barriers
  }
  if (valid && not_finite(acc)) s_undefined = 1;
  __syncthreads();
  if (s_undefined) {  // the same for all waves, as there are barriers in the sweeps; one block after the other
    Marks marks;
    const float room = room_for(range.end);
#pragma unroll 1
    for (int mode = kUp; mode <= kFinite; ++mode) {
      begin();
#pragma unroll 1
      for (int stage = first; stage < last; ++stage) {
        __syncthreads();  // the buffers have been read
        fetch_ids(stage);
        wait_vm_at_most<0>();
        find_rows(stage);
        __syncthreads();
        fetch_k(stage);
        fetch_v(stage);
        wait_vm_at_most<0>();
        __syncthreads();
#pragma unroll 1
        for (int k = 0; k < 2; ++k) {
          f32x16_p z;
          first_product<DT, DH>(s_k[(stage - first) & 1] + k * HALF, lane, qf, z);
          hide(z, stage * kStageRows + 32 * k);
          to_weights<true>(z, a.scale2, run, mode, room);
          if (mode == kFinite) rescale(acc, run);  // marks are counted, whatever the row behind them weighs
          second_product<DT, DH, true>(s_v[(stage - first) & 1] + k * HALF, lane, as_operand<DT>(z), acc, mode);
        }
      }
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
      else *reinterpret_cast<f32x4_p *>(a.part + row * DH + d) = x * inv;
    }
  if (half == 0) {
    if (single) store_lse(a, b, c, run.top, run.sum);
    else a.stats[row] = make_float2(run.top, run.sum);
  }
}

// Chunks of a column, in their order. A column's lanes take four components each, and for the weights a chunk each; loads of eight chunks are in flight
// together (one after the other, sixteen chunks took 12 us, now 5).
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
  float2 st[SHARE];
  float top = -INFINITY;
#pragma unroll
  for (int k = 0; k < SHARE; ++k) {
    const int i = k * PIECES + piece;
    st[k] = make_float2(-INFINITY, 0.0f);
    if (i < chunks) st[k] = a.stats[first + (size_t)i * a.tile_cols];
    top = fmaxf(top, st[k].x);
  }
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
  constexpr int BATCH = 8;
#pragma unroll
  for (int k = 0; k < SHARE; ++k) {
    for (int c0 = 0; c0 < PIECES && k * PIECES + c0 < a.n_chunks; c0 += BATCH) {  // the same for all lanes
      f32x4_p x[BATCH];
#pragma unroll
      for (int j = 0; j < BATCH; ++j) {
        const int i = k * PIECES + c0 + j;
        x[j] = f32x4_p{0.0f, 0.0f, 0.0f, 0.0f};
        if (i < chunks) x[j] = *reinterpret_cast<const f32x4_p *>(a.part + (first + (size_t)i * a.tile_cols) * DH + 4 * piece);
      }
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
PagedPlan plan_paged(const Shape &s, int n_rows) {
  PagedPlan p;
  const bool bf16 = s.esize == 2;
  const int64_t units = (int64_t)s.Bz * s.Hkv, cols = (int64_t)s.G * s.T;
  p.by_rows = cols <= (bf16 ? kMostRowsCols : kMostRowsColsF32);
  const int waves = units * ((cols + 255) / 256) >= kComputeUnits ? 8 : 4;
  p.tile_cols = p.by_rows ? kRowsCols : waves * 32;
  p.stage_rows = p.by_rows ? 32 : kStageRows;
  p.col_tiles = (int)((cols + p.tile_cols - 1) / p.tile_cols);
  const int64_t tiles = units * p.col_tiles;
  const bool two = !p.by_rows && waves == 4 && (bf16 || s.d == 64 || n_rows < 1024);
  int64_t chunks = (two ? 2 : 1) * kComputeUnits / tiles;
  const int least = p.by_rows ? (bf16 ? 256 : 128) : bf16 ? 512 : s.d == 64 ? 64 : 128;
  const int64_t most = p.by_rows && n_rows <= (bf16 ? 1024 : 256) ? 1 : (n_rows + least - 1) / least;
  if (chunks > most) chunks = most;
  if (chunks > kMostChunks) chunks = kMostChunks;
  if (chunks < 1) chunks = 1;
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
static void launch_paged_of(const PagedArgs &a, const PagedPlan &plan, int units, hipStream_t stream) {
  if (plan.by_rows) launch_paged_rows(a, DT == CKV_BF16, DH, stream);
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
                                  const int32_t *count, int n_rows, void *out, const int64_t *out_stride, float *lse, char *ws,
                                  hipStream_t stream) {
  const int units = s.Bz * s.Hkv;
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
