// Attention of new tokens over lists of pages for many columns (ckv_paged_attention, ckv_paged_tree_attention): a tile of columns by a workgroup.
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
#ifndef CKV_PAGED_TILE_H_
#define CKV_PAGED_TILE_H_

#include "ckv_paged.h"

namespace ckv {

constexpr int kStageRows = 64;  // two blocks of 32 rows

// A whole step in bf16, its instructions in the order that they are issued in: slot by slot a matrix product (the two kinds in turn), the operands
// of those two or four slots further on, and a share of the softmax: first the maximum, then a few exponentials each. Left to itself the compiler puts
// all products first, each behind a wait for its operand. `next` gets the logits of K's block, `weights` change from the block before to z's.
// TWO: the second product takes them in two terms, `rest` what the rounding of the first one leaves, with the first product's slot between the two.
template <int DT, int DH, bool TWO>
__device__ __forceinline__ void whole_step(const char *k_image, const char *v_image, int lane, const u32x4_d (&qf)[Image<DT, DH>::STEPS],
                                           const f32x16_p &z, f32x16_p &next, Weights<DT> &weights, Weights<DT> &rest, f32x16_p (&acc)[DH / 32],
                                           float scale2, Running &run) {
  constexpr int STEPS = DH / 16, DTILES = DH / 32, KINDS = TWO ? 3 : 2, SLOTS = KINDS * STEPS, MAX_SLOTS = SLOTS / 4, EXP_SLOTS = SLOTS - MAX_SLOTS;
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
  Weights<DT> made, left;
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int slot = 0; slot < SLOTS; ++slot) {
    const int i = slot / KINDS, kind = TWO && slot % 3 < 2 ? 1 - slot % 3 : slot % KINDS;  // 0: the first product, 1, 2: a term of the second
    if (kind == 0) {
      if (i + AHEAD < STEPS) kf[i + AHEAD] = k_operand(k_image, k_at, i + AHEAD);
      if (i == 0) {
#pragma unroll
        for (int r = 0; r < 16; ++r) next[r] = 0.0f;
      }
      mma_piece<CKV_BF16>(next, kf[i], qf[i]);
    } else {
      if (kind == 1 && i + AHEAD < STEPS) vf[i + AHEAD] = v_operand<DH>(v_image, v_at, (i + AHEAD) % DTILES, (i + AHEAD) / DTILES);
      mma_piece<CKV_BF16>(acc[i % DTILES], vf[i], (kind == 1 ? weights : rest).piece[i / DTILES]);
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
        if (r % 2) {
          const uint32_t both = pack_bf16(w[r - 1], w[r]);
          made.piece[r / 8][r / 2 % 4] = both;
          if (TWO) left.piece[r / 8][r / 2 % 4] = rest_of(w[r - 1], w[r], both);
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  run.sum += (part[0] + part[1]) + (part[2] + part[3]);
  weights = made;
  if (TWO) rest = left;
}

// Waves of a tile's kernel that a SIMD holds, for its __launch_bounds__.
constexpr int tile_occupancy(int dt, int d, int waves) { return waves == 4 && dt == CKV_F32 && d == 128 ? 1 : 2; }

// Args: PagedArgs, or TreeArgs, whose tokens see of the new ones what their words say. GROUPS = 2: half of the
// waves take the first half of the chunk's stages, the others the second half, for the same columns, each with buffers of its own, and they are joined
// in LDS: as many waves as two workgroups, whose sums would go through memory and a launch. us, bf16, two workgroups / groups: 500 tokens, 32/8 heads,
// batch 2, 4099 rows 117 / 106, 563 rows 37.5 / 28.6, 59 tokens, heads of 64, batch 12, 793 rows 27.7 / 21.5, 41 tokens, 16/2 heads, batch 8, 9312 rows 60.0 / 57.7.
template <int DT, int DH, int WAVES, int GROUPS, class Args>
__device__ __forceinline__ void attend_tile(const Args &a) {
  constexpr bool TREE = std::is_same<Args, TreeArgs>::value;
  constexpr bool TWO = TREE && DT == CKV_BF16;  // terms of the weights in the second product
  typedef Image<DT, DH> I;
  constexpr int BYTES = kStageRows * I::ROW;
  constexpr int MEMBERS = WAVES / GROUPS;           // waves of a group
  constexpr int LOADS = BYTES / 1024 / MEMBERS;     // of K per wave and stage, and of V
  static_assert(LOADS * MEMBERS * 1024 == BYTES && kStageRows == kWave, "whole loads, a lane for every row");
  static_assert(GROUPS == 1 || TREE, "the second group waits at as many barriers as the first, which are counted for trees");
  __shared__ __align__(1024) char s_all_k[GROUPS][2][BYTES];
  __shared__ __align__(1024) char s_all_v[GROUPS][2][BYTES];
  __shared__ __align__(256) int32_t s_all_ids[GROUPS][2][kWave];
  struct Offsets {
    int64_t k, v;
  };
  __shared__ Offsets s_all_at[GROUPS][4][kStageRows];
  __shared__ float2 s_stats[GROUPS > 1 ? MEMBERS : 1][32];
  __shared__ int s_missing, s_undefined;
  __shared__ __align__(256) uint32_t s_sees[TREE ? WAVES : 1][2][TREE ? 2 * kWave : 1];

  // The longest tiles first, of all lists; the lists side by side, so that with a multiple of eight of them a list's workgroups share an L2.
  const int units = a.workgroups / a.col_tiles / a.n_chunks;
  const int unit = blockIdx.x % units, chunk = blockIdx.x / units % a.n_chunks;
  const int tile = a.col_tiles - 1 - blockIdx.x / units / a.n_chunks;
  const int b = unit / a.Hkv, g = unit % a.Hkv;
  const int lane = threadIdx.x & 63, wave_in_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  const int group = GROUPS == 1 ? 0 : wave_in_all / MEMBERS, wave = GROUPS == 1 ? wave_in_all : wave_in_all % MEMBERS;
  auto &s_k = s_all_k[group];
  auto &s_v = s_all_v[group];
  auto &s_ids = s_all_ids[group];
  auto &s_at = s_all_at[group];
  const TileRange range = tile_range(a, unit, tile);
  if (range.cols <= 0) return;
  int first = chunk * range.per_chunk, last = min(first + range.per_chunk, range.stages);
  const bool single = a.n_chunks == 1;
  if (first >= last && !single) return;  // the merge reads the chunks that have stages
  const int most = GROUPS == 1 ? last - first : (last - first + 1) / 2;  // stages of the first group, which the second has too or one less
  if (GROUPS > 1) {
    const int between = first + most;
    if (group == 0) last = between;
    else first = between;
  }

  const int local = wave * 32 + (lane & 31);
  const bool valid = local < range.cols;
  const Column c = column(a, unit, tile, valid ? local : 0);
  const int start = TREE ? first_new(a, unit) : 0;
  const int sees_first = __builtin_amdgcn_readfirstlane(c.limit);  // the wave's first column sees the fewest rows
  const int sees_least = TREE ? min(sees_first, start) : sees_first;  // of a tree those in front of the new ones
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
    if (wave == stage % MEMBERS) dma_4(list + (row_of(stage) >> a.lists.shift), s_ids[stage & 1]);
  };
  auto find_rows = [&](int stage) CKV_INLINE {
    if (wave != stage % MEMBERS) return;
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

  // A wave's columns' words of the rows that it hides in a stage, from 32 rows in front of it on: three words, a stage ahead, two of each
  // column and then the third.
  auto fetch_sees = [&](int stage) CKV_INLINE {
    if constexpr (TREE) {
      const int w = (stage * kStageRows - 32 - start) >> 5;
      if (w + 2 < 0 || w >= a.words) return;  // the same for all lanes
      const uint32_t *own = words_of(a, unit) + (size_t)c.token * a.words;
      dma_4(own + min(max(w + half, 0), a.words - 1), s_sees[wave_in_all][stage & 1]);
      dma_4(own + min(w + 2, a.words - 1), s_sees[wave_in_all][stage & 1] + kWave);
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
  // logits of rows that the column does not see; `stage`: whose words are there, or -1
  auto hide = [&](f32x16_p &z, int z_row, int stage) CKV_INLINE {
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
    if constexpr (TREE) {
      const auto word = [&](int w) CKV_INLINE {
        if (stage < 0) return words_of(a, unit)[(size_t)c.token * a.words + w];
        return s_sees[wave_in_all][stage & 1][(w - ((stage * kStageRows - 32 - start) >> 5)) * 32 + (lane & 31)];
      };
      const uint32_t seen = rows_of_tree(a, c.limit, z_row, z_row - start, word) >> (4 * half);
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (!(seen >> block_row(r, 0) & 1) || !(there >> r & 1)) z[r] = -INFINITY;
    } else {
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (block_row(r, 0) >= sees || !(there >> r & 1)) z[r] = -INFINITY;
    }
  };
  constexpr int HALF = 32 * I::ROW;

  begin();
  if (first < last) {
    if constexpr (TREE) {  // the first two stages' rows, each by its wave
      for (int i = 0; i < 2; ++i) fetch_ids(first + i);
      wait_vm_at_most<0>();
      for (int i = 0; i < 2; ++i) find_rows(first + i);
      __syncthreads();
    } else {  // ... one behind the other
      for (int i = 0; i < 2; ++i) {
        fetch_ids(first + i);
        wait_vm_at_most<0>();
        find_rows(first + i);
        __syncthreads();
      }
    }
    fetch_ids(first + 2);
    fetch_k(first);
    fetch_sees(first);
    f32x16_p z;           // logits of the block in work
    Weights<DT> weights, rest;  // of the one before
    // Steps of the pipeline: the first product of a block, the softmax of the one before, the second product of the one before that, none
    // of which waits for another: the matrix cores have work while the vector units are at the softmax. What is a branch comes in
    // front, so that the rest is one block of instructions to be scheduled.
    auto softmax = [&]() CKV_INLINE {
      to_weights<false>(z, a.scale2, run, kFinite);
      weights = as_operand<DT>(z);
      if constexpr (TWO) rest = rest_of(z, weights);
    };
    auto step = [&](const char *k_image, int z_row, const char *v_image, int stage) CKV_INLINE {
      rescale(acc, run);
      hide(z, z_row, stage);
      f32x16_p next;
      if constexpr (DT == CKV_BF16) {
        whole_step<DT, DH, TWO>(k_image, v_image, lane, qf, z, next, weights, rest, acc, a.scale2, run);
      } else {
        first_product<DT, DH>(k_image, lane, qf, next);
        second_product<DT, DH, false>(v_image, lane, weights, acc, kFinite);
        softmax();
      }
      if constexpr (TWO) pin(rest, run.sum);
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
      if (stage + 1 <= last) fetch_sees(stage + 1);
    };
    f32x16_p next;
    advance(first);
    first_product<DT, DH>(s_k[0], lane, qf, z);
    hide(z, first * kStageRows, first);
    first_product<DT, DH>(s_k[0] + HALF, lane, qf, next);
    softmax();
    z = next;
    // buffers known at compile time: operands at fixed offsets from a few addresses
    auto stage_of = [&](auto parity, int stage) CKV_INLINE {
      constexpr int BUF = decltype(parity)::value;
      advance(stage);
      step(s_k[BUF], stage * kStageRows - 32, s_v[BUF ^ 1], stage);
      step(s_k[BUF] + HALF, stage * kStageRows, s_v[BUF ^ 1] + HALF, stage);
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
    if constexpr (TWO) second_product<DT, DH, false>(v, lane, weights, acc, kFinite, rest);
    else second_product<DT, DH, false>(v, lane, weights, acc, kFinite);
    hide(z, own_last * kStageRows - 32, own_last);
    softmax();
    rescale(acc, run);
    if constexpr (TWO) second_product<DT, DH, false>(v + HALF, lane, weights, acc, kFinite, rest);
    else second_product<DT, DH, false>(v + HALF, lane, weights, acc, kFinite);
    for (stage = own_last + 1; stage <= last; ++stage) advance(stage);  // the other waves' rows, and all barriers
  }
  if (GROUPS > 1 && last - first < most)
    for (int i = last > first ? 1 : 3; i > 0; --i) __syncthreads();  // of a stage; of the one stage and what is around it
  if (valid && not_finite(acc)) s_undefined = 1;
  __syncthreads();
  if (s_undefined) {  // the same for all waves, as there are barriers in the sweeps; one block after the other
    Marks marks;
    const float room = room_for(range.end);
#pragma unroll 1
    for (int mode = kUp; mode <= kFinite; ++mode) {
      begin();
#pragma unroll 1
      for (int stage = first; stage < first + most; ++stage) {
        const bool mine = GROUPS == 1 || stage < last;
        __syncthreads();  // the buffers have been read
        if (mine) fetch_ids(stage);
        wait_vm_at_most<0>();
        if (mine) find_rows(stage);
        __syncthreads();
        if (mine) fetch_k(stage);
        if (mine) fetch_v(stage);
        wait_vm_at_most<0>();
        __syncthreads();
        if (!mine) continue;
#pragma unroll 1
        for (int k = 0; k < 2; ++k) {
          f32x16_p z;
          first_product<DT, DH>(s_k[(stage - first) & 1] + k * HALF, lane, qf, z);
          hide(z, stage * kStageRows + 32 * k, -1);
          to_weights<true>(z, a.scale2, run, mode, room);
          if (mode == kFinite) rescale(acc, run);  // marks are counted, whatever the row behind them weighs
          const Weights<DT> operand = as_operand<DT>(z);
          if constexpr (TWO) second_product<DT, DH, true>(s_v[(stage - first) & 1] + k * HALF, lane, operand, acc, mode, rest_of(z, operand));
          else second_product<DT, DH, true>(s_v[(stage - first) & 1] + k * HALF, lane, operand, acc, mode);
        }
      }
      take_marks(marks, acc, mode);
    }
  }
  run.sum = over_halves(run.sum, [](float x, float y) { return x + y; });
  if constexpr (GROUPS > 1) {
    static_assert(GROUPS == 1 || (MEMBERS == 4 && I::DTILES * 4 * 1024 == BYTES), "a wave's sums take the place of a buffer");
    // The second group's sums, in its rows' places, joined with the first one's as chunks are.
    __syncthreads();
    char *sums = wave < 2 ? s_all_k[1][wave] : s_all_v[1][wave - 2];
    const auto place = [&](int t, int r) CKV_INLINE { return reinterpret_cast<f32x4_p *>(sums + (4 * t + r) * 1024 + lane * 16); };
    const float inv = inverse_sum(run.sum);
    if (group == 1) {
#pragma unroll
      for (int t = 0; t < I::DTILES; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) *place(t, r) = f32x4_p{acc[t][4 * r], acc[t][4 * r + 1], acc[t][4 * r + 2], acc[t][4 * r + 3]} * inv;
      if (half == 0) s_stats[wave][lane] = make_float2(run.top, run.sum);
    }
    __syncthreads();
    if (group == 1) return;
    const float2 other = s_stats[wave][lane & 31];
    const float top = fmaxf(run.top, other.x), ref = top == -INFINITY ? 0.0f : top;
    float mine = run.sum * __builtin_amdgcn_exp2f(run.top - ref), its = other.y * __builtin_amdgcn_exp2f(other.x - ref);
    const float sum = mine + its, share = inverse_sum(sum);
    mine *= share;
    its *= share;
#pragma unroll
    for (int t = 0; t < I::DTILES; ++t)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const f32x4_p own = f32x4_p{acc[t][4 * r], acc[t][4 * r + 1], acc[t][4 * r + 2], acc[t][4 * r + 3]} * inv;
        const f32x4_p x = add_part(add_part(f32x4_p{0.0f, 0.0f, 0.0f, 0.0f}, own, mine), *place(t, r), its);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[t][4 * r + e] = x[e];
      }
    run.top = top;
    run.sum = sum;
  }
  if (!valid) return;

  const size_t row = (((size_t)unit * a.col_tiles + tile) * a.n_chunks + chunk) * a.tile_cols + local;
  char *to = out_row(a, b, c);
  const float inv = GROUPS > 1 ? 1.0f : inverse_sum(run.sum);
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

}  // namespace ckv
#endif
