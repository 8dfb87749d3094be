// What the kernels of ckv_paged_attention share (private): the matrix forms of the two products, and how a call is shared out.
#ifndef CKV_PAGED_H_
#define CKV_PAGED_H_

#include <type_traits>

#include "ckv_pages.h"
#include <ckv_dma.h>

namespace ckv {

struct PagedArgs {
  const char *q, *k, *v;
  int64_t qs[3];       // BYTES between batch elements, query heads, tokens
  PageLists lists;
  char *out;
  int64_t os[3];       // BYTES, as qs
  float *lse;          // [Bz][Hq][n] natural log, or null
  float *part;         // [unit][column tile][chunk][column of the tile][d]: the chunk's own result, in fp32
  float2 *stats;       // [unit][column tile][chunk][column of the tile]: reference of its weights (log2), their sum
  int Hq, Hkv, G, n, n_rows;
  int tile_cols, col_tiles, stage_rows, n_chunks, workgroups;  // of the plan
  tag_t *marks;        // [unit][column tile][chunk] or null: who finds a tile's marks complete joins its chunks, no kernel behind this one
  tag_t tag;           // of the launch
  float scale2;        // softmax scale * log2(e)
};
constexpr int kMostChunks = 64;  // a lane for each

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_p;
typedef __attribute__((ext_vector_type(16))) float f32x16_p;
typedef __attribute__((ext_vector_type(4))) float f32x4_p;
typedef __attribute__((ext_vector_type(4))) short s16x4_p;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_p;

// Four 16-bit words a lane, transposed among 16 lanes: lane i gets word i % 4 of what lanes i / 4, 4 + i / 4, 8 + i / 4, 12 + i / 4 read.
__device__ __forceinline__ u32x2_p read_transposed(const char *lds) {
  typedef __attribute__((address_space(3))) s16x4_p lds_words;
  return __builtin_bit_cast(u32x2_p, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_words *)lds));
}

// Rows as they lie in LDS: one behind the other, the 16-byte pieces of a row permuted so that what one cycle reads (16 bytes of eight
// rows of K, 32 bytes of four rows of V) lies in different banks. Both permutations are their own inverses.
template <int DT, int DH>
struct Image {
  static constexpr int ROW = DH * (DT == CKV_BF16 ? 2 : 4);  // bytes
  static constexpr int PIECES = ROW / 16;
  static constexpr int ROWS_PER_LOAD = 1024 / ROW;           // a wave's load of 16 bytes a lane
  static constexpr int STEPS = PIECES / 2;                   // pieces of a row per half of the wave
  static constexpr int DTILES = DH / 32;
  static __device__ __forceinline__ int k_piece(int r, int c) { return c ^ (ROW == 128 ? (r >> 1) & 7 : r & 15); }
  static __device__ __forceinline__ int v_piece(int r, int c) {
    if (DT != CKV_BF16) return c;  // a cycle reads 32 lanes' words of one row
    return c ^ (4 * (ROW == 128 ? (r >> 1) & 1 : r & 3));
  }
};

// The rows that a tile's columns see, and how its chunks share them: whole stages.
struct TileRange {
  int cols;  // columns of the tile that exist
  int end;   // rows that the last of them sees
  int stages, per_chunk;
};
__device__ __forceinline__ TileRange tile_range(const PagedArgs &a, int unit, int tile) {
  TileRange t;
  const int count = new_rows(a.lists, unit, a.n), length = max(a.lists.length[unit], 0);
  t.cols = min(a.G * count - tile * a.tile_cols, a.tile_cols);
  const int last = (tile * a.tile_cols + t.cols - 1) / a.G;
  t.end = t.cols > 0 ? min(max(length - count + last + 1, 0), a.n_rows) : 0;
  t.stages = (t.end + a.stage_rows - 1) / a.stage_rows;
  t.per_chunk = max(1, (t.stages + a.n_chunks - 1) / a.n_chunks);
  return t;
}

// Column `local` of a tile: a token and one of the group's heads.
struct Column {
  int token, h;
  int limit;  // rows that it sees
};
__device__ __forceinline__ Column column(const PagedArgs &a, int unit, int tile, int local) {
  const int col = tile * a.tile_cols + local, g = unit % a.Hkv;
  Column c;
  c.token = col / a.G;
  c.h = g * a.G + col - c.token * a.G;
  c.limit = min(max(max(a.lists.length[unit], 0) - new_rows(a.lists, unit, a.n) + c.token + 1, 0), a.n_rows);
  return c;
}

// Over the two lanes (l, l ^ 32) that share a column.
template <class Op>
__device__ __forceinline__ float over_halves(float x, Op op) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return op(__uint_as_float(a[0]), __uint_as_float(a[1]));
}

// Over all lanes.
template <class Op>
__device__ __forceinline__ float over_wave(float x, float identity, Op op) {
  const auto bits = [=](uint32_t p, uint32_t q) { return __float_as_uint(op(__uint_as_float(p), __uint_as_float(q))); };
  return __uint_as_float(lane_value(wave_scan(__float_as_uint(x), __float_as_uint(identity), bits), kWave - 1));
}

// A column's operand of the first product: pieces 2 s + half of its query row.
template <int DT, int DH>
__device__ __forceinline__ void load_query(const PagedArgs &a, int b, const Column &c, bool valid, int half, u32x4_d (&qf)[Image<DT, DH>::STEPS]) {
#pragma unroll
  for (int s = 0; s < Image<DT, DH>::STEPS; ++s) {
    qf[s] = u32x4_d{0u, 0u, 0u, 0u};
    if (valid) qf[s] = *reinterpret_cast<const u32x4_d *>(a.q + b * a.qs[0] + c.h * a.qs[1] + c.token * a.qs[2] + (2 * s + half) * 16);
  }
}

// Eight (bf16) or four (f32) contraction indexes of each half of the wave.
template <int DT>
__device__ __forceinline__ void mma_piece(f32x16_p &acc, const u32x4_d &x, const u32x4_d &y) {
  if (DT == CKV_BF16) {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_p, x), __builtin_bit_cast(bf16x8_p, y), acc, 0, 0, 0);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(x[e]), __uint_as_float(y[e]), acc, 0, 0, 0);
  }
}

// First product of 32 rows of K: element r is the product of row block_row(r, half) with the lane's column (lane % 32).
__device__ __forceinline__ int block_row(int r, int half) { return 8 * (r / 4) + 4 * half + r % 4; }
// Bytes from an image of K to the lane's piece 0, and piece 2 s + half of its row: the permutation is an exclusive or of the piece's
// number, so a step is one of the address (images start at multiples of a row).
template <int DT, int DH>
__device__ __forceinline__ int k_lane(int lane) {
  typedef Image<DT, DH> I;
  return (lane & 31) * I::ROW + I::k_piece(lane & 31, lane >> 5) * 16;
}
__device__ __forceinline__ u32x4_d k_operand(const char *image, int at, int s) {
  return *reinterpret_cast<const u32x4_d *>(image + (at ^ (32 * s)));
}
template <int DT, int DH>
__device__ __forceinline__ void first_product(const char *image, int lane, const u32x4_d (&qf)[Image<DT, DH>::STEPS], f32x16_p &z) {
  const int at = k_lane<DT, DH>(lane);
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.0f;
#pragma unroll
  for (int s = 0; s < Image<DT, DH>::STEPS; ++s) mma_piece<DT>(z, k_operand(image, at, s), qf[s]);
}

// How a second sweep takes V's components: ones where there is an infinity of one sign or a NaN, or the finite ones only.
enum VMode { kUp, kDown, kFinite };
template <int DT>
__device__ __forceinline__ uint32_t v_word(uint32_t x, int mode) {
  if (DT == CKV_BF16) {
    uint32_t out = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t b = (x >> (16 * h)) & 0xffffu;
      const bool finite = (b & 0x7f80u) != 0x7f80u, nan = !finite && (b & 0x7fu);
      const bool marked = !finite && (nan || (mode == kUp) == !(b & 0x8000u));
      out |= (mode == kFinite ? (finite ? b : 0u) : (marked ? 0x3f80u : 0u)) << (16 * h);
    }
    return out;
  }
  const bool finite = (x & 0x7f800000u) != 0x7f800000u, nan = !finite && (x & 0x7fffffu);
  const bool marked = !finite && (nan || (mode == kUp) == !(x & 0x80000000u));
  return mode == kFinite ? (finite ? x : 0u) : (marked ? 0x3f800000u : 0u);
}

// Weights of a block as the second product takes them: in bf16 rounded to the type, to the nearest. For many columns that is all (2^-9 of each on
// average, of both signs, which over many rows is less than the output's own rounding); few columns, whose products wait for memory, take what the
// rounding leaves in a product more. us, one term / two: one token, kept rows of 16 sequences 10.2 / 10.7, over 32768 rows 84.3 / 84.5, five
// tokens over 9001 rows 29.1 / 30.5; many columns, where the matrix cores are the bound: 2048 tokens over 32768 rows 1005 / 1384, 4096 over
// themselves 259 / 338.
template <int DT>
struct Weights {
  u32x4_d piece[DT == CKV_BF16 ? 2 : 4];
};
template <int DT>
__device__ __forceinline__ Weights<DT> as_operand(const f32x16_p &w) {
  Weights<DT> out;
  if constexpr (DT == CKV_BF16) {
#pragma unroll
    for (int e = 0; e < 8; ++e) out.piece[e / 4][e % 4] = pack_bf16(w[2 * e], w[2 * e + 1]);
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) out.piece[e / 4][e % 4] = __float_as_uint(w[e]);
  }
  return out;
}

// What that rounding leaves of bf16 weights, rounded again: with it a weight is off by 2^-16 of itself.
__device__ __forceinline__ Weights<CKV_BF16> rest_of(const f32x16_p &w, const Weights<CKV_BF16> &first) {
  Weights<CKV_BF16> out;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t x = first.piece[e / 4][e % 4];
    out.piece[e / 4][e % 4] = pack_bf16(w[2 * e] - __uint_as_float(x << 16), w[2 * e + 1] - __uint_as_float(x & 0xffff0000u));
  }
  return out;
}

// The values are computed where this stands.
template <int DT>
__device__ __forceinline__ void pin(Weights<DT> &w, float &sum) {
#pragma unroll
  for (u32x4_d &piece : w.piece) asm volatile("" : "+v"(piece));
  asm volatile("" : "+v"(sum));
}

// V's operand in bf16, rows 16 j + 4 half + (0..3) and those eight further on, components 32 t + lane % 32: 16 lanes read four rows of 16
// components and get a component's four rows each. v_lane: the lane's bytes for t = 0, j = 0.
template <int DH>
__device__ __forceinline__ int v_lane(int lane) {
  typedef Image<CKV_BF16, DH> I;
  const int row = 4 * (lane >> 5) + (lane & 15) / 4, byte = 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
  return row * I::ROW + I::v_piece(row, byte / 16) * 16 + byte % 16;
}
template <int DH>
__device__ __forceinline__ u32x4_d v_operand(const char *image, int at, int t, int j) {
  constexpr int ROW = Image<CKV_BF16, DH>::ROW;
  const char *from = image + (at ^ (64 * t)) + 16 * j * ROW;
  const u32x2_p lo = read_transposed(from), hi = read_transposed(from + 8 * ROW);
  return u32x4_d{lo[0], lo[1], hi[0], hi[1]};
}
// Second product of 32 rows of V: component 32 t + block_row(r, half) of the lane's column is acc[t][r]. CAREFUL: V's components as `mode` says.
// rest: further terms of the weights, behind the first one, which leaves time to make them.
template <int DT, int DH, bool CAREFUL, class... Rest>
__device__ __forceinline__ void second_product(const char *image, int lane, const Weights<DT> &w, f32x16_p (&acc)[DH / 32], int mode, const Rest &...rest) {
  typedef Image<DT, DH> I;
  if constexpr (DT == CKV_BF16) {
    const int at = v_lane<DH>(lane);
    u32x4_d x[2][I::DTILES];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int t = 0; t < I::DTILES; ++t) {
        x[j][t] = v_operand<DH>(image, at, t, j);
        if (CAREFUL)
#pragma unroll
          for (int e = 0; e < 4; ++e) x[j][t][e] = v_word<DT>(x[j][t][e], mode);
        mma_piece<DT>(acc[t], x[j][t], w.piece[j]);
      }
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int t = 0; t < I::DTILES; ++t) (mma_piece<DT>(acc[t], x[j][t], rest.piece[j]), ...);
  } else {
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int row = block_row(r, lane >> 5);
#pragma unroll
      for (int t = 0; t < I::DTILES; ++t) {
        uint32_t x = *reinterpret_cast<const uint32_t *>(image + row * I::ROW + (32 * t + (lane & 31)) * 4);
        if (CAREFUL) x = v_word<DT>(x, mode);
        acc[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(x), __uint_as_float(w.piece[r / 4][r % 4]), acc[t], 0, 0, 0);
      }
    }
  }
}

// Online softmax of a lane's column: the reference of its weights (log2 domain, common to both halves of the wave; -inf before the first
// row) and the sum of this half's weights. The reference moves only where a block's maximum outgrows it by kSlack (weights up to
// 2^kSlack: fp32 and bf16 keep their relative precision), which it hardly ever does behind the first blocks. Weights of that size times V may be
// beyond fp32 where their mean is not. Then there is a second sweep, and its reference lies above the maximum by so much that the weights of all
// rows add up to less than one.
constexpr float kSlack = 6.0f;
__device__ __forceinline__ float room_for(int rows) { return (float)(33 - __builtin_clz(rows | 1)); }  // log2, up, and one
struct Running {
  float top, ref, sum;  // the reference; ref: top, or 0 where that is -inf
  float keep;           // what the sums of V so far have still to be multiplied by
  bool moved;           // whether that is not one for some lane of the wave
};
__device__ __forceinline__ Running none_yet() { return Running{-INFINITY, 0.0f, 0.0f, 1.0f, false}; }
// ... by the maximum of this half's rows (of the products, not yet scaled). A branch that stays one: without the statement in it
// both sides are computed. above: how far the reference lies above the maximum then, and slack: how far it may lie below.
__device__ __forceinline__ void take_maximum(float mx, float scale2, Running &run, float slack = kSlack, float above = 0.0f) {
  mx = over_halves(mx, [](float x, float y) { return fmaxf(x, y); }) * scale2;
  if (__any(mx > run.top + slack)) {
    asm volatile("" ::: "memory");
    const float now = mx > run.top + slack ? mx + above : run.top;
    run.ref = now == -INFINITY ? 0.0f : now;
    run.keep = now == run.top ? 1.0f : __builtin_amdgcn_exp2f(run.top - run.ref);
    run.sum *= run.keep;
    run.top = now;
    run.moved = true;
  }
}
// Logits of a block to weights. CAREFUL: with a reference `room` above the maximum, and with a mode other than kFinite the weights become ones.
template <bool CAREFUL>
__device__ __forceinline__ void to_weights(f32x16_p &z, float scale2, Running &run, int mode, float room = 0.0f) {
  float mx = z[0];
#pragma unroll
  for (int r = 1; r < 16; ++r) mx = fmaxf(mx, z[r]);
  if (CAREFUL) take_maximum(mx, scale2, run, -room, room);
  else take_maximum(mx, scale2, run);
  float part[4];  // the block's own sum first: a long list has thousands of blocks
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const float seen = CAREFUL && z[r] != -INFINITY ? 1.0f : 0.0f;
    z[r] = __builtin_amdgcn_exp2f(fmaf(z[r], scale2, -run.ref));
    part[r % 4] = r < 4 ? z[r] : part[r % 4] + z[r];
    if (CAREFUL && mode != kFinite) z[r] = seen;
  }
  run.sum += (part[0] + part[1]) + (part[2] + part[3]);
}

// The sums of V brought to the present reference.
template <int DTILES>
__device__ __forceinline__ void rescale(f32x16_p (&acc)[DTILES], Running &run) {
  if (run.moved) {
    asm volatile("" ::: "memory");
#pragma unroll
    for (int t = 0; t < DTILES; ++t) acc[t] *= run.keep;
    run.moved = false;
  }
}

// Whether a sweep has left something that is not finite, and what the sweeps over V's marks say of it.
template <int DTILES>
__device__ __forceinline__ bool not_finite(const f32x16_p (&acc)[DTILES]) {
  bool any = false;
#pragma unroll
  for (int t = 0; t < DTILES; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) any |= !(fabsf(acc[t][r]) < INFINITY);
  return any;
}
struct Marks {
  uint64_t up = 0, down = 0;  // bit 16 t + r
};
template <int DTILES>
__device__ __forceinline__ void take_marks(Marks &marks, f32x16_p (&acc)[DTILES], int mode) {
#pragma unroll
  for (int t = 0; t < DTILES; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const uint64_t bit = 1ull << (16 * t + r);
      if (mode == kUp) marks.up |= acc[t][r] > 0.0f ? bit : 0;
      else if (mode == kDown) marks.down |= acc[t][r] > 0.0f ? bit : 0;
      else if ((marks.up | marks.down) & bit) acc[t][r] += !(marks.up & bit) ? -INFINITY : !(marks.down & bit) ? INFINITY : NAN;
    }
}

// Partial results joined with weights that add up to one, so that nothing in between is larger than the largest part: what is infinite or NaN
// weighs in, however little its part weighs.
__device__ __forceinline__ f32x4_p add_part(f32x4_p num, const f32x4_p &x, float f) {
#pragma unroll
  for (int e = 0; e < 4; ++e) num[e] = fabsf(x[e]) < INFINITY ? fmaf(x[e], f, num[e]) : num[e] + x[e];
  return num;
}

// Four components of an output row.
template <int DT>
__device__ __forceinline__ void store_out(char *row, int d, const f32x4_p &x) {
  if (DT == CKV_BF16) *reinterpret_cast<uint2 *>(row + 2 * d) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
  else *reinterpret_cast<f32x4_p *>(row + 4 * d) = x;
}
__device__ __forceinline__ char *out_row(const PagedArgs &a, int b, const Column &c) {
  return a.out + b * a.os[0] + c.h * a.os[1] + c.token * a.os[2];
}
__device__ __forceinline__ float inverse_sum(float sum) { return sum == 0.0f ? 0.0f : 1.0f / sum; }
__device__ __forceinline__ void store_lse(const PagedArgs &a, int b, const Column &c, float top, float sum) {
  if (a.lse) a.lse[((size_t)b * a.Hq + c.h) * a.n + c.token] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * kLn2;
}

constexpr int kRowsCols = 32;  // columns of a tile of paged_rows_kernel
// Up to here it takes a call's columns, in tiles that read the same rows at the same time. bf16: two tiles (35 columns, 9k rows: 31.3 us with
// paged_tile_kernel, 30.5, 63 columns 33.2, 32.0; from three tiles on that one reads less). f32, where the products of the matrix cores take longer than the rows: their
// shares of the rows are what keeps the chip busy (200 columns, 1k rows 17.4 -> 13.1, 256, 2k 40 -> 34, 2048, 4k the other way round).
constexpr int kMostRowsCols = 64, kMostRowsColsF32 = 256;
// Columns of a call, and their product with the chunks, up to which a tile's chunks are joined in the launch that makes them: above, leaving and
// reading the sums past the caches takes one workgroup longer than a kernel of many behind this one takes with them. us, two launches / one: one
// token, 32/8 heads, 2000 rows 12.7 / 11.3 (4 x 8), batch 4, 32768 rows 86.0 / 84.5, 65000 rows 50.1 / 48.3 (4 x 32), 28/4 heads, batch 8,
// 9001 rows 26.9 / 25.7 (7 x 8); but with four tokens 29.4 / 30.6 (28 x 8), with five 30.5 / 32.4 (32 x 4), f32, 256 tokens, 2000 rows
// 33.9 / 38.8 (32 x 4). (A counter instead of the marks: 65000 rows 93, its 32 workgroups one behind the other.)
constexpr int kMostJoinedCols = 16;
constexpr int kMostJoined = 128;
void launch_paged_rows(const PagedArgs &a, bool bf16, int d, hipStream_t stream);

}  // namespace ckv
#endif
